// Packed causal attention in plain 32-bit arithmetic (FFMA), forward and backward.
//
// 256 threads as 16 x 16 over a 64 x 64 score tile, four rows and four columns each: eight float4 from
// shared memory feed 64 FMAs (the FMA pipe, not shared memory, is the limit).  The 16 threads of a row
// are half a warp, so its softmax is four shuffles; P passes through shared memory into the second
// product, whose 64 x D tile the threads share as four rows by D / 16 columns.
//
// 8 sequences of 600..700 tokens, 16 heads over 4, 128 columns: forward 0.57 ms (24.6 TFLOP/s counted; a causal tile's
// masked half included about 30), backward 2.2 ms (16 TFLOP/s, with seven products for the five counted).
#include "nat_attn.cuh"

namespace nat {
namespace attn {
namespace {

constexpr int kT = 64;         // tokens of a tile, queries and keys alike
constexpr int kThreads = 256;
constexpr int kLd = kT + 4;    // leading dimension of a score tile

// Row-major tile of 64 rows; four floats of padding put eight neighbouring rows into different banks.
template <int DP>
struct Tile {
  static constexpr int kLead = DP + 4, kFloats = kT * kLead;
  float* at;
  __device__ __forceinline__ float4 get(int r, int c) const {
    return *reinterpret_cast<const float4*>(at + r * kLead + c);
  }
  // Rows [lo, lo + 64) of one head, zero outside [lo, hi) and past D.
  __device__ __forceinline__ void load(const float* base, int64_t stride, int head, int D, int lo, int hi) {
#pragma unroll
    for (int i = 0; i < kT * DP / 4 / kThreads; ++i) {
      const int k = threadIdx.x + i * kThreads, r = k / (DP / 4), c = k % (DP / 4) * 4;
      const bool in = lo + r < hi && c < D;
      const float* src = in ? base + (int64_t)(lo + r) * stride + (int64_t)head * D + c : base;
      // asynchronous, so that the tiles of a step come together; zero bytes read is zeros written
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                       (uint32_t)__cvta_generic_to_shared(at + r * kLead + c)),
                   "l"(src), "r"(in ? 16 : 0)
                   : "memory");
    }
  }
};

// The tiles that were asked for are there, for all threads.
__device__ __forceinline__ void tiles_ready() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
}

// s[i][j] = row (ty + 16 i) of a . row (tx + 16 j) of b
template <int DP>
__device__ __forceinline__ void dots(const Tile<DP>& a, const Tile<DP>& b, int ty, int tx, float (&s)[4][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
  for (int c = 0; c < DP; c += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a.get(ty + 16 * i, c);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = b.get(tx + 16 * j, c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s[i][j] = fmaf(x[i].x, y[j].x, fmaf(x[i].y, y[j].y, fmaf(x[i].z, y[j].z, fmaf(x[i].w, y[j].w, s[i][j]))));
  }
}

// acc[i][.] += sum_k w[ty + 16 i][k] m[k][.] over the thread's columns tx 4 + 64 n.  With `masked` only the k
// in [first, last] of each row count: a weight of zero would not hide an infinity behind it.
template <int DP, bool MASKED>
__device__ __forceinline__ void accumulate(const float* w, const Tile<DP>& m, int ty, int tx, const int (&first)[4],
                                           const int (&last)[4], float (&acc)[4][DP / 16]) {
#pragma unroll 2
  for (int k = 0; k < kT; k += 4) {
    float4 p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const float4*>(w + (ty + 16 * i) * kLd + k);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      float y[DP / 16];
#pragma unroll
      for (int n = 0; n < DP / 64; ++n) {
        const float4 v = m.get(k + kk, tx * 4 + 64 * n);
        y[4 * n] = v.x; y[4 * n + 1] = v.y; y[4 * n + 2] = v.z; y[4 * n + 3] = v.w;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = kk == 0 ? p[i].x : kk == 1 ? p[i].y : kk == 2 ? p[i].z : p[i].w;
        if (!MASKED || (k + kk >= first[i] && k + kk <= last[i])) {
#pragma unroll
          for (int c = 0; c < DP / 16; ++c) acc[i][c] = fmaf(f, y[c], acc[i][c]);
        }
      }
    }
  }
}

template <int DP>
__device__ __forceinline__ void store_row(float* row, int D, int tx, const float (&acc)[DP / 16], float f) {
#pragma unroll
  for (int n = 0; n < DP / 64; ++n) {
    const int c = tx * 4 + 64 * n;
    if (c < D)
      *reinterpret_cast<float4*>(row + c) =
          make_float4(acc[4 * n] * f, acc[4 * n + 1] * f, acc[4 * n + 2] * f, acc[4 * n + 3] * f);
  }
}

struct Ptrs {
  const float *q, *k, *v, *out, *dout;
  float *o, *dq, *dk, *dv, *lse, *delta;
  nat_attn_params p;
};

__device__ __forceinline__ float sum16(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o, 16);
  return x;
}

// Every block takes its tile from the list or, without one, finds it; then the first one reports what is wrong
// with the batch.
__device__ __forceinline__ bool my_tile(const Batch& batch, const Entry* list, Head* head, Entry* e) {
  if (list) {
    const bool there = blockIdx.x < head->count[kPlanFwd];
    if (there) *e = list[blockIdx.x];
    return there;
  }
  uint32_t total, status;
  *e = find_entry(batch, blockIdx.x, &total, &status);
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) head->status = status;
  return blockIdx.x < total;
}

template <int DP>
__global__ void __launch_bounds__(kThreads) f32_fwd_kernel(Ptrs a, Batch batch, const Entry* list, Head* head) {
  extern __shared__ __align__(16) float smem[];
  Entry e;
  if (!my_tile(batch, list, head, &e)) return;
  Tile<DP> Q{smem}, K{smem + Tile<DP>::kFloats}, V{smem + 2 * Tile<DP>::kFloats};
  float* P = smem + 3 * Tile<DP>::kFloats;
  const int D = a.p.head_dim, h = blockIdx.y, kh = h / (a.p.n_heads / a.p.n_kv_heads);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  Q.load(a.q, a.p.q_stride, h, D, e.lo, e.seq_hi);
  float m[4], l[4], acc[4][DP / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) acc[i][c] = 0.f;
  }
  const int end = min(e.lo + kT, e.seq_hi), none[4] = {0, 0, 0, 0};
  for (int k0 = e.seq_lo; k0 < end; k0 += kT) {
    __syncthreads();
    K.load(a.k, a.p.k_stride, kh, D, k0, end);
    V.load(a.v, a.p.v_stride, kh, D, k0, end);
    tiles_ready();
    float s[4][4];
    dots<DP>(Q, K, ty, tx, s);
    int last[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      last[i] = e.lo + ty + 16 * i - k0;
      float top = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = tx + 16 * j <= last[i] ? s[i][j] * a.p.scale : -INFINITY;
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o, 16));
      const float base = top == -INFINITY ? 0.f : top;  // every score so far is minus infinity
      const float keep = expf(m[i] - base);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = expf(s[i][j] - base);
        sum += p;
        P[(ty + 16 * i) * kLd + tx + 16 * j] = p;
      }
      l[i] = fmaf(l[i], keep, sum16(sum));
      m[i] = top;
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) acc[i][c] *= keep;
    }
    __syncwarp();  // a row's P is written and read by one half warp
    if (k0 + kT > e.lo) accumulate<DP, true>(P, V, ty, tx, none, last, acc);
    else accumulate<DP, false>(P, V, ty, tx, none, last, acc);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = e.lo + ty + 16 * i;
    if (row >= e.seq_hi) continue;
    store_row<DP>(a.o + (int64_t)row * a.p.o_stride + (int64_t)h * D, D, tx, acc[i], 1.f / l[i]);
    if (tx == 0) a.lse[(int64_t)row * a.p.n_heads + h] = m[i] + logf(l[i]);
  }
}

// dq of 64 queries of a head; also leaves delta = do . o for the keys' kernel.
template <int DP>
__global__ void __launch_bounds__(kThreads) f32_dq_kernel(Ptrs a, Batch batch, const Entry* list, Head* head) {
  extern __shared__ __align__(16) float smem[];
  Entry e;
  if (!my_tile(batch, list, head, &e)) return;
  Tile<DP> Q{smem}, G{smem + Tile<DP>::kFloats}, K{smem + 2 * Tile<DP>::kFloats}, V{smem + 3 * Tile<DP>::kFloats};
  float* P = smem + 4 * Tile<DP>::kFloats;
  const int D = a.p.head_dim, h = blockIdx.y, kh = h / (a.p.n_heads / a.p.n_kv_heads);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  Q.load(a.q, a.p.q_stride, h, D, e.lo, e.seq_hi);
  G.load(a.dout, a.p.o_stride, h, D, e.lo, e.seq_hi);
  K.load(a.out, a.p.o_stride, h, D, e.lo, e.seq_hi);
  tiles_ready();
  float delta[4], lse[4], acc[4][DP / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = e.lo + ty + 16 * i;
    float d = 0.f;
#pragma unroll
    for (int n = 0; n < DP / 64; ++n) {
      const float4 x = G.get(ty + 16 * i, tx * 4 + 64 * n), y = K.get(ty + 16 * i, tx * 4 + 64 * n);
      d = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, d))));
    }
    delta[i] = sum16(d);
    const int64_t at = (int64_t)row * a.p.n_heads + h;
    lse[i] = row < e.seq_hi ? a.lse[at] : 0.f;
    if (row < e.seq_hi && tx == 0) a.delta[at] = delta[i];
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) acc[i][c] = 0.f;
  }
  const int end = min(e.lo + kT, e.seq_hi), none[4] = {0, 0, 0, 0};
  for (int k0 = e.seq_lo; k0 < end; k0 += kT) {
    __syncthreads();
    K.load(a.k, a.p.k_stride, kh, D, k0, end);
    V.load(a.v, a.p.v_stride, kh, D, k0, end);
    tiles_ready();
    float s[4][4], dp[4][4];
    dots<DP>(Q, K, ty, tx, s);
    dots<DP>(G, V, ty, tx, dp);
    int last[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      last[i] = e.lo + ty + 16 * i - k0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        P[(ty + 16 * i) * kLd + tx + 16 * j] =
            tx + 16 * j <= last[i] ? expf(s[i][j] * a.p.scale - lse[i]) * (dp[i][j] - delta[i]) : 0.f;
    }
    __syncwarp();
    if (k0 + kT > e.lo) accumulate<DP, true>(P, K, ty, tx, none, last, acc);
    else accumulate<DP, false>(P, K, ty, tx, none, last, acc);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = e.lo + ty + 16 * i;
    if (row < e.seq_hi)
      store_row<DP>(a.dq + (int64_t)row * a.p.q_stride + (int64_t)h * D, D, tx, acc[i], a.p.scale);
  }
}

// dk and dv of 64 keys of a key head: all query heads of its group, all later queries, in order.
template <int DP>
__global__ void __launch_bounds__(kThreads) f32_dkv_kernel(Ptrs a, Batch batch, const Entry* list, Head* head) {
  extern __shared__ __align__(16) float smem[];
  Entry e;
  if (!my_tile(batch, list, head, &e)) return;
  Tile<DP> Q{smem}, G{smem + Tile<DP>::kFloats}, K{smem + 2 * Tile<DP>::kFloats}, V{smem + 3 * Tile<DP>::kFloats};
  float *P = smem + 4 * Tile<DP>::kFloats, *S = P + kT * kLd;
  const int D = a.p.head_dim, kh = blockIdx.y, group = a.p.n_heads / a.p.n_kv_heads;
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  K.load(a.k, a.p.k_stride, kh, D, e.lo, e.seq_hi);
  V.load(a.v, a.p.v_stride, kh, D, e.lo, e.seq_hi);
  float dk[4][DP / 16], dv[4][DP / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) dk[i][c] = dv[i][c] = 0.f;
  const int all[4] = {kT, kT, kT, kT};
  for (int h = kh * group; h < (kh + 1) * group; ++h)
    for (int q0 = e.lo; q0 < e.seq_hi; q0 += kT) {
      __syncthreads();
      Q.load(a.q, a.p.q_stride, h, D, q0, e.seq_hi);
      G.load(a.dout, a.p.o_stride, h, D, q0, e.seq_hi);
      float lse[4], delta[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = q0 + tx + 16 * j;
        const int64_t at = (int64_t)row * a.p.n_heads + h;
        lse[j] = row < e.seq_hi ? a.lse[at] : 0.f;
        delta[j] = row < e.seq_hi ? a.delta[at] : 0.f;
      }
      tiles_ready();
      float s[4][4], dp[4][4];
      dots<DP>(K, Q, ty, tx, s);
      dots<DP>(V, G, ty, tx, dp);
      int first[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        first[i] = e.lo + ty + 16 * i - q0;  // the key's own token is the first query that sees it
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = tx + 16 * j, at = (ty + 16 * i) * kLd + c;
          const bool seen = c >= first[i] && q0 + c < e.seq_hi;
          const float p = seen ? expf(s[i][j] * a.p.scale - lse[j]) : 0.f;
          P[at] = p;
          S[at] = seen ? p * (dp[i][j] - delta[j]) : 0.f;
        }
      }
      __syncwarp();
      if (q0 < e.lo + kT) {
        accumulate<DP, true>(P, G, ty, tx, first, all, dv);
        accumulate<DP, true>(S, Q, ty, tx, first, all, dk);
      } else {
        accumulate<DP, false>(P, G, ty, tx, first, all, dv);
        accumulate<DP, false>(S, Q, ty, tx, first, all, dk);
      }
    }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = e.lo + ty + 16 * i;
    if (key >= e.seq_hi) continue;
    store_row<DP>(a.dk + (int64_t)key * a.p.k_stride + (int64_t)kh * D, D, tx, dk[i], a.p.scale);
    store_row<DP>(a.dv + (int64_t)key * a.p.v_stride + (int64_t)kh * D, D, tx, dv[i], 1.f);
  }
}

Ptrs ptrs(const Args& a, const Layout& l) {
  Ptrs p{};
  p.q = (const float*)a.q; p.k = (const float*)a.k; p.v = (const float*)a.v; p.out = (const float*)a.out;
  p.dout = (const float*)a.dout; p.o = (float*)a.out; p.dq = (float*)a.dq; p.dk = (float*)a.dk;
  p.dv = (float*)a.dv; p.lse = a.lse; p.delta = delta(a, l); p.p = a.p;
  return p;
}

template <typename K>
int launch(K kernel, size_t smem, std::atomic<uint64_t>* allowed, const Device& dev, const Args& a, const Layout& l,
           int heads, const char* name) {
  int s = allow_smem(kernel, smem, dev, allowed);
  if (s != NAT_OK) return s;
  kernel<<<dim3((unsigned)l.entries[kPlanFwd], (unsigned)heads), kThreads, smem, a.stream>>>(
      ptrs(a, l), batch(a, l, kPlanFwd), l.listed ? entries(a, l, kPlanFwd) : nullptr, head(a));
  NAT_LAUNCH_CHECK(name);
  return NAT_OK;
}

// All three kernels have the same tiles, so the forward's list serves them all.
template <int DP>
int fwd(const Args& a, const Layout& l) {
  static std::atomic<uint64_t> allowed;
  Device dev;
  int s = device(&dev);
  if (s == NAT_OK && l.listed) s = launch_plan(a, l, kPlanFwd);
  if (s != NAT_OK) return s;
  const size_t smem = (3 * Tile<DP>::kFloats + kT * kLd) * sizeof(float);
  return launch(f32_fwd_kernel<DP>, smem, &allowed, dev, a, l, a.p.n_heads, "f32_fwd_kernel");
}

template <int DP>
int bwd(const Args& a, const Layout& l) {
  static std::atomic<uint64_t> allowed[2];
  Device dev;
  int s = device(&dev);
  if (s == NAT_OK && l.listed) s = launch_plan(a, l, kPlanFwd);
  if (s != NAT_OK) return s;
  const size_t smem = (4 * Tile<DP>::kFloats + kT * kLd) * sizeof(float);
  s = launch(f32_dq_kernel<DP>, smem, &allowed[0], dev, a, l, a.p.n_heads, "f32_dq_kernel");
  if (s != NAT_OK) return s;
  return launch(f32_dkv_kernel<DP>, smem + kT * kLd * sizeof(float), &allowed[1], dev, a, l, a.p.n_kv_heads,
                "f32_dkv_kernel");
}

}  // namespace

int f32_fwd(const Args& a, const Layout& l) {
  return a.p.head_dim <= 64 ? fwd<64>(a, l) : fwd<128>(a, l);
}
int f32_bwd(const Args& a, const Layout& l) {
  return a.p.head_dim <= 64 ? bwd<64>(a, l) : bwd<128>(a, l);
}

}  // namespace attn
}  // namespace nat
