// Packed causal attention in plain 32-bit arithmetic (FFMA), forward and backward.
//
// Four neighbouring threads share a row (a query; in the keys' kernel a key): each takes every
// fourth of 32 columns of the score tile and every fourth float4 of the head's columns, so the
// row's softmax is two shuffles and P passes through shared memory inside one warp only.
#include "nat_attn.cuh"

namespace nat {
namespace attn {
namespace {

constexpr int kT = 32;         // tokens of a tile, queries and keys alike
constexpr int kThreads = 128;  // four threads a row

// Rows [lo, lo + 32) of one head into shared memory, zero outside [lo, hi) and past D.
template <int DP>
__device__ __forceinline__ void load_tile(float (*dst)[DP + 4], const float* base, int64_t stride,
                                          int head, int D, int lo, int hi) {
  for (int i = threadIdx.x; i < kT * DP; i += kThreads) {
    const int r = i / DP, c = i % DP;
    dst[r][c] = (lo + r < hi && c < D) ? base[(int64_t)(lo + r) * stride + (int64_t)head * D + c] : 0.f;
  }
}

// s[j] = a-row . b-row (quad + 4 j)
template <int DP>
__device__ __forceinline__ void dots(const float* a, const float (*b)[DP + 4], int quad, float (&s)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = 0.f;
  for (int c = 0; c < DP; c += 4) {
    const float4 x = *reinterpret_cast<const float4*>(a + c);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float4 y = *reinterpret_cast<const float4*>(&b[quad + 4 * j][c]);
      s[j] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s[j]))));
    }
  }
}

// acc[.] += sum_k w[k] m[k][.] over the thread's float4 columns quad + 4 i.  Only the rows
// [first, last) that the mask leaves: a weight of zero would not hide an infinity behind it.
template <int DP>
__device__ __forceinline__ void accumulate(const float* w, const float (*m)[DP + 4], int first,
                                           int last, int quad, float (&acc)[DP / 4]) {
  for (int k = first; k < last; ++k) {
    const float p = w[k];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      const float4 y = *reinterpret_cast<const float4*>(&m[k][(quad + 4 * i) * 4]);
      acc[4 * i] = fmaf(p, y.x, acc[4 * i]);
      acc[4 * i + 1] = fmaf(p, y.y, acc[4 * i + 1]);
      acc[4 * i + 2] = fmaf(p, y.z, acc[4 * i + 2]);
      acc[4 * i + 3] = fmaf(p, y.w, acc[4 * i + 3]);
    }
  }
}

template <int DP>
__device__ __forceinline__ void store_row(float* row, int D, int quad, const float (&acc)[DP / 4], float f) {
#pragma unroll
  for (int i = 0; i < DP / 16; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = (quad + 4 * i) * 4 + j;
      if (c < D) row[c] = acc[4 * i + j] * f;
    }
}

struct Ptrs {
  const void *q, *k, *v, *out, *dout;
  void *o, *dq, *dk, *dv;
  float *lse, *delta;
  nat_attn_params p;
};

template <int DP>
__global__ void __launch_bounds__(kThreads)
f32_fwd_kernel(Ptrs a, Batch batch, Head* head) {
  extern __shared__ float smem[];
  uint32_t total;
  const Entry e = find_entry(batch, blockIdx.x, &total);  // by every warp for itself
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) head->status = batch_status(batch, total);
  if (blockIdx.x >= total) return;
  float(*Q)[DP + 4] = reinterpret_cast<float(*)[DP + 4]>(smem);
  float(*K)[DP + 4] = Q + kT;
  float(*V)[DP + 4] = K + kT;
  float(*P)[kT + 1] = reinterpret_cast<float(*)[kT + 1]>(V + kT);
  const int D = a.p.head_dim, h = blockIdx.y, kh = h / (a.p.n_heads / a.p.n_kv_heads);
  const int r = threadIdx.x >> 2, quad = threadIdx.x & 3, row = e.lo + r;
  load_tile<DP>(Q, (const float*)a.q, a.p.q_stride, h, D, e.lo, e.seq_hi);
  float m = -INFINITY, l = 0.f, acc[DP / 4];
#pragma unroll
  for (int i = 0; i < DP / 4; ++i) acc[i] = 0.f;
  const int last = min(e.lo + kT, e.seq_hi);
  for (int k0 = e.seq_lo; k0 < last; k0 += kT) {
    __syncthreads();
    load_tile<DP>(K, (const float*)a.k, a.p.k_stride, kh, D, k0, last);
    load_tile<DP>(V, (const float*)a.v, a.p.v_stride, kh, D, k0, last);
    __syncthreads();
    float s[8];
    dots<DP>(Q[r], K, quad, s);
    float top = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[j] = (k0 + quad + 4 * j <= row) ? s[j] * a.p.scale : -INFINITY;
      top = fmaxf(top, s[j]);
    }
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    const float base = top == -INFINITY ? 0.f : top;  // every score so far is minus infinity
    const float keep = expf(m - base);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = expf(s[j] - base);
      sum += p;
      P[r][quad + 4 * j] = p;
    }
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
    l = fmaf(l, keep, sum);
    m = top;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < DP / 4; ++i) acc[i] *= keep;
    accumulate<DP>(P[r], V, 0, min(kT, row - k0 + 1), quad, acc);
  }
  if (row < e.seq_hi) {
    store_row<DP>((float*)a.o + (int64_t)row * a.p.o_stride + (int64_t)h * D, D, quad, acc, 1.f / l);
    if (quad == 0) a.lse[(int64_t)row * a.p.n_heads + h] = m + logf(l);
  }
}

// dq of 32 queries of a head; also leaves delta = do . o for the keys' kernel.
template <int DP>
__global__ void __launch_bounds__(kThreads)
f32_dq_kernel(Ptrs a, Batch batch, Head* head) {
  extern __shared__ float smem[];
  uint32_t total;
  const Entry e = find_entry(batch, blockIdx.x, &total);  // by every warp for itself
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) head->status = batch_status(batch, total);
  if (blockIdx.x >= total) return;
  float(*Q)[DP + 4] = reinterpret_cast<float(*)[DP + 4]>(smem);
  float(*G)[DP + 4] = Q + kT;
  float(*K)[DP + 4] = G + kT;
  float(*V)[DP + 4] = K + kT;
  float(*P)[kT + 1] = reinterpret_cast<float(*)[kT + 1]>(V + kT);
  const int D = a.p.head_dim, h = blockIdx.y, kh = h / (a.p.n_heads / a.p.n_kv_heads);
  const int r = threadIdx.x >> 2, quad = threadIdx.x & 3, row = e.lo + r;
  load_tile<DP>(Q, (const float*)a.q, a.p.q_stride, h, D, e.lo, e.seq_hi);
  load_tile<DP>(G, (const float*)a.dout, a.p.o_stride, h, D, e.lo, e.seq_hi);
  load_tile<DP>(K, (const float*)a.out, a.p.o_stride, h, D, e.lo, e.seq_hi);
  __syncthreads();
  float delta = 0.f;
  for (int c = quad; c < DP; c += 4) delta = fmaf(G[r][c], K[r][c], delta);
  delta += __shfl_xor_sync(0xFFFFFFFFu, delta, 1);
  delta += __shfl_xor_sync(0xFFFFFFFFu, delta, 2);
  const int64_t at = (int64_t)row * a.p.n_heads + h;
  const float lse = row < e.seq_hi ? a.lse[at] : 0.f;
  if (row < e.seq_hi && quad == 0) a.delta[at] = delta;
  float acc[DP / 4];
#pragma unroll
  for (int i = 0; i < DP / 4; ++i) acc[i] = 0.f;
  const int last = min(e.lo + kT, e.seq_hi);
  for (int k0 = e.seq_lo; k0 < last; k0 += kT) {
    __syncthreads();
    load_tile<DP>(K, (const float*)a.k, a.p.k_stride, kh, D, k0, last);
    load_tile<DP>(V, (const float*)a.v, a.p.v_stride, kh, D, k0, last);
    __syncthreads();
    float s[8], dp[8];
    dots<DP>(Q[r], K, quad, s);
    dots<DP>(G[r], V, quad, dp);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool seen = k0 + quad + 4 * j <= row;
      P[r][quad + 4 * j] = seen ? expf(s[j] * a.p.scale - lse) * (dp[j] - delta) : 0.f;
    }
    __syncwarp();
    accumulate<DP>(P[r], K, 0, min(kT, row - k0 + 1), quad, acc);
  }
  if (row < e.seq_hi)
    store_row<DP>((float*)a.dq + (int64_t)row * a.p.q_stride + (int64_t)h * D, D, quad, acc, a.p.scale);
}

// dk and dv of 32 keys of a key head: all query heads of its group, all later queries, in order.
template <int DP>
__global__ void __launch_bounds__(kThreads)
f32_dkv_kernel(Ptrs a, Batch batch, Head* head) {
  extern __shared__ float smem[];
  uint32_t total;
  const Entry e = find_entry(batch, blockIdx.x, &total);  // by every warp for itself
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) head->status = batch_status(batch, total);
  if (blockIdx.x >= total) return;
  float(*Q)[DP + 4] = reinterpret_cast<float(*)[DP + 4]>(smem);
  float(*G)[DP + 4] = Q + kT;
  float(*K)[DP + 4] = G + kT;
  float(*V)[DP + 4] = K + kT;
  float(*P)[kT + 1] = reinterpret_cast<float(*)[kT + 1]>(V + kT);
  float(*S)[kT + 1] = P + kT;
  const int D = a.p.head_dim, kh = blockIdx.y, group = a.p.n_heads / a.p.n_kv_heads;
  const int r = threadIdx.x >> 2, quad = threadIdx.x & 3, key = e.lo + r;
  load_tile<DP>(K, (const float*)a.k, a.p.k_stride, kh, D, e.lo, e.seq_hi);
  load_tile<DP>(V, (const float*)a.v, a.p.v_stride, kh, D, e.lo, e.seq_hi);
  float dk[DP / 4], dv[DP / 4];
#pragma unroll
  for (int i = 0; i < DP / 4; ++i) dk[i] = dv[i] = 0.f;
  for (int h = kh * group; h < (kh + 1) * group; ++h)
    for (int q0 = e.lo; q0 < e.seq_hi; q0 += kT) {
      __syncthreads();
      load_tile<DP>(Q, (const float*)a.q, a.p.q_stride, h, D, q0, e.seq_hi);
      load_tile<DP>(G, (const float*)a.dout, a.p.o_stride, h, D, q0, e.seq_hi);
      __syncthreads();
      float s[8], dp[8];
      dots<DP>(K[r], Q, quad, s);
      dots<DP>(V[r], G, quad, dp);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = quad + 4 * j, row = q0 + i;
        float p = 0.f, ds = 0.f;
        if (row >= key && row < e.seq_hi) {
          const int64_t at = (int64_t)row * a.p.n_heads + h;
          p = expf(s[j] * a.p.scale - a.lse[at]);
          ds = p * (dp[j] - a.delta[at]);
        }
        P[r][i] = p;
        S[r][i] = ds;
      }
      __syncwarp();
      accumulate<DP>(P[r], G, max(0, key - q0), kT, quad, dv);
      accumulate<DP>(S[r], Q, max(0, key - q0), kT, quad, dk);
    }
  if (key < e.seq_hi) {
    store_row<DP>((float*)a.dk + (int64_t)key * a.p.k_stride + (int64_t)kh * D, D, quad, dk, a.p.scale);
    store_row<DP>((float*)a.dv + (int64_t)key * a.p.v_stride + (int64_t)kh * D, D, quad, dv, 1.f);
  }
}

Ptrs ptrs(const Args& a, const Layout& l) {
  Ptrs p{};
  p.q = a.q; p.k = a.k; p.v = a.v; p.out = a.out; p.dout = a.dout; p.o = a.out; p.dq = a.dq;
  p.dk = a.dk; p.dv = a.dv; p.lse = a.lse; p.delta = delta(a, l); p.p = a.p;
  return p;
}

template <typename K>
int launch(K kernel, size_t smem, const Args& a, const Layout& l, Plan which, int heads, const char* name) {
  NAT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  kernel<<<dim3((unsigned)l.entries[which], (unsigned)heads), kThreads, smem, a.stream>>>(
      ptrs(a, l), batch(a, l, which), head(a));
  NAT_LAUNCH_CHECK(name);
  return NAT_OK;
}

template <int DP>
int fwd(const Args& a, const Layout& l) {
  const size_t smem = (3 * kT * (DP + 4) + kT * (kT + 1)) * sizeof(float);
  return launch(f32_fwd_kernel<DP>, smem, a, l, kPlanFwd, a.p.n_heads, "f32_fwd_kernel");
}

template <int DP>
int bwd(const Args& a, const Layout& l) {
  const size_t smem = (4 * kT * (DP + 4) + 2 * kT * (kT + 1)) * sizeof(float);
  int s = launch(f32_dq_kernel<DP>, smem, a, l, kPlanDq, a.p.n_heads, "f32_dq_kernel");
  if (s != NAT_OK) return s;
  return launch(f32_dkv_kernel<DP>, smem, a, l, kPlanDkv, a.p.n_kv_heads, "f32_dkv_kernel");
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
