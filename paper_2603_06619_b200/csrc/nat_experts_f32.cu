// Products grouped by expert in plain 32-bit arithmetic.
//
// 256 threads share a 128 x 128 tile of the result, eight rows by eight columns each, and go through the contraction 16
// at a time: the next slices of both operands are on their way in registers while the present ones, in shared
// memory with the contraction slowest, feed 64 multiply-adds a thread from four 16-byte reads.
#include "nat_experts.cuh"
#include "nat_f32x2.cuh"

namespace nat {
namespace experts {
namespace {

constexpr int kT = kF32Tile, kK = 16, kThreads = 256, kLd = kT + 4;

struct F32Args {
  const float *a, *b;
  float* c;
  int64_t a_stride, b_stride, c_stride;  // a matrix's row to the next
  int64_t b_expert, c_slice;             // an expert's matrix to the next
  int n_cols, k_size;                    // kFwd, kDx
  int m_size;                            // kDw: rows of the result
  int E, parts;
  bool accumulate;
  const int32_t* offsets;
  int64_t cap;
  Head* head;
};

// A slice [kK][kT] of an operand: rows or columns [o0, o_end) by [k0, k_end) of the contraction, zero outside.
// ALONG: the matrix is contiguous along the contraction.
template <bool ALONG>
struct Slice {
  float4 v[2];
  __device__ __forceinline__ void load(const float* m, int64_t stride, int o0, int o_end, int k0, int k_end) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int o = ALONG ? o0 + (int)threadIdx.x / 4 + 64 * i : o0 + (int)threadIdx.x % 32 * 4;
      const int k = ALONG ? k0 + (int)threadIdx.x % 4 * 4 : k0 + (int)threadIdx.x / 32 + 8 * i;
      // sizes along the contiguous dimension are multiples of four, so that four elements are in or out together
      const bool in = o < o_end && k < k_end;
      v[i] = in ? *reinterpret_cast<const float4*>(m + (ALONG ? (int64_t)o * stride + k : (int64_t)k * stride + o))
                : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ void put(float (*s)[kLd]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (ALONG) {
        const int o = threadIdx.x / 4 + 64 * i, k = threadIdx.x % 4 * 4;
        s[k][o] = v[i].x;
        s[k + 1][o] = v[i].y;
        s[k + 2][o] = v[i].z;
        s[k + 3][o] = v[i].w;
      } else {
        *reinterpret_cast<float4*>(&s[threadIdx.x / 32 + 8 * i][threadIdx.x % 32 * 4]) = v[i];
      }
    }
  }
};

// Tile number `index` of all row tiles in the experts' order, found by one warp (the same in every lane; empty where there
// are fewer), and what is wrong with the offsets.  A few hundred cycles for every 32 experts: less than a kernel
// in front that lists the tiles.
__device__ __forceinline__ Tile find_tile(const F32Args& g, int64_t index, unsigned* faults) {
  const int lane = threadIdx.x & 31;
  int64_t before = 0;
  Tile found{0, 0, 0, 0};
  *faults = 0u;
  for (int base = 0; base < g.E; base += 32) {
    const int e = base + lane;
    int lo = 0, hi = 0;
    unsigned fault = 0u;
    if (e < g.E) {
      expert_rows(g.offsets, e, g.cap, lo, hi);
      fault = offsets_fault(g.offsets, e, g.cap);
    }
    *faults |= __reduce_or_sync(0xFFFFFFFFu, fault);
    const int count = (hi - lo + kT - 1) / kT;
    int run = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int left = __shfl_up_sync(0xFFFFFFFFu, run, o);
      if (lane >= o) run += left;
    }
    const int64_t first = before + run - count;
    const unsigned who = __ballot_sync(0xFFFFFFFFu, index >= first && index < first + count);
    if (who) {
      const int from = __ffs(who) - 1;
      found.expert = base + from;
      found.lo = __shfl_sync(0xFFFFFFFFu, lo, from) + (int)(index - __shfl_sync(0xFFFFFFFFu, first, from)) * kT;
      found.hi = min(found.lo + kT, __shfl_sync(0xFFFFFFFFu, hi, from));
    }
    before += __shfl_sync(0xFFFFFFFFu, run, 31);
  }
  return found;
}

template <int WHICH>
__global__ void __launch_bounds__(kThreads) f32_kernel(const F32Args g) {
  __shared__ __align__(16) float sa[2][kK][kLd], sb[2][kK][kLd];
  __shared__ Tile shared_tile;
  __shared__ unsigned shared_faults;
  if (threadIdx.x < 32) {
    unsigned faults;
    const Tile t = find_tile(g, blockIdx.x, &faults);
    if (threadIdx.x == 0) {
      shared_tile = t;
      shared_faults = faults;
      if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) {
        g.head->status = faults ? NAT_DEV_CAPACITY : 0u;
        g.head->broken = (faults & kBroken) ? 1u : 0u;
      }
    }
  }
  __syncthreads();
  if (shared_faults & kBroken) return;
  int expert, m0, m_end, k0, k_end, slice = 0;
  const int n0 = blockIdx.y * kT;
  if (WHICH == kDw) {
    const int m_tiles = (g.m_size + kT - 1) / kT;
    expert = blockIdx.x / m_tiles;
    m0 = (blockIdx.x - expert * m_tiles) * kT;
    m_end = g.m_size;
    int lo, hi, b_lo, b_hi;
    expert_rows(g.offsets, expert, g.cap, lo, hi);
    part_range((hi - lo + kK - 1) / kK, blockIdx.z, g.parts, b_lo, b_hi);
    k0 = lo + b_lo * kK;
    k_end = min(lo + b_hi * kK, hi);
    slice = blockIdx.z * g.E + expert;
  } else {
    const Tile t = shared_tile;
    expert = t.expert;
    m0 = t.lo;
    m_end = t.hi;
    k0 = 0;
    k_end = g.k_size;
    if (m0 >= m_end) return;
  }
  const float* b = g.b + (WHICH == kDw ? 0 : expert * g.b_expert);
  Slice<WHICH != kDw> na;
  Slice<WHICH == kFwd> nb;
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  float2 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = both(0.f);
  na.load(g.a, g.a_stride, m0, m_end, k0, k_end);
  nb.load(b, g.b_stride, n0, g.n_cols, k0, k_end);
  int turn = 0;
  for (int k = k0; k < k_end; k += kK, turn ^= 1) {
    na.put(sa[turn]);
    nb.put(sb[turn]);
    __syncthreads();  // and the other buffers are free: all threads are past their last reads
    if (k + kK < k_end) {
      na.load(g.a, g.a_stride, m0, m_end, k + kK, k_end);
      nb.load(b, g.b_stride, n0, g.n_cols, k + kK, k_end);
    }
#pragma unroll
    for (int kk = 0; kk < kK; ++kk) {
      // a thread's rows and columns are two runs of four, 64 apart
      const float4 a0 = *reinterpret_cast<const float4*>(&sa[turn][kk][ty * 4]);
      const float4 a1 = *reinterpret_cast<const float4*>(&sa[turn][kk][64 + ty * 4]);
      const float4 b0 = *reinterpret_cast<const float4*>(&sb[turn][kk][tx * 4]);
      const float4 b1 = *reinterpret_cast<const float4*>(&sb[turn][kk][64 + tx * 4]);
      const float x[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
      const float2 y[4] = {make_float2(b0.x, b0.y), make_float2(b0.z, b0.w), make_float2(b1.x, b1.y),
                           make_float2(b1.z, b1.w)};
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fma2(both(x[i]), y[j], acc[i][j]);
    }
  }
  float* c = g.c + (int64_t)slice * g.c_slice;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = m0 + i / 4 * 64 + ty * 4 + i % 4;
    if (r >= m_end) continue;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int col = n0 + j * 64 + tx * 4;
      if (col >= g.n_cols) continue;
      float4* at = reinterpret_cast<float4*>(c + (int64_t)r * g.c_stride + col);
      float4 v = make_float4(acc[i][2 * j].x, acc[i][2 * j].y, acc[i][2 * j + 1].x, acc[i][2 * j + 1].y);
      if (WHICH == kDw && g.accumulate && g.parts == 1) {
        const float4 old = *at;
        v = make_float4(old.x + v.x, old.y + v.y, old.z + v.z, old.w + v.w);
      }
      *at = v;
    }
  }
}

}  // namespace

int f32_product(const Args& a, const Layout& l, Product which) {
  const nat_experts_params& p = a.p;
  F32Args g{};
  g.E = p.n_experts;
  g.parts = 1;
  g.offsets = a.offsets;
  g.cap = a.cap;
  g.head = head(a);
  g.accumulate = p.accumulate != 0;
  if (which == kDw) {
    g.a = (const float*)a.dy;
    g.b = (const float*)a.x;
    g.c = l.parts > 1 ? partial(a, l) : a.dw;
    g.a_stride = p.y_stride;
    g.b_stride = p.x_stride;
    g.c_stride = p.n_in;
    g.c_slice = (int64_t)p.n_in * p.n_out;
    g.n_cols = p.n_in;
    g.m_size = p.n_out;
    g.parts = l.parts;
    const dim3 grid((unsigned)(p.n_experts * ((p.n_out + kT - 1) / kT)), (unsigned)((p.n_in + kT - 1) / kT),
                    (unsigned)l.parts);
    f32_kernel<kDw><<<grid, kThreads, 0, a.stream>>>(g);
    NAT_LAUNCH_CHECK("experts_dw_f32");
    return NAT_OK;
  }
  const bool fwd = which == kFwd;
  g.a = (const float*)(fwd ? a.x : a.dy);
  g.b = (const float*)a.w;
  g.c = (float*)(fwd ? a.y : a.dx);
  g.a_stride = fwd ? p.x_stride : p.y_stride;
  g.b_stride = p.n_in;
  g.b_expert = (int64_t)p.n_in * p.n_out;
  g.c_stride = fwd ? p.y_stride : p.x_stride;
  g.n_cols = fwd ? p.n_out : p.n_in;
  g.k_size = fwd ? p.n_in : p.n_out;
  const dim3 grid((unsigned)l.most_tiles, (unsigned)((g.n_cols + kT - 1) / kT));
  if (fwd) f32_kernel<kFwd><<<grid, kThreads, 0, a.stream>>>(g);
  else f32_kernel<kDx><<<grid, kThreads, 0, a.stream>>>(g);
  NAT_LAUNCH_CHECK("experts_f32");
  return NAT_OK;
}

}  // namespace experts
}  // namespace nat
