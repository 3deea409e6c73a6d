// Products grouped by expert in plain 32-bit arithmetic.
//
// 256 threads share a T x T tile of the result, R x R elements each (T = 16 R), and go through the contraction 16 at a
// time, three slices of both operands ahead by asynchronous copies; four steps of the contraction are 2 R reads of
// 16 bytes for 2 R^2 packed multiply-adds.  T = 128, or 64 for small problems, which wait for memory rather than
// compute.  8000 rows over four experts, 1024 x 1024: forward 453 us (37 TFLOP/s of 74), the rows' gradient 413, the weights'
// 426.
#include <atomic>

#include "nat_experts.cuh"
#include "nat_f32x2.cuh"

namespace nat {
namespace experts {
namespace {

constexpr int kK = 16, kThreads = 256, kStages = 4;

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

// Slices of an operand on their way: T rows or columns of the result by kK of the contraction, zero outside
// [o0, o_end) and [k0, k_end).  ALONG: the matrix, and the slice, are contiguous along the contraction.
template <bool ALONG, int R>
struct Operand {
  static constexpr int T = 16 * R, kLd = (ALONG ? kK : T) + 4, kFloats = (ALONG ? T : kK) * kLd;
  float* at;
  const float* m;
  int64_t stride;
  int o0, o_end, k_end;
  __device__ __forceinline__ void fetch(int stage, int k0) const {
#pragma unroll
    for (int i = 0; i < R / 4; ++i) {
      const int c = threadIdx.x + i * kThreads;  // chunk of four
      const int r = ALONG ? c / (kK / 4) : c / (T / 4), q = (ALONG ? c % (kK / 4) : c % (T / 4)) * 4;
      const int o = o0 + (ALONG ? r : q), k = k0 + (ALONG ? q : r);
      // sizes along the contiguous dimension are multiples of four, so that four elements are in or out together
      const bool in = o < o_end && k < k_end;
      const float* src = in ? m + (ALONG ? (int64_t)o * stride + k : (int64_t)k * stride + o) : m;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                       (uint32_t)__cvta_generic_to_shared(at + stage * kFloats + r * kLd + q)),
                   "l"(src), "r"(in ? 16 : 0)
                   : "memory");
    }
  }
  // v[j][i]: step j of four from kk on, element i of the thread's R (runs of four, 64 apart), t its place among 16
  __device__ __forceinline__ void get(int stage, int kk, int t, float (&v)[4][R]) const {
    const float* s = at + stage * kFloats;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (ALONG) {
        const float4 x = *reinterpret_cast<const float4*>(s + (i / 4 * 64 + i % 4 * 16 + t) * kLd + kk);
        v[0][i] = x.x; v[1][i] = x.y; v[2][i] = x.z; v[3][i] = x.w;
      } else if (i % 4 == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float4 x = *reinterpret_cast<const float4*>(s + (kk + j) * kLd + i / 4 * 64 + t * 4);
          v[j][i] = x.x; v[j][i + 1] = x.y; v[j][i + 2] = x.z; v[j][i + 3] = x.w;
        }
      }
    }
  }
  // the place in the tile of the thread's element i
  static __device__ __forceinline__ int place(int i, int t) { return ALONG ? i / 4 * 64 + i % 4 * 16 + t : i / 4 * 64 + t * 4 + i % 4; }
};

// Tile number `index` of all row tiles in the experts' order, found by one warp (the same in every lane; empty where there
// are fewer), and what is wrong with the offsets.  A few hundred cycles for every 32 experts: less than a kernel
// in front that lists the tiles.
__device__ __forceinline__ Tile find_tile(const F32Args& g, int64_t index, int tile_rows, unsigned* faults) {
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
    const int count = (hi - lo + tile_rows - 1) / tile_rows;
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
      found.lo = __shfl_sync(0xFFFFFFFFu, lo, from) + (int)(index - __shfl_sync(0xFFFFFFFFu, first, from)) * tile_rows;
      found.hi = min(found.lo + tile_rows, __shfl_sync(0xFFFFFFFFu, hi, from));
    }
    before += __shfl_sync(0xFFFFFFFFu, run, 31);
  }
  return found;
}

template <int WHICH, int R>
__global__ void __launch_bounds__(kThreads) f32_kernel(const F32Args g) {
  using A = Operand<WHICH != kDw, R>;
  using B = Operand<WHICH == kFwd, R>;
  constexpr int kT = A::T;
  extern __shared__ __align__(16) float smem[];
  __shared__ Tile shared_tile;
  __shared__ unsigned shared_faults;
  if (threadIdx.x < 32) {
    unsigned faults;
    const Tile t = find_tile(g, blockIdx.x, kT, &faults);
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
  const A oa{smem, g.a, g.a_stride, m0, m_end, k_end};
  const B ob{smem + kStages * A::kFloats, g.b + (WHICH == kDw ? 0 : expert * g.b_expert), g.b_stride, n0, g.n_cols, k_end};
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  // kFwd: a pair is the sums over even and odd steps, neighbours in registers as they come (453 us; neighbouring columns,
  // which have to be brought together, 471); elsewhere it is two neighbouring columns
  constexpr int kCols = WHICH == kFwd ? R : R / 2;
  float2 acc[R][kCols];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < kCols; ++j) acc[i][j] = both(0.f);
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    if (k0 + i * kK < k_end) {
      oa.fetch(i, k0 + i * kK);
      ob.fetch(i, k0 + i * kK);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  int stage = 0;
  for (int k = k0; k < k_end; k += kK) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncthreads();  // the slice is there for all, and all are done with the one that the next copies replace
    const int ahead = k + (kStages - 1) * kK, to = stage == 0 ? kStages - 1 : stage - 1;
    if (ahead < k_end) {
      oa.fetch(to, ahead);
      ob.fetch(to, ahead);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
    for (int kk = 0; kk < kK; kk += 4) {
      float x[4][R], y[4][R];
      oa.get(stage, kk, ty, x);
      ob.get(stage, kk, tx, y);
#pragma unroll
      for (int j = 0; j < 4; j += WHICH == kFwd ? 2 : 1)
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            if (WHICH == kFwd)
              acc[i][c] = fma2(make_float2(x[j][i], x[j + 1][i]), make_float2(y[j][c], y[j + 1][c]), acc[i][c]);
            else
              acc[i][c] = fma2(both(x[j][i]), make_float2(y[j][2 * c], y[j][2 * c + 1]), acc[i][c]);
          }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  float* c = g.c + (int64_t)slice * g.c_slice;
  const bool add = WHICH == kDw && g.accumulate && g.parts == 1;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = m0 + A::place(i, ty);
    if (r >= m_end) continue;
    float* row = c + (int64_t)r * g.c_stride;
#pragma unroll
    for (int j = 0; j < R; j += 4) {
      if (WHICH == kFwd) {  // a thread's columns are 16 apart
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = n0 + B::place(j + e, tx);
          if (col < g.n_cols) row[col] = acc[i][(j + e) % kCols].x + acc[i][(j + e) % kCols].y;
        }
      } else {
        const float v[4] = {acc[i][j / 2].x, acc[i][j / 2].y, acc[i][j / 2 + 1].x, acc[i][j / 2 + 1].y};
        const int col = n0 + B::place(j, tx);
        if (col >= g.n_cols) continue;
        float4* at = reinterpret_cast<float4*>(row + col);
        const float4 old = add ? *at : make_float4(0.f, 0.f, 0.f, 0.f);
        *at = add ? make_float4(old.x + v[0], old.y + v[1], old.z + v[2], old.w + v[3]) : make_float4(v[0], v[1], v[2], v[3]);
      }
    }
  }
}

template <int WHICH, int R>
int launch(const F32Args& g, int64_t m_tiles, cudaStream_t stream) {
  constexpr size_t smem = kStages * (Operand<WHICH != kDw, R>::kFloats + Operand<WHICH == kFwd, R>::kFloats) * sizeof(float);
  static std::atomic<uint64_t> allowed{0};  // a bit for each device whose shared-memory limit is raised
  int dev = 0;
  NAT_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return fail(NAT_ERR_UNSUPPORTED, "device index %d is beyond the 64 this library tracks", dev);
  if (smem > 48 * 1024 && !(allowed.load(std::memory_order_relaxed) >> dev & 1u)) {
    NAT_CUDA(cudaFuncSetAttribute(f32_kernel<WHICH, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  const dim3 grid((unsigned)m_tiles, (unsigned)((g.n_cols + 16 * R - 1) / (16 * R)), (unsigned)g.parts);
  f32_kernel<WHICH, R><<<grid, kThreads, smem, stream>>>(g);
  NAT_LAUNCH_CHECK("experts_f32");
  return NAT_OK;
}
template <int WHICH>
int launch(const F32Args& g, const Layout& l, int64_t m_tiles, cudaStream_t stream) {
  return l.tile_rows[WHICH] == 128 ? launch<WHICH, 8>(g, m_tiles, stream) : launch<WHICH, 4>(g, m_tiles, stream);
}

}  // namespace

int f32_tile(const nat_experts_params& p, Product which, int64_t cap) {
  // tiles of 64 where those of 128 would leave half of the multiprocessors idle: 508 rows over 16 experts, 408 x 112
  // forward 48 us with 128, 25 with 64; 2000 rows, 1024 x 1024 (128 tiles) 111, 191
  // where one would leave half of a tile of 128 empty: 27,802 rows, 248 x 64 forward 62 us with 128, 31 with 64
  const int narrow = which == kFwd ? p.n_out : which == kDx ? p.n_in : min(p.n_out, p.n_in);
  if (narrow <= 64) return 64;
  auto tiles = [](int64_t n) { return (n + 127) / 128; };
  const int64_t n = which == kDw ? p.n_experts * tiles(p.n_out) * tiles(p.n_in)
                                 : tiles(cap) * tiles(which == kFwd ? p.n_out : p.n_in);
  return n < 148 / 2 ? 64 : 128;
}

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
    return launch<kDw>(g, l, p.n_experts * ((p.n_out + l.tile_rows[kDw] - 1) / l.tile_rows[kDw]), a.stream);
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
  const int64_t m_tiles = most_tiles(p, a.cap, l.tile_rows[which]);
  return fwd ? launch<kFwd>(g, l, m_tiles, a.stream) : launch<kDx>(g, l, m_tiles, a.stream);
}

}  // namespace experts
}  // namespace nat
