// 8-bit activation checkpoints of packed rows: store (quantise) and load.
//
// Bound by HBM: a bfloat16 element moves 2 + 1 + 4/128 bytes either way (166,001 rows of 4096, stored and
// loaded: 716 us, 5.74 TB/s, 0.88 of the measured copy bandwidth).  Half a warp owns a
// group of 128 columns (one 16-byte load a lane), so a group's largest magnitude is four
// shuffles away and no shared memory is used.
#include "nat_common.cuh"
#include "nat_rows.cuh"

namespace nat {
namespace {

using rows::kChunk;
using rows::kGroup;

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // groups in flight per half warp

// A block's 16 half warps cover `gx` neighbouring groups of 16 / gx rows; gx is the power of two
// (at most 16) that covers a row's groups, so that narrow rows leave few lanes idle.
struct Shape {
  int64_t d;
  int groups, gx_log2;
};

template <typename T, bool LOAD>
__global__ void __launch_bounds__(kThreads)
ckpt8_kernel(const T* __restrict__ src, T* __restrict__ dst, int8_t* __restrict__ codes,
             float* __restrict__ scales, Shape s, const int32_t* __restrict__ n_rows, int64_t cap) {
  const int64_t n = n_rows ? min((int64_t)max(*n_rows, 0), cap) : cap;
  const int half = threadIdx.x >> 4, lane = threadIdx.x & 15;
  const int gx = 1 << s.gx_log2, ry = (kThreads / 16) >> s.gx_log2;
  const int g0 = blockIdx.y * gx + (half & (gx - 1));
  const int64_t col = (int64_t)g0 * kGroup + lane * kChunk;
  const bool in_row = col < s.d;  // all lanes stay for the shuffles
  const int64_t step = (int64_t)gridDim.x * ry;
  // the loop's bound is the block's, so that both halves of every warp take the same turns
  for (int64_t base = (int64_t)blockIdx.x * ry; base < n; base += step * kUnroll) {
    if (LOAD) {
      uint2 c[kUnroll];
      float sc[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t row = base + u * step + (half >> s.gx_log2);
        c[u] = make_uint2(0u, 0u);
        sc[u] = 0.f;
        if (in_row && row < n) {
          c[u] = __ldcs(reinterpret_cast<const uint2*>(codes + row * s.d + col));
          sc[u] = __ldg(scales + row * s.groups + g0);
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t row = base + u * step + (half >> s.gx_log2);
        if (in_row && row < n) {
          float2 x[rows::kPairs];
          rows::widen_codes(c[u], sc[u], x);
          rows::Raw<T> raw;
          rows::narrow(x, raw);
          rows::store_raw(dst + row * s.d + col, raw);
        }
      }
    } else {
      rows::Raw<T> raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t row = base + u * step + (half >> s.gx_log2);
        raw[u] = (in_row && row < n) ? rows::load_raw(src + row * s.d + col) : rows::zero_raw<T>();
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t row = base + u * step + (half >> s.gx_log2);
        float2 x[rows::kPairs];
        rows::widen(raw[u], x);
        const rows::GroupScale gs = rows::group_scale(rows::group_top(raw[u]));
        if (in_row && row < n) {
          __stcs(reinterpret_cast<uint2*>(codes + row * s.d + col), rows::group_codes(x, gs.inv));
          if (lane == 0) scales[row * s.groups + g0] = gs.scale;
        }
      }
    }
  }
}

int check(const char* who, int32_t dtype, int64_t d, int64_t cap, const void* x, const void* codes,
          const void* scales) {
  if (dtype != NAT_F32 && dtype != NAT_BF16)
    return fail(NAT_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
  if (d <= 0 || cap < 0 || cap > 0x7FFFFFFFll)
    return fail(NAT_ERR_INVALID_ARG, "%s: d must be positive and cap in [0, 2^31)", who);
  if (d % kChunk != 0 || d > (1 << 20))
    return fail(NAT_ERR_UNSUPPORTED, "%s: d must be a multiple of 8, at most 2^20 (d = %lld)", who,
                (long long)d);
  if (cap == 0) return NAT_OK;
  if (!x || !codes || !scales) return fail(NAT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (((uintptr_t)x | (uintptr_t)codes) & 15u)
    return fail(NAT_ERR_INVALID_ARG, "%s: rows and codes must be 16-byte aligned", who);
  if ((uintptr_t)scales & 3u)
    return fail(NAT_ERR_INVALID_ARG, "%s: scales must be 4-byte aligned", who);
  return NAT_OK;
}

template <typename T, bool LOAD>
int launch(const void* src, void* dst, int8_t* codes, float* scales, int64_t d,
           const int32_t* n_rows, int64_t cap, cudaStream_t stream) {
  Shape s;
  s.d = d;
  s.groups = (int)((d + kGroup - 1) / kGroup);
  s.gx_log2 = 0;
  while ((1 << s.gx_log2) < s.groups && s.gx_log2 < 4) ++s.gx_log2;
  const int gx = 1 << s.gx_log2, ry = (kThreads / 16) / gx;
  const int64_t col_blocks = (s.groups + gx - 1) / gx;
  // rows are dealt to at most eight waves of 148 x 8 blocks
  int64_t row_blocks = (cap + ry - 1) / ry;
  const int64_t most = max((int64_t)1, (int64_t)148 * 8 * 8 / col_blocks);
  if (row_blocks > most) row_blocks = most;
  ckpt8_kernel<T, LOAD><<<dim3((unsigned)row_blocks, (unsigned)col_blocks), kThreads, 0, stream>>>(
      (const T*)src, (T*)dst, codes, scales, s, n_rows, cap);
  NAT_LAUNCH_CHECK(LOAD ? "ckpt8_load" : "ckpt8_store");
  return NAT_OK;
}

}  // namespace
}  // namespace nat

extern "C" {

int nat_ckpt8_store(int32_t dtype, int64_t d, const void* src, const int32_t* n_rows, int64_t cap,
                    int8_t* codes, float* scales, void* stream) {
  const int s = nat::check("nat_ckpt8_store", dtype, d, cap, src, codes, scales);
  if (s != NAT_OK || cap == 0) return s;
  return dtype == NAT_F32
             ? nat::launch<float, false>(src, nullptr, codes, scales, d, n_rows, cap, (cudaStream_t)stream)
             : nat::launch<__nv_bfloat16, false>(src, nullptr, codes, scales, d, n_rows, cap,
                                                 (cudaStream_t)stream);
}

int nat_ckpt8_load(int32_t dtype, int64_t d, const int8_t* codes, const float* scales,
                   const int32_t* n_rows, int64_t cap, void* dst, void* stream) {
  const int s = nat::check("nat_ckpt8_load", dtype, d, cap, dst, codes, scales);
  if (s != NAT_OK || cap == 0) return s;
  int8_t* c = const_cast<int8_t*>(codes);
  float* sc = const_cast<float*>(scales);
  return dtype == NAT_F32
             ? nat::launch<float, true>(nullptr, dst, c, sc, d, n_rows, cap, (cudaStream_t)stream)
             : nat::launch<__nv_bfloat16, true>(nullptr, dst, c, sc, d, n_rows, cap,
                                                (cudaStream_t)stream);
}

}  // extern "C"
