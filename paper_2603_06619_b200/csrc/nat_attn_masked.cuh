// What an infinity or a NaN behind the causal mask leaves in the products of the tensor cores, put right.
//
// A masked score gives the weight zero, and zero times an infinity is a NaN: through the tile on the diagonal one
// in v reaches out of tokens before it, and in the backward pass one in k, q or dout reaches dq, dk and dv in the
// same way.  Every thread looks whether its row of results is finite, a few packed instructions.  Where one
// was not, the block goes through its rows again once its pipeline is done (no role waits for another then, however
// long it takes): a row that is not finite although its softmax is, and in a column where the mask hides such
// values that the row's own tokens do not have, is added up anew from global memory without the masked terms, a
// thread a row.
//
// The look costs 10 of 595 us in 64 sequences of 256..2048 tokens (16 heads over 8, 128 columns), where a unit has four
// or five steps, and nothing measurable in longer ones.  A repair takes the latency of a thread's walk along its
// row: of 33,000 tokens, 8 heads over 2, forward 105 ms where it is 1.9, backward 640 ms where it is 5.9 at worst.
#pragma once

#include "nat_attn_tc.cuh"

namespace nat {
namespace attn {

// Zero, or NaN if one of the 32 is not finite.
__device__ __forceinline__ float2 finite32(const float* o, float2 z) {
  float2 y[4] = {z, both(0.f), both(0.f), both(0.f)};
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i & 3] = fma2(make_float2(o[2 * i], o[2 * i + 1]), both(0.f), y[i & 3]);
  return add2(add2(y[0], y[1]), add2(y[2], y[3]));
}
__device__ __forceinline__ bool is_finite(float2 z) { return z.x == 0.f && z.y == 0.f; }

// A head's rows in global memory, of tokens with a stride.
struct Rows {
  const __nv_bfloat16* base;
  int64_t stride;
  __device__ __forceinline__ const uint4* at(int token, int head, int D) const {
    return reinterpret_cast<const uint4*>(base + (int64_t)token * stride + (int64_t)head * D);
  }
};

__device__ __forceinline__ void widen8(uint4 v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ float row_dot(const uint4* a, const uint4* b, int D) {
  float s = 0.f;
#pragma unroll 4
  for (int c = 0; c < D / 8; ++c) {
    float x[8], y[8];
    widen8(a[c], x);
    widen8(b[c], y);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(x[i], y[i], s);
  }
  return s;
}

// acc += w row, the columns [8 first, 8 (first + n)) of it
template <int N>
__device__ __forceinline__ void row_add(float (&acc)[N], float w, const uint4* row, int first, int D) {
#pragma unroll
  for (int c = 0; c < N / 8; ++c)
    if ((first + c) * 8 < D) {
      float x[8];
      widen8(row[first + c], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[c * 8 + i] = fmaf(w, x[i], acc[c * 8 + i]);
    }
}

// Whether all of a row's results from column `first` on, up to `last`, are finite: bfloat16 as written by this block,
// or a piece's, N floats apart.
__device__ __forceinline__ bool finite_row(const __nv_bfloat16* row, int first, int last) {
  bool fine = true;
  for (int c = first; c < last; c += 8) {
    const uint4 v = __ldcg(reinterpret_cast<const uint4*>(row + c));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) fine = fine && (w[i] & 0x7F80u) != 0x7F80u && (w[i] & 0x7F800000u) != 0x7F800000u;
  }
  return fine;
}
template <int N>
__device__ __forceinline__ bool finite_piece(const float* slot, int first, int last) {
  float z = 0.f;
  for (int c = first; c < last; ++c) z = fmaf(__ldcg(slot + c * N), 0.f, z);
  return z == 0.f;
}

// The same rounding as that of P and dS on their way to the tensor cores.
__device__ __forceinline__ float as_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

// Whether some column is finite in all tokens [seen_lo, seen_hi) of the heads, and is not in those of
// [hidden_lo, hidden_hi).
__device__ __forceinline__ bool hidden_only(const Rows& r, int head, int heads, int D, int hidden_lo, int hidden_hi,
                                            int seen_lo, int seen_hi) {
  for (int c = 0; c < D / 8; ++c) {
    auto odd = [&](int lo, int hi) {  // bit i: column i of the eight holds an infinity or a NaN
      uint32_t m = 0u;
      for (int t = lo; t < hi; ++t)
        for (int h = head; h < head + heads; ++h) {
          const uint4 v = r.at(t, h, D)[c];
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            m |= (w[i] & 0x7F80u) == 0x7F80u ? 1u << (2 * i) : 0u;
            m |= (w[i] & 0x7F800000u) == 0x7F800000u ? 2u << (2 * i) : 0u;
          }
        }
      return m;
    };
    const uint32_t hidden = odd(hidden_lo, hidden_hi);
    if (hidden && (hidden & ~odd(seen_lo, seen_hi))) return true;
  }
  return false;
}

}  // namespace attn
}  // namespace nat
