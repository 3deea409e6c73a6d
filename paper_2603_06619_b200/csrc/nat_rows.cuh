// Helpers of the packed-row operators (residual join, 8-bit checkpoints): eight consecutive
// elements of a row per thread, in 32 bits whatever the rows' type.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

namespace nat {
namespace rows {

constexpr int kChunk = 8;          // elements a thread moves at a time (16 bytes of bfloat16)
constexpr int kGroup = 128;        // columns that share a checkpoint scale: 16 chunks, half a warp
constexpr int kGroupLanes = kGroup / kChunk;

// Eight elements as they lie in memory: loads can be issued rows ahead without the registers
// their 32-bit values would take.
template <typename T>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
  uint4 v;
};
template <>
struct Raw<float> {
  float4 a, b;
};

__device__ __forceinline__ Raw<__nv_bfloat16> load_raw(const __nv_bfloat16* p) {
  return {__ldcs(reinterpret_cast<const uint4*>(p))};
}
__device__ __forceinline__ Raw<float> load_raw(const float* p) {
  return {__ldcs(reinterpret_cast<const float4*>(p)), __ldcs(reinterpret_cast<const float4*>(p) + 1)};
}
template <typename T>
__device__ __forceinline__ Raw<T> zero_raw();
template <>
__device__ __forceinline__ Raw<__nv_bfloat16> zero_raw<__nv_bfloat16>() {
  return {make_uint4(0u, 0u, 0u, 0u)};
}
template <>
__device__ __forceinline__ Raw<float> zero_raw<float>() {
  return {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
}

__device__ __forceinline__ void widen(const Raw<__nv_bfloat16>& r, float (&x)[kChunk]) {
  const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // a bfloat16 is the upper half of the float of the same value
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void widen(const Raw<float>& r, float (&x)[kChunk]) {
  x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w;
  x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// Rounds to the rows' type (once, to nearest even).
__device__ __forceinline__ void narrow(const float (&x)[kChunk], Raw<__nv_bfloat16>& r) {
  r.v = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                   pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ void narrow(const float (&x)[kChunk], Raw<float>& r) {
  r.a = make_float4(x[0], x[1], x[2], x[3]);
  r.b = make_float4(x[4], x[5], x[6], x[7]);
}

__device__ __forceinline__ void store_raw(__nv_bfloat16* p, const Raw<__nv_bfloat16>& r) {
  __stcs(reinterpret_cast<uint4*>(p), r.v);
}
__device__ __forceinline__ void store_raw(float* p, const Raw<float>& r) {
  __stcs(reinterpret_cast<float4*>(p), r.a);
  __stcs(reinterpret_cast<float4*>(p) + 1, r.b);
}

__device__ __forceinline__ void load_weights(const float* p, float (&w)[kChunk]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p));
  const float4 b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
}

// ---- 8-bit checkpoints ----------------------------------------------------------------
// A group of 128 columns holds codes q = round(x 127 / top) and one scale top / 127, top the
// group's largest magnitude: an even grid, so that an element is off by at most half a
// 127th of the largest magnitude beside it.  Two cases leave that rule: a group whose largest
// magnitude is below 2^-120 (127 / top would overflow) is stored as zeros, and a group that
// holds an infinity or a NaN is stored with a NaN scale, so that it reads back as NaN and not
// as plausible numbers.

// Largest magnitude among the 16 lanes of a group, as the bits of a float: the order of
// unsigned integers is that of non-negative floats, with NaN above infinity.
__device__ __forceinline__ uint32_t group_top(const float (&x)[kChunk]) {
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < kChunk; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
  for (int o = kGroupLanes / 2; o > 0; o >>= 1)
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o, kGroupLanes));
  return top;
}

struct GroupScale {
  float inv, scale;
};

__device__ __forceinline__ GroupScale group_scale(uint32_t top_bits) {
  const float top = __uint_as_float(top_bits);
  if (top_bits >= 0x7F800000u) return {0.f, __uint_as_float(0x7FC00000u)};
  if (top_bits < (7u << 23)) return {0.f, 0.f};  // below 2^(7 - 127)
  return {__fdiv_rn(127.f, top), __fdiv_rn(top, 127.f)};
}

// Codes of eight elements as eight bytes.  |x inv| <= 127 (1 + 2^-22), so adding 1.5 2^23
// leaves the nearest integer (ties to even) in the low mantissa bits; the product is rounded on its own
// (an FMA would break ties by its lost bits).
__device__ __forceinline__ uint2 group_codes(const float (&x)[kChunk], float inv) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < kChunk; ++i) {
    const float s = inv != 0.f ? __fmul_rn(x[i], inv) : 0.f;  // 0 * infinity would be a NaN
    const uint32_t q = __float_as_uint(__fadd_rn(s, 12582912.f)) & 0xFFu;
    w[i >> 2] |= q << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void widen_codes(uint2 c, float scale, float (&x)[kChunk]) {
#pragma unroll
  for (int i = 0; i < kChunk; ++i) {
    const uint32_t w = i < 4 ? c.x : c.y;
    x[i] = (float)(int8_t)(w >> (8 * (i & 3))) * scale;
  }
}

}  // namespace rows
}  // namespace nat
