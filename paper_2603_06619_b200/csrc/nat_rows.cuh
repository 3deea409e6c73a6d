// Helpers of the packed-row operators (residual join, 8-bit checkpoints): eight consecutive
// elements of a row per thread, in 32 bits whatever the rows' type.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "nat_f32x2.cuh"

namespace nat {
namespace rows {

constexpr int kPairs = 4;          // a chunk as pairs for packed arithmetic
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
// A thread's 32 bytes of floats go in one access where their address allows (rows are multiples of 32 bytes, so
// that is the same for all): in two of 16 each sector of L2 is asked for twice (the join of 14,648 float32 rows
// of 4096, forward: 250 us in halves, 219 whole).
__device__ __forceinline__ bool wide(const float* p) { return ((uintptr_t)p & 31u) == 0; }
__device__ __forceinline__ Raw<float> load_raw(const float* p) {
  if (wide(p)) {
    Raw<float> r;
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(r.a.x), "=f"(r.a.y), "=f"(r.a.z), "=f"(r.a.w), "=f"(r.b.x), "=f"(r.b.y), "=f"(r.b.z), "=f"(r.b.w)
                 : "l"(p));
    return r;
  }
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

__device__ __forceinline__ void widen(const Raw<__nv_bfloat16>& r, float2 (&x)[kPairs]) {
  const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
  for (int i = 0; i < kPairs; ++i)  // a bfloat16 is the upper half of the float of the same value
    x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ void widen(const Raw<float>& r, float2 (&x)[kPairs]) {
  x[0] = make_float2(r.a.x, r.a.y);
  x[1] = make_float2(r.a.z, r.a.w);
  x[2] = make_float2(r.b.x, r.b.y);
  x[3] = make_float2(r.b.z, r.b.w);
}

__device__ __forceinline__ uint32_t pack_bf16(float2 v) {
  __nv_bfloat162 p = __float22bfloat162_rn(v);
  return *reinterpret_cast<uint32_t*>(&p);
}

// Rounds to the rows' type (once, to nearest even).
__device__ __forceinline__ void narrow(const float2 (&x)[kPairs], Raw<__nv_bfloat16>& r) {
  r.v = make_uint4(pack_bf16(x[0]), pack_bf16(x[1]), pack_bf16(x[2]), pack_bf16(x[3]));
}
__device__ __forceinline__ void narrow(const float2 (&x)[kPairs], Raw<float>& r) {
  r.a = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
  r.b = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
}

__device__ __forceinline__ void store_raw(__nv_bfloat16* p, const Raw<__nv_bfloat16>& r) {
  __stcs(reinterpret_cast<uint4*>(p), r.v);
}
__device__ __forceinline__ void store_raw(float* p, const Raw<float>& r) {
  if (wide(p)) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(r.a.x), "f"(r.a.y),
                 "f"(r.a.z), "f"(r.a.w), "f"(r.b.x), "f"(r.b.y), "f"(r.b.z), "f"(r.b.w)
                 : "memory");
    return;
  }
  __stcs(reinterpret_cast<float4*>(p), r.a);
  __stcs(reinterpret_cast<float4*>(p) + 1, r.b);
}

// Asynchronous copies of a thread's own elements into its own slots of shared memory: rows are
// fetched ahead without registers, and as nobody else reads a slot no barrier is involved, only the
// thread's wait for its own copies.
template <int BYTES>
__device__ __forceinline__ void copy_async(void* smem, const void* src) {
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(smem);
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest `ahead` groups of copies have landed.
__device__ __forceinline__ void copies_wait(int ahead) {
  if (ahead >= 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// ---- 8-bit checkpoints ----------------------------------------------------------------
// A group of 128 columns holds codes q = round(x ((1 / top) 127)) and one scale top / 127, top the
// group's largest magnitude: an even grid, so that an element is off by at most half a
// 127th of the largest magnitude beside it.  Two cases leave that rule: a group whose largest
// magnitude is below 2^-120 (127 / top would overflow) is stored as zeros, and a group that
// holds an infinity or a NaN is stored with a NaN scale, so that it reads back as NaN and not
// as plausible numbers.

// Largest magnitude among the lanes of a group (16, or the row's where it is shorter), as the bits of a
// float: the order of unsigned integers is that of non-negative floats, with NaN above infinity.
template <int LANES = kGroupLanes>
__device__ __forceinline__ uint32_t group_top(const Raw<float>& r) {
  float2 x[kPairs];
  widen(r, x);
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < kPairs; ++i)
    top = max(top, max(__float_as_uint(x[i].x) & 0x7FFFFFFFu, __float_as_uint(x[i].y) & 0x7FFFFFFFu));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1)
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o, LANES));
  return top;
}
// Two bfloat16 at a time; a NaN wins.
template <int LANES = kGroupLanes>
__device__ __forceinline__ uint32_t group_top(const Raw<__nv_bfloat16>& r) {
  const uint32_t w[4] = {r.v.x & 0x7FFF7FFFu, r.v.y & 0x7FFF7FFFu, r.v.z & 0x7FFF7FFFu, r.v.w & 0x7FFF7FFFu};
  auto top2 = [](uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  };
  uint32_t top = top2(top2(w[0], w[1]), top2(w[2], w[3]));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1)
    top = top2(top, __shfl_xor_sync(0xFFFFFFFFu, top, o, LANES));
  return max(top << 16, top & 0xFFFF0000u);
}

struct GroupScale {
  float inv, scale;
};

__device__ __forceinline__ GroupScale group_scale(uint32_t top_bits) {
  const float top = __uint_as_float(top_bits);
  if (top_bits >= 0x7F800000u) return {0.f, __uint_as_float(0x7FC00000u)};
  if (top_bits < (7u << 23)) return {0.f, 0.f};  // below 2^(7 - 127)
  // top / 127 by Markstein's division: an FMA gives the exact remainder of the first quotient, which
  // the second FMA corrects to the rounded one
  constexpr float kInv = 1.f / 127.f;
  const float q = __fmul_rn(top, kInv);
  // 1 / top with the mantissa of top (in [1, 2)), so that no step leaves the normal range: the
  // approximate reciprocal, which one Newton step rounds correctly; then the factor and, exactly, the
  // power of two (127 / 2, so that the power stays normal).  The tests hold both quotients against float64 for
  // every mantissa, at 2^-120 (where the scale is subnormal), around 1 and at the largest exponents; between
  // those only the power differs.
  const float b = __uint_as_float((top_bits & 0x007FFFFFu) | 0x3F800000u);
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(b));
  y = __fmaf_rn(__fmaf_rn(-b, y, 1.f), y, y);
  const float power = __uint_as_float((255u << 23) - (top_bits & 0x7F800000u));
  return {__fmul_rn(__fmul_rn(63.5f, y), power), __fmaf_rn(__fmaf_rn(-q, 127.f, top), kInv, q)};
}

// Codes of eight elements as eight bytes.  |x inv| <= 127 (1 + 2^-22), so adding 1.5 2^23
// leaves the nearest integer (ties to even) in the low mantissa bits; the product is rounded on its own
// (an FMA would break ties by its lost bits).
__device__ __forceinline__ uint2 group_codes(const float2 (&x)[kPairs], float inv) {
  uint32_t q[kChunk];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {  // the packed forms are contracted to an FMA
    q[2 * i] = __float_as_uint(__fadd_rn(__fmul_rn(x[i].x, inv), 12582912.f));
    q[2 * i + 1] = __float_as_uint(__fadd_rn(__fmul_rn(x[i].y, inv), 12582912.f));
  }
  auto low_bytes = [&](int i) {
    return __byte_perm(__byte_perm(q[i], q[i + 1], 0x0040), __byte_perm(q[i + 2], q[i + 3], 0x0040), 0x5410);
  };
  if (inv == 0.f) return make_uint2(0u, 0u);  // zero times an infinity would be a NaN
  return make_uint2(low_bytes(0), low_bytes(4));
}

__device__ __forceinline__ void widen_codes(uint2 c, float scale, float2 (&x)[kPairs]) {
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const uint32_t w = (i < 2 ? c.x : c.y) >> (16 * (i & 1));
    x[i] = mul2(make_float2((float)(int8_t)w, (float)(int8_t)(w >> 8)), both(scale));
  }
}

}  // namespace rows
}  // namespace nat
