// Tensor-core helpers of the packed attention beyond nat_tc.cuh: an A operand in tensor memory,
// tensor-memory stores, 3-D tile loads, and the operand tiles' geometry.
#pragma once

#include "nat_elect.cuh"
#include "nat_f32x2.cuh"
#include "nat_tc.cuh"

namespace nat {
namespace attn {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRows = 128;                          // rows of every operand tile
constexpr uint32_t kPanel = kRows * 128;            // 128 rows of 64 bfloat16 columns, 128-byte swizzle

// Descriptors of 128-byte-swizzled operand tiles, split in words: the upper word (stride offset
// 1024 bytes, version 1, swizzle mode 2) is the same for all, the lower one holds the address and
// the leading offset.  A step along the contraction is then one 32-bit addition: one thread
// issues every MMA, and building 64-bit descriptors for each would take it longer than the MMA.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);

// A tile whose contiguous columns are the contraction: step kk covers 16 of them.
__device__ __forceinline__ uint32_t desc_kmajor(uint32_t tile) { return (tile >> 4) | (1u << 16); }
constexpr __host__ __device__ uint32_t step_kmajor(int kk) {
  return (uint32_t)(kk >> 2) * (kPanel >> 4) + (uint32_t)(kk & 3) * 2u;
}
// A tile whose rows are the contraction: step kk covers 16 of them.
__device__ __forceinline__ uint32_t desc_mnmajor(uint32_t tile) {
  return (tile >> 4) | ((kPanel >> 4) << 16);
}
constexpr __host__ __device__ uint32_t step_mnmajor(int kk) { return (uint32_t)kk * (2048u >> 4); }

// D[tmem] (+)= A[smem] * B[smem]
__device__ __forceinline__ void umma_ss(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc,
                                        bool accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      ".reg .b64 a, b;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "mov.b64 a, {%1, %5};\n"
      "mov.b64 b, {%2, %5};\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n"
      "}\n" ::"r"(tmem_d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"((uint32_t)accumulate), "r"(kDescHi)
      : "memory");
}

// D[tmem] (+)= A[tmem] * B[smem], A of bf16 pairs packed along K into 32-bit columns.
__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t idesc,
                                        bool accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      ".reg .b64 b;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "mov.b64 b, {%2, %5};\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n"
      "}\n" ::"r"(tmem_d),
      "r"(tmem_a), "r"(b_lo), "r"(idesc), "r"((uint32_t)accumulate), "r"(kDescHi)
      : "memory");
}

// S[tmem] = A B^T of two tiles with D columns each (DP at most), of N rows of B.
template <int DP, int N = 128>
__device__ __forceinline__ void product_kk(uint32_t tmem_d, uint32_t a_tile, uint32_t b_tile, int ksteps) {
  constexpr uint32_t kIdesc = tc::instr_desc_bf16(128, N, 0, 0);
  const uint32_t a = desc_kmajor(a_tile), b = desc_kmajor(b_tile);
#pragma unroll
  for (int kk = 0; kk < DP / 16; ++kk)
    if (kk < ksteps) umma_ss(tmem_d, a + step_kmajor(kk), b + step_kmajor(kk), kIdesc, kk > 0);
}

// 32 consecutive 32-bit columns of this thread's lane; complete after tmem_st_wait().
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
      "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
      "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
      "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}

// 16 columns, complete on return.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}

// 64 columns, complete on return.
__device__ __forceinline__ void tmem_ld64(uint32_t addr, float (&x)[64]) {
  uint32_t r[64];
  tc::tmem_ld32_issue(addr, r);
  tc::tmem_ld32_issue(addr + 32, r + 32);
  tc::tmem_ld_wait(r);
  tc::tmem_ld_pin(r + 32);
#pragma unroll
  for (int c = 0; c < 64; ++c) x[c] = __uint_as_float(r[c]);
}

__device__ __forceinline__ void tmem_st_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tma_load_3d(uint32_t smem_dst, const CUtensorMap* map, uint64_t* bar,
                                            int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_dst),
      "l"(map), "r"(tc::smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// Whether every head's row of a tensor starts on a 32-byte boundary.
__device__ __forceinline__ bool wide_rows(const void* base, int64_t stride, int head_dim) {
  return (((uintptr_t)base | (uintptr_t)(stride * 2) | (uintptr_t)(head_dim * 2)) & 31u) == 0;
}

// 32 columns of a row, times f, rounded; columns at or after `left` are not there.  Each lane writes a
// row of its own, so the stores' cost is their number times 32 lines: 32 bytes at a time where
// the alignment allows.
__device__ __forceinline__ void store_row32(__nv_bfloat16* dst, const float* o, float f, int left, bool wide) {
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = bf16_pair(o[2 * i] * f, o[2 * i + 1] * f);
  if (wide) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (16 * i < left)
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + 16 * i), "r"(w[8 * i]),
                     "r"(w[8 * i + 1]), "r"(w[8 * i + 2]), "r"(w[8 * i + 3]), "r"(w[8 * i + 4]), "r"(w[8 * i + 5]),
                     "r"(w[8 * i + 6]), "r"(w[8 * i + 7])
                     : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * i < left)
        *reinterpret_cast<uint4*>(dst + 8 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}

// A wait of a whole warp: all lanes go on, or all give up.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
  return __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar, parity, abort_flag));
}

// Registers a thread of the calling warpgroup from here on; the shares of a block must add up to
// what it was launched with.
template <int N>
__device__ __forceinline__ void regs_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

using tc::elect_one;
using tc::uniform;

// Tensor map of [cap, heads, D] bfloat16 with a token stride: boxes of 64 columns x box_heads x
// box_tokens, zero outside.
int make_map(CUtensorMap* map, const void* base, int D, int heads, int64_t cap, int64_t stride,
             int box_heads, int box_tokens);

// Zeroes rows [first, 128) of a tile of NP panels that TMA has finished writing (one warp), for
// the tensor cores to read: the rows belong to another sequence, or to none, and a weight of
// zero would not hide an infinity or a NaN in them.
template <int NP>
__device__ __forceinline__ void zero_rows(uint8_t* tile, int first, int lane) {
  for (int i = lane; i < (kRows - first) * 8 * NP; i += 32) {
    const int panel = i / ((kRows - first) * 8), in = i % ((kRows - first) * 8);
    *reinterpret_cast<uint4*>(tile + panel * kPanel + first * 128 + in * 16) = make_uint4(0u, 0u, 0u, 0u);
  }
  tc::fence_proxy_async();
  __syncwarp();
}

}  // namespace attn
}  // namespace nat
