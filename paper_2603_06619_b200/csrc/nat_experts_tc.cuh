// Tensor-core helpers that both kernels of the products grouped by expert share: tile geometry, loads, tensor maps.
#pragma once

#include <atomic>

#include "nat_experts.cuh"
#include "nat_tc.cuh"

namespace nat {
namespace experts {

constexpr int BM = 128, BK = 64;
constexpr int kBox = 64 * 64 * 2;  // bytes of a 64 x 64 box of an operand that is contiguous across the contraction

__device__ __forceinline__ uint32_t pack_bf16(uint32_t lo, uint32_t hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
  return *reinterpret_cast<uint32_t*>(&v);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline int encode(CUtensorMap* map, CUtensorMapDataType type, int dims, uintptr_t base, const cuuint64_t* size,
           const cuuint64_t* pitch, const cuuint32_t* box) {
  static std::atomic<EncodeTiledFn> cached{nullptr};
  EncodeTiledFn fn = cached.load(std::memory_order_relaxed);
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    NAT_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found));
    if (found != cudaDriverEntryPointSuccess || !p)
      return fail(NAT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    fn = reinterpret_cast<EncodeTiledFn>(p);
    cached.store(fn, std::memory_order_relaxed);
  }
  const cuuint32_t one[3] = {1, 1, 1};
  const CUresult r = fn(map, type, (cuuint32_t)dims, reinterpret_cast<void*>(base), size, pitch, box, one,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(NAT_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  return NAT_OK;
}

// Rows of a matrix [rows, cols] of bfloat16: boxes of 64 columns.
inline int map_rows(CUtensorMap* map, const void* base, int cols, int64_t rows, int64_t stride, int box_rows) {
  const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, pitch[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (uintptr_t)base, size, pitch, box);
}
// The experts' weights [E, n_out, n_in]: boxes of 64 columns by box_rows of one expert.
inline int map_weights(CUtensorMap* map, const nat_experts_params& p, const void* w, int box_rows) {
  const cuuint64_t size[3] = {(cuuint64_t)p.n_in, (cuuint64_t)p.n_out, (cuuint64_t)p.n_experts};
  const cuuint64_t pitch[2] = {(cuuint64_t)p.n_in * 2, (cuuint64_t)p.n_in * p.n_out * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, (uintptr_t)w, size, pitch, box);
}

int device_index(int* dev);  // of the current device, below 64

}  // namespace experts
}  // namespace nat
