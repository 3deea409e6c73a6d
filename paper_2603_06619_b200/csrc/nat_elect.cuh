// How one lane of a warp issues loads and MMAs with their operands in uniform registers.
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

namespace nat {
namespace tc {

// One lane of a converged warp.  Together with a warp index and a tensor-memory address that the
// compiler knows to be the same in all lanes (uniform()) this keeps the operands of the MMAs in
// uniform registers: moved there one by one they cost 75 cycles an MMA, more than its 64.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "elect.sync _|p, 0xffffffff;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(one));
  return one != 0;
}
template <typename T>
__device__ __forceinline__ T uniform(T x) {
  return __shfl_sync(0xFFFFFFFFu, x, 0);
}

}  // namespace tc
}  // namespace nat
