// Direct loads into LDS and the wait that orders them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w4a8 {

// Direct load of 16 bytes per active lane into LDS at dst + 16 * lane.
// Written as an instruction the compiler does not model: through the builtin
// it cannot tell a copy into one slot from reads of another, and waits for
// every outstanding load before reading LDS.  The copies are ordered by the
// explicit wait and barrier at the top of the stage that reads them.
// M0 is named as clobbered; nothing else in these kernels keeps a value in it.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_dma16(const uint8_t *src, const void *dst) {
  const uint32_t m0 =
      (uint32_t)(uintptr_t)(const void __attribute__((address_space(3))) *)dst;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(src), "s"(m0)
               : "memory", "m0");
}
// The same from a scalar base and a 32-bit offset of the lane.
__device__ __forceinline__ void lds_dma16(const uint8_t *base, uint32_t off, const void *dst) {
  const uint32_t m0 =
      (uint32_t)(uintptr_t)(const void __attribute__((address_space(3))) *)dst;
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(m0)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// All but this wave's youngest N vector memory operations are done, its LDS
// reads too, and so for every other wave of the workgroup.
template <int N>
__device__ __forceinline__ void wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

}  // namespace w4a8
