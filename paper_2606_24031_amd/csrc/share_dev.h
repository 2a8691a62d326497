// Results that one workgroup of a launch hands to another.
//
// Workgroups may run on different XCDs, whose L2 caches do not see each
// other's ordinary stores.  What is handed over is written and read with the
// agent-scope bit, past those caches; fences that write back and drop whole
// caches cost 2 to 4 times the attention itself (48 rows over 6000 keys: 260
// us a call against 59 when that was measured).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w4a8 {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr int AGENT = 1 << 4;                    // sc1
typedef __amdgpu_buffer_rsrc_t Rsrc;
__device__ __forceinline__ Rsrc shared_at(void *p) {
  return __builtin_amdgcn_make_buffer_rsrc(p, 0, 0x7FFFFFFF, 0x00027000);
}
// `at` in floats.
__device__ __forceinline__ void share(Rsrc r, int at, v4f x) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, x), r, at * 4, 0, AGENT);
}
__device__ __forceinline__ void share(Rsrc r, int at, v2f x) {
  __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(v2u, x), r, at * 4, 0, AGENT);
}
__device__ __forceinline__ v4f shared4(Rsrc r, int at) {
  return __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(r, at * 4, 0, AGENT));
}
__device__ __forceinline__ v2f shared2(Rsrc r, int at) {
  return __builtin_bit_cast(v2f, __builtin_amdgcn_raw_buffer_load_b64(r, at * 4, 0, AGENT));
}

// Counts an arrival at *c; true in the last of n, which sets it back to 0.
// Every wave first waits for its stores, so whoever finds the count complete
// loads after all of them.
__device__ __forceinline__ bool last_of(int *c, int n, int *flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const int old = __hip_atomic_fetch_add(c, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = old == n - 1;
    if (old == n - 1) __hip_atomic_store(c, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return *flag;
}

}  // namespace w4a8
