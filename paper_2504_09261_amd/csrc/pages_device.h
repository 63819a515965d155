// What the kernels over caches in pages share: lengths and page numbers as they find them in device memory.  HIP device code only.
#pragma once

#include "device_util.h"
#include "pages_internal.h"

namespace hack {
namespace dev {

// Loads through the scalar cache: tables and lengths do not change while a kernel runs.
typedef const __attribute__((address_space(4))) int32_t* ConstInts;
__device__ __forceinline__ ConstInts as_const(const int32_t* p) { return (ConstInts)(uintptr_t)p; }

__device__ __forceinline__ void report(const Pages& c) { __hip_atomic_store(c.fault, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM); }
// A number from memory, brought into [0, most]; raised says that it was not.
__device__ __forceinline__ int within(const Pages& c, int x, int most) {
  if (__builtin_expect((unsigned)x > (unsigned)most, 0)) {
    report(c);
    return x < 0 ? 0 : most;
  }
  return x;
}
__device__ __forceinline__ int rows_of(const Pages& c, int entry) { return within(c, c.len[entry], c.max_len); }
__device__ __forceinline__ int fresh_of(const Pages& c, int b) { return c.fresh ? within(c, c.fresh[b], c.n) : c.n; }

}  // namespace dev
}  // namespace hack
