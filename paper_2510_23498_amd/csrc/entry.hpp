// What the C entry points of all translation units share: recording of HIP errors (rampde_strerror reports the thread's
// last one) and checks of arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/rampde.h"

namespace rampde {

__attribute__((visibility("hidden"))) int hip_fail(hipError_t e, const char* where);  // RAMPDE_EHIP

#define HIP_TRY(expr)                                          \
  do {                                                         \
    hipError_t e_ = (expr);                                    \
    if (e_ != hipSuccess) return rampde::hip_fail(e_, #expr);  \
  } while (0)

inline bool aligned_to(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
inline bool known_type(rampde_dtype t) { return t == RAMPDE_F32 || t == RAMPDE_F16 || t == RAMPDE_BF16; }
// a launch has less than 2^32 threads along an axis
inline bool launchable(int64_t workgroups, int64_t threads) { return workgroups < ((int64_t)1 << 32) / threads; }
inline size_t type_size(rampde_dtype t) { return t == RAMPDE_F32 ? 4 : 2; }

}  // namespace rampde
