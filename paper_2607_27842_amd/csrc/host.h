// Host-side helpers shared by the files behind the C ABI: error reporting and small checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "featfix.h"

namespace ff {

// Records the message of the failing call on this thread (ff_last_error) and returns code.
ff_status fail(ff_status code, const char* fmt, ...);
// Clears the message.
ff_status ok();
ff_status hip_fail(hipError_t e, const char* where);
#define HIP_TRY(expr, where)              \
  do {                                    \
    hipError_t _e = (expr);               \
    if (_e != hipSuccess) return ::ff::hip_fail(_e, where); \
  } while (0)

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace ff
