// What the host sides of the C ABI share.  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>

namespace rtams {

// Notes what rtams_last_error() says on this thread and returns the code.
int fail(int code, const char *fmt, ...);

inline size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace rtams

#define HIP_TRY(expr)                                                                  \
  do {                                                                                 \
    hipError_t e_ = (expr);                                                            \
    if (e_ != hipSuccess)                                                              \
      return rtams::fail(RTAMS_EHIP, "%s failed: %s", #expr, hipGetErrorString(e_));   \
  } while (0)
