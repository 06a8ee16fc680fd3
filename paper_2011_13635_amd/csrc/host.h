// What the files with C entries share: the message of the calling thread's last error.
#pragma once
#include <hip/hip_runtime.h>

namespace mslt {
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));   // records the message, returns code
}  // namespace mslt

#define HIP_TRY(expr)                                                                       \
  do {                                                                                      \
    hipError_t e__ = (expr);                                                                \
    if (e__ != hipSuccess) return fail(MSLT_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e__)); \
  } while (0)
