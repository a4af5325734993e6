// Error reporting of the C ABI's host code: the message of the last failed call, one per host thread.
#pragma once

#include "../../include/slp.h"

#include <hip/hip_runtime.h>

namespace slp {
// Stores the message slp_last_error returns and gives `code` back.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
}  // namespace slp

#define HIP_TRY(expr)                                                                                  \
  do {                                                                                                 \
    hipError_t e__ = (expr);                                                                           \
    if (e__ != hipSuccess) return slp::fail(SLP_ERR_DEVICE, "%s: %s", #expr, hipGetErrorString(e__)); \
  } while (0)
