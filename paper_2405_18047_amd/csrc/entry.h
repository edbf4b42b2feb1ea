// What the C entry points share: the error text behind a status, and the checks of a HIP call.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include "../../include/tbp.h"

namespace tbp {

// Stores the text that tbp_last_error() returns on this thread and passes the code on.
tbp_status fail(tbp_status code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace tbp

#define TBP_HIP(expr)                                                                             \
  do {                                                                                            \
    hipError_t e__ = (expr);                                                                      \
    if (e__ != hipSuccess) return tbp::fail(TBP_EDEVICE, "%s: %s", #expr, hipGetErrorString(e__)); \
  } while (0)
