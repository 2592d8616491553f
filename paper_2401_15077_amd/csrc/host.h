// What the host files of libeagle share: error texts and launch checks.
#pragma once
#include "../../include/eagle.h"
#include <hip/hip_runtime.h>

// Stores the calling thread's error text (eagle_last_error) and returns `code`.
__attribute__((visibility("hidden"), format(printf, 2, 3))) int fail(int code, const char* fmt, ...);

#define HIPCHK(x)                                                                                         \
  do {                                                                                                    \
    hipError_t e_ = (x);                                                                                  \
    if (e_ != hipSuccess) return fail(EAGLE_EHIP, "%s failed: %s (%s:%d)", #x, hipGetErrorString(e_), __FILE__, __LINE__); \
  } while (0)
#define LAUNCH_CHECK() HIPCHK(hipGetLastError())
