// Error returns of the C entry points (internal to libringada).
#pragma once
#include <hip/hip_runtime.h>

#include "ringada.h"

namespace rg {
// sets the calling thread's message and returns s
ringada_status fail(ringada_status s, const char* fmt, ...);
}  // namespace rg

#define RG_HIP(x)                                                                              \
  do {                                                                                         \
    hipError_t e_ = (x);                                                                       \
    if (e_ != hipSuccess)                                                                      \
      return ::rg::fail(RINGADA_E_HIP, "%s failed: %s", #x, hipGetErrorString(e_));            \
  } while (0)

#define RG_TRY(x)                                                                              \
  do {                                                                                         \
    ringada_status s_ = (x);                                                                   \
    if (s_ != RINGADA_OK) return s_;                                                           \
  } while (0)
