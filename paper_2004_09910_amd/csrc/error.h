// Status and message of a failed call, shared by the C entry points.
#pragma once
#include <hip/hip_runtime.h>

#include "tgp.h"

namespace tgpk {

// Keeps the formatted message for tgp_last_error (per thread); returns s.
tgp_status fail(tgp_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace tgpk

#define HIPCHK(expr, name)                                                         \
  do {                                                                             \
    hipError_t e_ = (expr);                                                        \
    if (e_ != hipSuccess)                                                          \
      return ::tgpk::fail(TGP_EHIP, "%s: %s", name, hipGetErrorString(e_));        \
  } while (0)
