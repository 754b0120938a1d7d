// entry.h -- what the entry points share: argument checks that become status
// codes, the device capability check, HIP errors as status codes.
#pragma once

#include "acrl_internal.h"

namespace acrl {

acrl_status check_device();                               // the current device is a gfx950
acrl_status hip_status(hipError_t e, const char* what);
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace acrl

#define ACRL_REQUIRE(cond, ...)       \
  do {                                \
    if (!(cond)) {                    \
      acrl::set_error(__VA_ARGS__);   \
      return ACRL_ERR_INVALID_ARG;    \
    }                                 \
  } while (0)
