// entry.h -- what the entry points share: argument checks that become status
// codes, the device capability check, HIP errors as status codes.
#pragma once

#include "acrl_internal.h"

namespace acrl {

acrl_status check_device();                               // the current device is a gfx950
acrl_status hip_status(hipError_t e, const char* what);
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
// Whether the values of a residual r [M, N] lie in y's memory without being y's own, value for value.  Rows of the same
// pitch may interleave (columns of one matrix).  Types: acrl_out_type; M < 2^26, row distances below 2^34.
inline bool overlaps(const void* residual, int64_t ldr, int r_type, const void* out, int64_t ldy, int y_type, int64_t M,
                     int64_t N) {
  if (M == 0) return false;
  const int64_t ys = y_type == ACRL_OUT_F32 ? 4 : 2, rs = r_type == ACRL_OUT_F32 ? 4 : 2, py = ldy * ys, pr = ldr * rs;
  const uintptr_t y = (uintptr_t)out, r = (uintptr_t)residual;
  const uintptr_t y_end = y + (uintptr_t)((M - 1) * py + N * ys), r_end = r + (uintptr_t)((M - 1) * pr + N * rs);
  if (r >= y_end || y >= r_end) return false;
  if (r == y && ys == rs && (py == pr || M == 1)) return false;
  if (py != pr) return true;
  const int64_t ahead = r >= y ? (int64_t)(r - y) % py : (py - (int64_t)(y - r) % py) % py;  // of r's columns to y's
  return ahead < N * ys || py - ahead < N * rs;
}

}  // namespace acrl

#define ACRL_REQUIRE(cond, ...)       \
  do {                                \
    if (!(cond)) {                    \
      acrl::set_error(__VA_ARGS__);   \
      return ACRL_ERR_INVALID_ARG;    \
    }                                 \
  } while (0)
