// lanes.h -- a wave's lanes among each other: 64-bit keys and values, reductions
// by DPP alone.
#pragma once

#include "acrl_internal.h"

namespace acrl {

#ifdef __HIPCC__

__device__ __forceinline__ double shfl_xor_f64(double v, int m) {
  return __hiloint2double(__shfl_xor(__double2hiint(v), m), __shfl_xor(__double2loint(v), m));
}
__device__ __forceinline__ int read_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ double read_lane(double v, int lane) {
  return __hiloint2double(read_lane(__double2hiint(v), lane), read_lane(__double2loint(v), lane));
}
__device__ __forceinline__ int lowest(uint64_t mask) { return __builtin_ctzll(mask); }

// fp64 values in their order as integers (-0 as 0), and back.  The order of -infinity is above 0.
__device__ __forceinline__ uint64_t score_key(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v == 0.0 ? 0.0 : v);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double score_of(uint64_t k) {
  return __longlong_as_double((long long)(k >> 63 ? k & ~(1ull << 63) : ~k));
}

template <int CTRL>
__device__ __forceinline__ uint64_t max_step(uint64_t v) {
  const int lo = (int)(uint32_t)v, hi = (int)(v >> 32);
  const uint64_t o = (uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(hi, hi, CTRL, 0xF, 0xF, false) << 32 |
                     (uint32_t)__builtin_amdgcn_update_dpp(lo, lo, CTRL, 0xF, 0xF, false);
  return max(v, o);
}
// The largest of a wave's keys, in every lane: DPP steps alone (row_shr 1, 2, 4, 8, then rows into the rows behind them),
// whose latency counts where one result is waited for after another.
__device__ __forceinline__ uint64_t largest(uint64_t v) {
  v = max_step<0x111>(v);
  v = max_step<0x112>(v);
  v = max_step<0x114>(v);
  v = max_step<0x118>(v);
  v = max_step<0x142>(v);
  v = max_step<0x143>(v);
  return (uint64_t)(uint32_t)read_lane((int)(v >> 32), 63) << 32 | (uint32_t)read_lane((int)(uint32_t)v, 63);
}

// Workgroup barrier behind this wave's LDS operations that leaves loads into registers under way.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

#endif  // __HIPCC__

}  // namespace acrl
