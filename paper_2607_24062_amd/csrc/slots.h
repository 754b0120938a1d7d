// slots.h -- what the per-response kernels share: sums over wavefronts and
// workgroups by fixed trees, loads of a [B, L] batch's slots, launches by
// workgroup size.
#pragma once

#include <type_traits>

#include "acrl_internal.h"

namespace acrl {
namespace {

constexpr int kRedThreads = 256;
constexpr int kSlots = 4;  // slots a thread takes per turn

// Sum / maximum over groups of N = 4, 16 or 64 consecutive lanes: DPP inside
// each row of 16, lane exchanges across rows.
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double v) {
  const long long b = __double_as_longlong(v);
  const int lo = __builtin_amdgcn_mov_dpp((int)b, CTRL, 0xF, 0xF, true);
  const int hi = __builtin_amdgcn_mov_dpp((int)(b >> 32), CTRL, 0xF, 0xF, true);
  return __longlong_as_double(((long long)hi << 32) | (unsigned)lo);
}
template <int N>
__device__ __forceinline__ double lane_sum(double v) {
  v += dpp_f64<0xB1>(v);                      // quad_perm [1,0,3,2]
  v += dpp_f64<0x4E>(v);                      // quad_perm [2,3,0,1]
  if constexpr (N >= 16) {
    v += dpp_f64<0x124>(v);                   // row_ror:4
    v += dpp_f64<0x128>(v);                   // row_ror:8
  }
  if constexpr (N == 64) {
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
  }
  return v;
}
template <int N>
__device__ __forceinline__ double lane_max(double v) {
  v = fmax(v, dpp_f64<0xB1>(v));
  v = fmax(v, dpp_f64<0x4E>(v));
  if constexpr (N >= 16) {
    v = fmax(v, dpp_f64<0x124>(v));
    v = fmax(v, dpp_f64<0x128>(v));
  }
  if constexpr (N == 64) {
    v = fmax(v, __shfl_xor(v, 16));
    v = fmax(v, __shfl_xor(v, 32));
  }
  return v;
}

__device__ __forceinline__ double first_lane(double v) {
  const long long b = __double_as_longlong(v);
  const int lo = __builtin_amdgcn_readfirstlane((int)b), hi = __builtin_amdgcn_readfirstlane((int)(b >> 32));
  return __longlong_as_double(((long long)hi << 32) | (unsigned)lo);
}

// Sums of NS values and the maximum of mx over a workgroup of NT = 64, 256 or
// 1024 threads, one barrier (none for a wavefront): trees inside each
// wavefront, then every thread's lane group of NT / 64 lanes takes one
// wavefront's result each and adds them by the same tree.  Deterministic.
// (The serial sum over the wavefronts, one dependent LDS read after another,
// made the 1024-thread batch statistics 13.5 us long.)
template <int NS, int NT>
struct BlockShared {
  double s[NT / 64][NS];
  double mx[NT / 64];
};
template <int NS, int NT>
__device__ __forceinline__ void block_stats(double (&v)[NS], double& mx, BlockShared<NS, NT>& sh) {
  constexpr int NW = NT / 64;
  static_assert(NW == 1 || NW == 4 || NW == 16, "1, 4 or 16 wavefronts");
#pragma unroll
  for (int k = 0; k < NS; ++k) v[k] = lane_sum<64>(v[k]);
  mx = lane_max<64>(mx);
  if constexpr (NW > 1) {
    const int w = threadIdx.x >> 6, q = threadIdx.x & (NW - 1);
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < NS; ++k) sh.s[w][k] = v[k];
      sh.mx[w] = mx;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NS; ++k) v[k] = lane_sum<NW>(sh.s[q][k]);
    mx = lane_max<NW>(sh.mx[q]);
  }
}

template <int NT, bool VEC>
__device__ __forceinline__ int64_t first_slot() {
  return VEC ? (int64_t)threadIdx.x * kSlots : (int64_t)threadIdx.x;
}
// The mask of the thread's slots from slot j on of the response at `base`
// (slots past L: 0) and four values of x there, 0 past L.
template <int NT, bool VEC>
__device__ __forceinline__ void load_mask(const uint8_t* __restrict__ mask, int64_t base, int64_t j, int64_t L,
                                          uint8_t (&m)[kSlots]) {
  if constexpr (VEC) {
    const uchar4 t = *reinterpret_cast<const uchar4*>(mask + base + j);
    m[0] = t.x; m[1] = t.y; m[2] = t.z; m[3] = t.w;
  } else {
#pragma unroll
    for (int k = 0; k < kSlots; ++k) m[k] = j + k * NT < L ? mask[base + j + k * NT] : (uint8_t)0;
  }
}
template <int NT, bool VEC>
__device__ __forceinline__ void load_slots(const float* __restrict__ x, int64_t base, int64_t j, int64_t L,
                                           float (&v)[kSlots]) {
  if constexpr (VEC) {
    const float4 t = *reinterpret_cast<const float4*>(x + base + j);
    v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
  } else {
#pragma unroll
    for (int k = 0; k < kSlots; ++k) v[k] = j + k * NT < L ? x[base + j + k * NT] : 0.0f;
  }
}

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned(const void* q, uintptr_t a) { return ((uintptr_t)q & (a - 1)) == 0; }

// launch(workgroup size, 16-byte slots) of a per-response kernel of nt threads.
template <typename F>
inline void launch_seq(int nt, bool vec, F&& launch) {
  auto with = [&](auto n) {
    if (vec) launch(n, std::true_type{});
    else launch(n, std::false_type{});
  };
  switch (nt) {
    case 64: return with(std::integral_constant<int, 64>{});
    case 1024: return with(std::integral_constant<int, 1024>{});
    default: return with(std::integral_constant<int, kRedThreads>{});
  }
}

}  // namespace
}  // namespace acrl
