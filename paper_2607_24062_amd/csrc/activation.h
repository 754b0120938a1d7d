// activation.h -- the activations of acrl_linear_fp8 and acrl_moe_fp8, in fp32.
//
// FINE: within 6e-7 of the exact value, relative to its size, or within 1.3e-36
// (the reciprocal of 1 + e^-s is 0 below fp32's normal range, 1.2e-38, and meets a
// value of at most 104 there).  Otherwise, for results that become bf16 (half a
// step: 2e-3 .. 4e-3): within 5e-5, or 1.3e-36, in fewer instructions, which stand
// after a product with nothing to hide them (8192 x 13824 x 5120, bf16 out, fine
// and short: GELU 575 and 547 us, GELU_TANH 597 and 532, SILU 537 and 526; 511 with
// no activation).
#pragma once

#include <type_traits>

#include "acrl_internal.h"

namespace acrl {

#ifdef __HIPCC__

// e^x.  The product with log2(e) is kept in two parts: rounded to one fp32 it
// would be off by |x| 2^-24, and the result, relatively, by as much.
template <bool FINE = true>
__device__ __forceinline__ float exp_f32(float x) {
  if (!FINE) return __builtin_amdgcn_exp2f(x * kLog2e);
  const float t = x * kLog2e;
  const float rest = fmaf(x, 1.9259629911266174e-8f, fmaf(x, kLog2e, -t));  // (log2(e) less its fp32 value)
  const float e = __builtin_amdgcn_exp2f(t);
  return fabsf(t) < 127.0f ? fmaf(e * rest, kLn2, e) : e;  // (infinities have no rest)
}

// x / (1 + e^-s)
template <bool FINE>
__device__ __forceinline__ float times_sigmoid(float x, float s) {
  return x * __builtin_amdgcn_rcpf(1.0f + exp_f32<FINE>(-s));
}

// erfc(z), z >= 0: e^(-z^2) times a polynomial in t = 1 / (1 + z / 2), fitted to
// e^(z^2) erfc(z) over 0 <= z <= 14 for the least relative error (4.3e-8; 3.1e-7 as
// evaluated in fp32).  square = z^2 in two parts.
__device__ __forceinline__ float erfc_of(float z, float square, float square_rest) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.5f, z, 1.0f));
  float p = -0.05882089212536812f;
  p = fmaf(p, t, 0.28327813744544983f);
  p = fmaf(p, t, -0.4842751920223236f);
  p = fmaf(p, t, 0.27434107661247253f);
  p = fmaf(p, t, -0.023677371442317963f);
  p = fmaf(p, t, 0.20118770003318787f);
  p = fmaf(p, t, 0.24359264969825745f);
  p = fmaf(p, t, 0.28227686882019043f);
  p = fmaf(p, t, 0.2820975184440613f);
  p = fmaf(p, t, -5.319922706803482e-07f);
  const float e = exp_f32(-square);
  return p * fmaf(-e, square_rest, e);
}

// 2 sqrt(2 / pi) (v + 0.044715 v^3) = v (c1 + c3 v^2) in two parts: far below 0 the result is v e^(2 u), and one fp32
// for 2 u would leave it |2 u| 2^-24 and more off, relatively.  (No contraction: the parts are of the very products.)
__device__ __forceinline__ float twice_u(float v, float& rest) {
#pragma clang fp contract(off)
  constexpr double kC1 = 1.5957691216057307, kC3 = kC1 * 0.044715;
  constexpr float c1 = (float)kC1, c3 = (float)kC3, c1_rest = (float)(kC1 - c1), c3_rest = (float)(kC3 - c3);
  const float q = v * v, a = c3 * q;
  const float a_rest = fmaf(c3, q, -a) + (c3 * fmaf(v, v, -q) + c3_rest * q);
  const float g = c1 + a, back = g - c1;
  const float g_rest = ((c1 - (g - back)) + (a - back)) + (a_rest + c1_rest);
  const float s = v * g;
  rest = fmaf(v, g, -s) + v * g_rest;
  return s;
}

// GELU in 15 instructions: v Phi(v) = max(v, 0) - a erfc(a / sqrt 2) / 2, a = |v|, with a shorter polynomial for
// erfc / 2 (3.4e-5).  (From 20 on erfc is 0 and a may end, which keeps infinity from meeting it.  The minimum keeps NaN.
// -infinity does meet it, and is NaN as in the fine form: by the last minimum, 2 us of 567 at 8192 x 13824 x 5120.)
__device__ __forceinline__ float gelu_short(float v) {
  const float a = __builtin_elementwise_minimum(fabsf(v), 20.0f);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.35355339059327376f, a, 1.0f));
  float p = -0.0337139293551445f;
  p = fmaf(p, t, 0.0092944344505667686f);
  p = fmaf(p, t, 0.13621488213539124f);
  p = fmaf(p, t, 0.10261718928813934f);
  p = fmaf(p, t, 0.14475198090076447f);
  p = fmaf(p, t, 0.14081886410713196f);
  return fmaf(fminf(v, -a), p * t * __builtin_amdgcn_exp2f(a * a * (-0.5f * kLog2e)), fmaxf(v, 0.0f));
}

template <int ACT, bool FINE>
__device__ __forceinline__ float activate(float v) {
  if constexpr (ACT == ACRL_ACT_RELU) {
    return v < 0.0f ? 0.0f : v;
  } else if constexpr (ACT == ACRL_ACT_SILU) {
    return times_sigmoid<FINE>(v, v);
  } else if constexpr (ACT == ACRL_ACT_GELU) {
    if (!FINE) return gelu_short(v);
    // v Phi(v) = v erfc(-v / sqrt 2) / 2, by erfc of |v| / sqrt 2 on either side: no digits are lost far below 0
    const float a = fminf(fabsf(v), 20.0f), s = 0.5f * a * a;  // (erfc is 0 in fp32 from 14.2 / sqrt 2 on)
    const float half = 0.5f * erfc_of(0.70710678118654752f * a, s, fmaf(0.5f * a, a, -s));
    return v * (v < 0.0f ? half : 1.0f - half);
  } else if constexpr (ACT == ACRL_ACT_GELU_TANH) {
    // 1 + tanh(u) = 2 / (1 + e^(-2 u)), u = sqrt(2 / pi) (v + 0.044715 v^3)
    if (!FINE) {  // (the factor log2(e) with the others)
      constexpr float c1 = (float)(-1.5957691216057307 * 1.4426950408889634), c3 = (float)(-0.0713548162726 * 1.4426950408889634);
      return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * fmaf(c3, v * v, c1)));
    }
    float rest;
    const float s = twice_u(v, rest), e = exp_f32(-s);
    return v * __builtin_amdgcn_rcpf(1.0f + (fabsf(s) < 87.0f ? fmaf(-e, rest, e) : e));
  } else {
    return v;
  }
}

// f with the activation as a constant.
template <typename F>
__device__ __forceinline__ void for_activation(int act, F&& f) {
  switch (act) {
    case ACRL_ACT_RELU: f(std::integral_constant<int, ACRL_ACT_RELU>{}); break;
    case ACRL_ACT_SILU: f(std::integral_constant<int, ACRL_ACT_SILU>{}); break;
    case ACRL_ACT_GELU: f(std::integral_constant<int, ACRL_ACT_GELU>{}); break;
    case ACRL_ACT_GELU_TANH: f(std::integral_constant<int, ACRL_ACT_GELU_TANH>{}); break;
    default: f(std::integral_constant<int, ACRL_ACT_NONE>{});
  }
}

#endif  // __HIPCC__

}  // namespace acrl
