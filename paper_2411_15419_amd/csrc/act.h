// Expert activations.
#pragma once

#include "luffy_common.h"

namespace luffy {

// From the device math library, for results that stay in float32: the error is a
// few 2^-24 of |z|.
template <int ACT>
__device__ __forceinline__ float act_f32(float z) {
  if constexpr (ACT == LUFFY_ACT_GELU) {
    return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
  } else {
    return z / (1.0f + expf(-z));
  }
}

// The same with a small error relative to the value, a few 2^-24 (1 + z^2), also
// where 1 + erf cancels (z < -3: act_f32 leaves 57 % of GELU(-5.5)).
template <int ACT>
__device__ __forceinline__ float act_f32_relative(float z) {
  if constexpr (ACT == LUFFY_ACT_GELU) {
    return 0.5f * z * erfcf(z * -0.70710678118654752f);
  } else {
    return act_f32<ACT>(z);
  }
}

// Activation code of a plain product (no activation), used by the backward.
constexpr int kActNone = 2;

// For results that are rounded to bf16 (relative step 2^-8): a dozen VALU
// operations instead of the library erf, which dominated the epilogue of the
// first product.  The error is small beside the largest values of a row, not
// beside the value: 1.4e-7 |z| for GELU, so that GELU(-5.5) = -1.0e-7 comes as
// -2.4e-7 and anything below -6 as 0.
//   GELU: erf from Abramowitz & Stegun 7.1.26 (Hastings' rational
//   approximation), erf(u) = 1 - q(u), q(u) = t (a1 + t (a2 + ... + t a5))
//   e^{-u^2}, t = 1 / (1 + p u), u >= 0, |error| <= 1.5e-7.  With
//   u = |z| / sqrt(2): GELU(z) = z (1 - q/2) for z >= 0 and z q/2 for z < 0,
//   evaluated as |z| (1 - q) / 2 + z / 2.
//   SiLU: z / (1 + 2^{-z log2 e}).
// The hardware exp2 and reciprocal are accurate to about 1 ulp.
template <int ACT>
__device__ __forceinline__ float act_fast(float z) {
  if constexpr (ACT == kActNone) {
    return z;
  } else if constexpr (ACT == LUFFY_ACT_GELU) {
    // Hastings' erf(u) = 1 - t (a1 + a2 t + ... + a5 t^4) e^{-u^2},
    // t = 1 / (1 + p u), u = |z| / sqrt(2), with the a_i halved here so
    // that w = 1/2 - t e P(t) = erf(u) / 2.  Then z Phi(z) = |z| w + z / 2
    // for either sign of z (Phi(z) = 1/2 + sign(z) erf(u) / 2): 10 vector
    // operations and two transcendentals per element.
    constexpr float kPs = 0.3275911f * 0.70710678118654752f;   // p / sqrt(2)
    constexpr float kB1 = 0.5f * 0.254829592f, kB2 = 0.5f * -0.284496736f, kB3 = 0.5f * 1.421413741f;
    constexpr float kB4 = 0.5f * -1.453152027f, kB5 = 0.5f * 1.061405429f;
    constexpr float kHalfLog2e = -0.72134752044448170f;   // -log2(e) / 2
    const float a = fabsf(z);
    const float t = __builtin_amdgcn_rcpf(fmaf(kPs, a, 1.0f));
    const float pt = fmaf(t, fmaf(t, fmaf(t, fmaf(t, kB5, kB4), kB3), kB2), kB1);
    const float e = __builtin_amdgcn_exp2f(z * z * kHalfLog2e);   // e^{-u^2}
    const float w = fmaf(-(t * e), pt, 0.5f);
    return fmaf(a, w, 0.5f * z);
  } else {
    constexpr float kNegLog2e = -1.44269504088896341f;
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * kNegLog2e));
  }
}

// For results that are rounded relative to their own size (blocks under a scale
// of their largest value, where a block may hold nothing but small values): the
// negative tail keeps its relative accuracy, at one operation more than act_fast.
//   GELU(z) = max(z, 0) - a Phi(-a), a = |z|: nothing cancels for z < 0.
//   Phi(-a) = e^{-a^2 / 2} t P(t), t = 1 / (1 + p a); t P(t) approximates
//   erfcx(a / sqrt(2)) / 2, the six coefficients of P by a linear program for the
//   least largest relative error over 0 <= a <= 14, weighted by 1 / (1 + a^2)
//   (what the rounding of a^2 / 2 costs anyway).  Relative error of the whole:
//   at most 10^-6 (1 + z^2) down to z = -13, where GELU leaves float32's normal
//   numbers.
//   SiLU: act_fast's keeps its relative accuracy down to z = -87 (0 below).
template <int ACT>
__device__ __forceinline__ float act_relative(float z) {
  if constexpr (ACT == LUFFY_ACT_GELU) {
    constexpr float kP = 0.295f;
    constexpr float kC1 = 0.11853463f, kC2 = 0.10662275f, kC3 = 0.16428097f, kC4 = -0.05983869f;
    constexpr float kC5 = 0.25534352f, kC6 = -0.08494314f;
    constexpr float kHalfLog2e = -0.72134752044448170f;   // -log2(e) / 2
    const float a = fabsf(z);
    const float t = __builtin_amdgcn_rcpf(fmaf(kP, a, 1.0f));
    const float pt = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, kC6, kC5), kC4), kC3), kC2), kC1);
    const float e = __builtin_amdgcn_exp2f(z * z * kHalfLog2e);   // e^{-a^2 / 2}
    return fmaf(-a, t * e * pt, fmaxf(z, 0.0f));
  } else {
    return act_fast<ACT>(z);
  }
}

}  // namespace luffy
