// Distribution function of the normal distribution, as the gated feed-forward block's bf16 epilogues take it.  No device header is
// needed, so that its error can be measured on the host.
#pragma once

#include <math.h>

#if defined(__HIPCC__)
#define SCMOE_CDF_FN __host__ __device__ __forceinline__
#else
#define SCMOE_CDF_FN static inline
#endif

namespace scmoe {

// Phi(v), and e = e^(-v^2 / 2).  Below zero Phi(v) = e M(|v|), above 1 - that, with M(z) ~ t P(t), t = 1 / (1 + a z) (Hastings' form): the
// smallest error where v is small, and everywhere a fiftieth of bf16's rounding or less: v Phi(v) is multiplied by other factors, so what
// lies far below zero counts relative to itself (a polynomial in v, clamped as in gelu.hpp, is off by 1.2e-5 in Phi, a quarter of it at -4).
// a and P: least largest error over 0 <= z <= 13.5, allowed to grow tenfold from z = 0.5 to 3.5.
//   relative error of Phi   v >= -1: 8.3e-6, >= -2: 2.9e-5, >= -13: 7.4e-5;  absolute: 3.5e-6;  below -13.2 e underflows
// The exponential and the reciprocal are the hardware's (1 ulp each); +-inf and NaN come out as in the formula.
SCMOE_CDF_FN float normal_cdf(float v, float& e) {
  const float u = v * v * -0.72134752044448170f;          // log2 of e
  const float w = fmaf(0.36504852f, fabsf(v), 1.0f);
#if defined(__HIP_DEVICE_COMPILE__)
  e = __builtin_amdgcn_exp2f(u);
  const float t = __builtin_amdgcn_rcpf(w);
#else
  e = exp2f(u);
  const float t = 1.0f / w;
#endif
  float p = -0.091783f;
  p = fmaf(p, t, 0.2233249f);
  p = fmaf(p, t, 0.06596848f);
  p = fmaf(p, t, 0.15774335f);
  p = fmaf(p, t, 0.14474287f);
  const float q = e * (t * p);
  return v < 0.0f ? q : 1.0f - q;
}

}  // namespace scmoe
