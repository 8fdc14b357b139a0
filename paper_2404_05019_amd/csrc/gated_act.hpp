// The activation of the gated feed-forward block: its value and its slope.
#pragma once
#include "common.hpp"
#include "normal_cdf.hpp"

namespace scmoe {

// a = act(g), s = act'(g).
//   SiLU        p = 1 / (1 + e^-g):              a = g p,   s = p (1 + g (1 - p))
//   GELU, erf   P = Phi(g):                      a = g P,   s = P + g e^(-g^2/2) / sqrt(2 pi)
//   GELU, tanh  p = 1 / (1 + e^(-2 c (g + b g^3))): a = g p, s = p + g p (1 - p) 2 c (1 + 3 b g^2)
// EXACT (fp32 storage): the library's exponential and complementary error function and a division.  Otherwise (bf16) the hardware's
// exponential and reciprocal (1 ulp each), and Phi as in normal_cdf.hpp.  p and P are right relative to themselves as far as fp32 goes
// down (p: to 2 |t| 2^-24 and some roundings; P: EXACT 2 g^2 2^-24, else 7.4e-5, beside the 2^-8 of the store): far below zero, where act(g) is
// small, u, dh and weights may be large.  (0.5 (1 + erf) in fp32, or a polynomial in g, lose P there: 5 % at -5, a quarter at -4.)
// ACT is a parameter of the kernels: as an argument every element had a branch of its own, and its exponential and reciprocal waited for
// by themselves (32768 rows, d = 2048, F = 8192, E = 16, forward 2469 us, so 2302).
// g^2 is held below 1e8, where the products with p (1 - p) = 0 would be infinity times zero; an infinite g still gives what the
// formula gives.
template <bool EXACT>
__device__ __forceinline__ float sigmoid_of(float t_log2e, float t) {     // 1 / (1 + e^-t), t_log2e = t log2(e)
  if constexpr (EXACT) return 1.0f / (1.0f + expf(-t));
  else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-t_log2e));
}

template <bool EXACT, int ACT>
__device__ __forceinline__ float gated_act(float g) {
  constexpr float LOG2E = 1.4426950408889634f;
  if constexpr (ACT == SCMOE_SILU) {
    return g * sigmoid_of<EXACT>(g * LOG2E, g);
  } else if constexpr (ACT == SCMOE_GELU_TANH) {
    const float t = g * fmaf(0.07135481627f, g * g, 1.5957691216057308f);
    return g * sigmoid_of<EXACT>(t * LOG2E, t);
  } else if constexpr (EXACT) {
    return 0.5f * g * erfcf(g * -0.70710678118654752f);
  } else {
    float e;
    return g * normal_cdf(g, e);
  }
}

template <bool EXACT, int ACT>
__device__ __forceinline__ void gated_act_slope(float g, float& a, float& s) {
  constexpr float LOG2E = 1.4426950408889634f;
  if constexpr (ACT == SCMOE_SILU) {
    const float p = sigmoid_of<EXACT>(g * LOG2E, g);
    a = g * p;
    s = p * fmaf(g, 1.0f - p, 1.0f);
  } else if constexpr (ACT == SCMOE_GELU_TANH) {
    const float g2 = fminf(g * g, 1e8f);
    const float t = g * fmaf(0.07135481627f, g2, 1.5957691216057308f);
    const float p = sigmoid_of<EXACT>(t * LOG2E, t);
    a = g * p;
    s = fmaf(a * (1.0f - p), fmaf(0.21406444881f, g2, 1.5957691216057308f), p);
  } else {
    float p, e;
    if constexpr (EXACT) {
      p = 0.5f * erfcf(g * -0.70710678118654752f);
      e = expf(-0.5f * (g * g));
    } else {
      p = normal_cdf(g, e);
    }
    a = g * p;
    s = fmaf(g * 0.3989422804014327f, e, p);
  }
}

}  // namespace scmoe
