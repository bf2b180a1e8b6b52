// Activations of the gated feed-forward block and their derivatives.
#pragma once

#include <cuda_runtime.h>

#include "../../include/fh.h"
#include "fh_device.cuh"

namespace fh {

constexpr float kTanhA = 1.5957691216057308f, kTanhB = 0.07135481627260025f;  // tanh's form of the gelu: 2 sqrt(2 / pi), and that times the cube's factor, 0.044715

// The normal distribution below g, Phi(g) = 1 - Phi(-g), for results of type DT, given e = exp(-g^2 / 2).  (1 + erf would leave nothing of it below -5.)
// In fp32 by the complementary error function.  In bf16 that made the gated backward pass of 4096 x 8192 take 122 us instead of 88: there Phi(-a) = e R(a),
// R (which falls as 1 / a does) as t Q(t), t = 1 / (1 + 0.21 a), Q the polynomial of degree 8 whose largest error relative to R for a up to 14.6 is least
// (2e-8; 1e-6 with its evaluation and a quotient that is two places off; beyond, e is 0).
template <int DT>
__device__ __forceinline__ float normal_below(float g, float e) {
  if (DT == kF32) return 0.5f * erfcf(-0.7071067811865476f * g);
  const float t = __fdividef(1.0f, __fmaf_rn(0.21f, fabsf(g), 1.0f));
  float r = -0.0712238997f;
  r = __fmaf_rn(r, t, 0.281454891f);
  r = __fmaf_rn(r, t, -0.325757146f);
  r = __fmaf_rn(r, t, 0.344124019f);
  r = __fmaf_rn(r, t, -0.0901580527f);
  r = __fmaf_rn(r, t, 0.123199955f);
  r = __fmaf_rn(r, t, 0.0696428269f);
  r = __fmaf_rn(r, t, 0.085001573f);
  r = __fmaf_rn(r, t, 0.0837158337f);
  const float q = e * (r * t);
  return g < 0.0f ? q : 1.0f - q;
}

// act(g), for a result of type DT.  silu and tanh's form of the gelu are g / (1 + exp(-v)), v = g and g (A + B g^2).  The exponential is that of -|v|, which
// never overflows, so that values next to nothing are not lost, and the fast quotient, two places off at most, has denominators from 1 to 2 (an exact one, 4096 x
// 8192 x 4096 in fp32 412 us, 210 so).  For bf16 the exponential is the fast one too, up to 1e-5 of the value off, a hundredth of what rounding it is.
template <int ACT, int DT>
__device__ __forceinline__ float act_of(float g) {
  if (ACT == FH_SILU || ACT == FH_GELU_TANH) {
    const float v = ACT == FH_SILU ? g : g * __fmaf_rn(kTanhB, g * g, kTanhA);
    const float e = DT == kF32 ? expf(-fabsf(v)) : __expf(-fabsf(v)), top = v < 0.0f ? g * e : g;
    return __fdividef(top, 1.0f + e);
  }
  if (ACT == FH_GELU) return g * normal_below<DT>(g, DT == kF32 ? 0.0f : __expf(-0.5f * g * g));
  return g > 0.0f ? g : (g != g ? g : 0.0f);
}

// act(g) and its derivative.  (Full-precision functions: behind this a gradient may be rounded to whole numbers, where an error in the last
// places turns over more of them than it has to; the quotient of 1 and 1 to 2 is a fast one where the gradient is rounded to bf16 first: 4096 x 8192 102 us and 79.)
template <int ACT, int DT>
__device__ __forceinline__ void act_and_slope(float g, float& a, float& slope) {
  if (ACT == FH_SILU || ACT == FH_GELU_TANH) {
    // p = 1 / (1 + exp(-v)) and q = 1 - p, both from exp(-|v|), so that neither is what is left of 1; the derivative is p (1 + g v' q).  From 64 on tanh's p
    // is 0 or 1 whatever g is, and beyond some 1e19 its v' would be infinite.
    const float c = ACT == FH_SILU ? g : max_nan(min_nan(g, 64.0f), -64.0f), cc = c * c;
    const float v = ACT == FH_SILU ? g : c * __fmaf_rn(kTanhB, cc, kTanhA), along = ACT == FH_SILU ? g : c * __fmaf_rn(3.0f * kTanhB, cc, kTanhA);
    const float e = expf(-fabsf(v)), r = DT == kF32 ? 1.0f / (1.0f + e) : __fdividef(1.0f, 1.0f + e), p = v < 0.0f ? e * r : r, q = v < 0.0f ? r : e * r;
    a = g * p;
    slope = p * __fmaf_rn(along, q, 1.0f);
  } else if (ACT == FH_GELU) {
    const float e = expf(-0.5f * g * g), p = normal_below<DT>(g, e);
    a = g * p;
    slope = __fmaf_rn(g * 0.3989422804014327f, e, p);
  } else {
    const bool on = g > 0.0f;
    a = on ? g : (g != g ? g : 0.0f);
    slope = on ? 1.0f : 0.0f;
  }
}

}  // namespace fh
