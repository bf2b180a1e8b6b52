// Activations of the gated feed-forward block and their derivatives.
#pragma once

#include <cuda_runtime.h>

#include "../../include/fh.h"

namespace fh {

constexpr float kTanhC = 0.7978845608028654f, kTanhK = 0.044715f;  // tanh's form of the gelu: sqrt(2 / pi), and the cube's factor

// act(g).
template <int ACT>
__device__ __forceinline__ float act_of(float g) {
  if (ACT == FH_SILU) return __fdividef(g, 1.0f + __expf(-g));
  if (ACT == FH_GELU) return 0.5f * g * (1.0f + erff(g * 0.7071067811865476f));
  if (ACT == FH_GELU_TANH) {  // 0.5 g (1 + tanh w) = g / (1 + exp(-2 w))
    const float w = kTanhC * __fmaf_rn(kTanhK * g * g, g, g);
    return __fdividef(g, 1.0f + __expf(-2.0f * w));
  }
  return g > 0.0f ? g : (g != g ? g : 0.0f);
}

// act(g) and its derivative.  (Full-precision functions: behind this a gradient may be rounded to whole numbers, where an error in the last
// places turns over more of them than it has to.)
template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float& a, float& slope) {
  if (ACT == FH_SILU) {
    const float p = 1.0f / (1.0f + expf(-g));
    a = g * p;
    slope = p * __fmaf_rn(g, 1.0f - p, 1.0f);
  } else if (ACT == FH_GELU) {
    const float p = 0.5f * (1.0f + erff(g * 0.7071067811865476f));
    a = g * p;
    slope = __fmaf_rn(g * 0.3989422804014327f, expf(-0.5f * g * g), p);
  } else if (ACT == FH_GELU_TANH) {  // (1 + tanh w) / 2 = p, (1 - tanh w) / 2 = q
    const float e = expf(-2.0f * kTanhC * __fmaf_rn(kTanhK * g * g, g, g)), p = 1.0f / (1.0f + e), q = e <= 1.0f ? e * p : 1.0f - p;
    a = g * p;
    slope = __fmaf_rn(2.0f * g * p * q, kTanhC * __fmaf_rn(3.0f * kTanhK * g, g, 1.0f), p);
  } else {
    const bool on = g > 0.0f;
    a = on ? g : (g != g ? g : 0.0f);
    slope = on ? 1.0f : 0.0f;
  }
}

}  // namespace fh
