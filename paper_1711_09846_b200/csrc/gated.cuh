// Gated units of a population: declarations shared by the entry points (gated.cu) and the tensor-core kernels.
#pragma once
#include "dropout.cuh"

namespace pbt {
namespace gated {

enum Activation : int { kSilu = 0, kGelu = 1, kRelu = 2, kSigmoid = 3 };

#ifdef __CUDACC__
// act(g)
__device__ __forceinline__ float activation(int kind, float g) {
  if (kind == kRelu) return g <= 0.f ? 0.f : g;                       // (NaN stays NaN)
  if (kind == kGelu) return g * (0.5f * erfcf(g * -0.70710678f));     // (erfc: no cancellation where g is negative)
  const float s = __fdividef(1.f, 1.f + __expf(-g));
  return kind == kSilu ? g * s : s;
}
// act(g) and act'(g).  1 - sigmoid is taken without a difference of nearly equal numbers.
__device__ __forceinline__ float activation(int kind, float g, float* slope) {
  if (kind == kRelu) {
    *slope = g > 0.f ? 1.f : 0.f;
    return g <= 0.f ? 0.f : g;
  }
  if (kind == kGelu) {
    const float cdf = 0.5f * erfcf(g * -0.70710678f);
    *slope = fmaf(g * 0.39894228f, __expf(-0.5f * g * g), cdf);
    return g * cdf;
  }
  const float e = __expf(-g), s = __fdividef(1.f, 1.f + e), closed = g > 0.f ? e * s : 1.f - s;
  *slope = kind == kSilu ? s * fmaf(g, closed, 1.f) : s * closed;
  return kind == kSilu ? g * s : s;
}
#endif

}  // namespace gated
}  // namespace pbt
