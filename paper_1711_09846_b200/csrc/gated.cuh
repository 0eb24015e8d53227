// Gated units of a population: declarations shared by the entry points (gated.cu) and the tensor-core kernels.
#pragma once
#include "dropout.cuh"

namespace pbt {
namespace gated {

enum Activation : int { kSilu = 0, kGelu = 1, kRelu = 2, kSigmoid = 3 };

// An operand of the tensor cores: [members][rows][...], 16-byte aligned rows; member 0: the same for all members.
struct Operand {
  const bf16* p;
  long long row, member;
};
// bf16 (gated_tc.cu): h (or null) and g, u in fp32 (or null), [members][rows][2][pitch]
bool tc_aligned(const void* p, long long row, long long member, int members);
struct PackSource {
  Operand from;
  bf16* to;                      // rows of a multiple of 8 elements
  int members, rows, cols;
};
cudaError_t tc_pack(const PackSource* src, int n, cudaStream_t s);      // one or two
cudaError_t tc_forward(const pbt_gated_desc* d, const Operand& x, const Operand& w, void* h, float* z, int pitch, cudaStream_t s);
// dx = [dg du] W by CTAs that share a contraction, for few rows
bool tc_dx_few(const pbt_gated_desc* d);
cudaError_t tc_dx(const pbt_gated_desc* d, const Operand& dz, const Operand& w, cudaStream_t s);
// dW of a few rows
bool tc_outer_supported(const pbt_gated_desc* d);
cudaError_t tc_outer(const pbt_gated_desc* d, const bf16* dz, int dz_pitch, const Operand& x, cudaStream_t s);
// float (gated_f32.cu): h (or null) and g, u (or null); dx and dW
cudaError_t f32_forward(const pbt_gated_desc* d, float* h, float* z, int pitch, cudaStream_t s);
cudaError_t f32_backward(const pbt_gated_desc* d, const float* dz, int dz_pitch, cudaStream_t s);

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
