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
cudaError_t tc_forward(const pbt_gated_desc* d, const Operand& x, const Operand& w, void* h, float* z, int pitch, bool packed, cudaStream_t s);      // packed: tc_pack is its predecessor
// dx = [dg du] W by CTAs that share a contraction, for few rows; launched right behind the kernel that makes dg and du
bool tc_dx_few(const pbt_gated_desc* d);
cudaError_t tc_dx(const pbt_gated_desc* d, const Operand& dz, const Operand& w, cudaStream_t s);
// dx and dW of still fewer rows in one launch
bool tc_gradients_few(const pbt_gated_desc* d);
cudaError_t tc_gradients(const pbt_gated_desc* d, const Operand& dz, const Operand& w, const Operand& x, cudaStream_t s);
// float (gated_f32.cu): h (or null) and g, u (or null); dx and dW
cudaError_t f32_forward(const pbt_gated_desc* d, float* h, float* z, int pitch, cudaStream_t s);
cudaError_t f32_backward(const pbt_gated_desc* d, const float* dz, int dz_pitch, cudaStream_t s);

#ifdef __CUDACC__
// Eight bf16 elements from any place, of which the first n (1 to 8) exist and the others come as zeros: the 16-byte pieces that hold them, the second one
// only if one of the n lies in it (nothing is read beyond the piece that holds the last of them), shifted together.
struct Pieces {
  uint4 a, b;
  int off, n;
};
__device__ __forceinline__ Pieces pieces_of(const bf16* from, int n) {
  Pieces p;
  const uintptr_t addr = (uintptr_t)from;
  const uint4* piece = reinterpret_cast<const uint4*>(addr & ~(uintptr_t)15);
  p.off = (int)(addr & 15) / 2;
  p.n = n;
  p.a = __ldg(piece);
  p.b = p.off + n > 8 ? __ldg(piece + 1) : make_uint4(0u, 0u, 0u, 0u);
  return p;
}
__device__ __forceinline__ uint4 joined(const Pieces& p) {
  uint32_t w[8] = {p.a.x, p.a.y, p.a.z, p.a.w, p.b.x, p.b.y, p.b.z, p.b.w};      // (off + 7 < 16)
  if (p.off & 4)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  if (p.off & 2)
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  const uint32_t bits = (p.off & 1) * 16;
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __funnelshift_r(w[i], w[i + 1], bits);
  if (p.n < 8)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = 2 * i >= p.n ? 0u : 2 * i + 1 >= p.n ? o[i] & 0xFFFFu : o[i];
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Launches clusters of `cluster` CTAs; `after`: they may begin while the predecessor in the stream still runs (see launch_after).
template <typename... KArgs, typename... Args>
cudaError_t launch_clusters(dim3 grid, unsigned threads, size_t smem, unsigned cluster, bool after, cudaStream_t s, void (*kernel)(KArgs...), Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = after ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(static_cast<Args&&>(args))...);
}

// What goes into a bf16 number takes the short exponential, off by 2 + 1.2 |v| ulp at most, and the short quotient, by 2 ulp more (an ulp is at most 2^-23 of the
// value; a bf16 result's rounding is 2^-8, 2^15 of them); fp32 results take expf and the rounded quotient.
template <typename T>
__device__ __forceinline__ float exponential(float v) {
  if constexpr (sizeof(T) == 4) return expf(v);
  else return __expf(v);
}
template <typename T>
__device__ __forceinline__ float sigmoid(float e) {      // of -log(e)
  if constexpr (sizeof(T) == 4) return __fdiv_rn(1.f, 1.f + e);
  else return __fdividef(1.f, 1.f + e);
}
// act(g)
template <typename T>
__device__ __forceinline__ float activation(int kind, float g) {
  if (kind == kRelu) return g <= 0.f ? 0.f : g;                       // (NaN stays NaN)
  if (kind == kGelu) return g * (0.5f * erfcf(g * -0.70710678f));     // (erfc: no cancellation where g is negative)
  const float s = sigmoid<T>(exponential<T>(-g));
  return kind == kSilu ? g * s : s;
}
// The same for a bf16 result.  The error function's complement in the form t exp(-x^2 + P(t)), t = 1 / (1 + x / 2), of Press, Teukolsky, Vetterling and Flannery, Numerical
// Recipes, section 6.2, with a P of degree five fitted to it: 8e-6 of the value off at most where fp32 holds it (x < 10), a 500th of the result's rounding, in 14 instructions
// (erfcf, three times as many, made the epilogue the limit: 3 x 777 rows, 784 -> 1000: 21.4 us, with silu 17.7).  The backward pass takes erfcf.
__device__ __forceinline__ float activation_bf16(int kind, float g) {
  if (kind != kGelu) return activation<bf16>(kind, g);
  const float x = fabsf(g) * 0.70710678f, t = __fdividef(1.f, fmaf(0.5f, x, 1.f));
  float q = fmaf(0.33007830f, t, -1.02315712f);        // P / ln 2, less 1 for the half in front of erfc
  q = fmaf(q, t, 0.68456119f);
  q = fmaf(q, t, 0.36707783f);
  q = fmaf(q, t, 1.46868443f);
  q = fmaf(q, t, -2.82723355f);
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(x * x, -1.44269504f, q)));
  const float tail = t * e;
  return g * (g < 0.f ? tail : 1.f - tail);
}
// act(g) and act'(g).  1 - sigmoid is taken without a difference of nearly equal numbers.
template <typename T>
__device__ __forceinline__ float activation(int kind, float g, float* slope) {
  if (kind == kRelu) {
    *slope = g > 0.f ? 1.f : 0.f;
    return g <= 0.f ? 0.f : g;
  }
  if (kind == kGelu) {
    const float cdf = 0.5f * erfcf(g * -0.70710678f);
    *slope = fmaf(g * 0.39894228f, exponential<T>(-0.5f * g * g), cdf);
    return g * cdf;
  }
  const float e = exponential<T>(-g), s = sigmoid<T>(e), closed = g > 0.f ? e * s : 1.f - s;
  *slope = kind == kSilu ? s * fmaf(g, closed, 1.f) : s * closed;
  return kind == kSilu ? g * s : s;
}
#endif

}  // namespace gated
}  // namespace pbt
