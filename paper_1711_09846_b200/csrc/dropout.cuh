// Dropout's draws: what the stand-alone kernel (dropout.cu) and the gated unit share.
#pragma once
#include "pbt_common.cuh"

namespace pbt {
namespace dropout {

// 0 or the error that pbt_last_error has a message for
int check_rule(const pbt_drop_rule* r, long long members, long long rows, long long width);

// columns that one block of the generator serves
constexpr int kGroup = 8;

#ifdef __CUDACC__
// What a thread has to know to draw for one member.
struct Draw {
  uint32_t member, step, stream;
  uint64_t seed;
  uint32_t limit;     // a 16-bit draw d is kept where d << 16 > limit; only for `on`
  float scale;        // of what is kept
  bool on;            // false: a rate that rounds to 0, nothing is drawn
};
__device__ __forceinline__ Draw draw_of(const pbt_drop_rule& r, int m) {
  Draw d;
  d.member = (uint32_t)(r.first_member + m);
  d.step = (uint32_t)(r.steps ? __ldg(reinterpret_cast<const long long*>(r.steps) + m) : (long long)r.step);
  d.stream = kStreamDropout + (uint32_t)r.site;
  d.seed = r.seed;
  const float rate = r.rate ? __ldg(r.rate + m) : r.rate_all;
  const uint32_t t = (uint32_t)rintf(fminf(fmaxf(rate, 0.f), 1.f) * 65536.f);
  d.on = t != 0;
  d.limit = (t << 16) - 1u;                               // (t = 65536: no draw is above it)
  d.scale = t < 65536u ? __fdiv_rn(65536.f, (float)(65536u - t)) : 0.f;
  return d;
}
// The draws of eight neighbouring columns, and whether column c of them is kept (an odd column has the upper half of its word; what the
// lower half adds below it changes no comparison with limit, whose lower half is all ones).
__device__ __forceinline__ U4 draw_group(const Draw& d, uint32_t block) { return philox4x32_10(d.member, d.step, d.stream, block, d.seed); }
__device__ __forceinline__ bool kept(const U4& w, int c, uint32_t limit) { return ((c & 1) ? w.x[c >> 1] : w.x[c >> 1] << 16) > limit; }
#endif

}  // namespace dropout
}  // namespace pbt
