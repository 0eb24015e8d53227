// Dropout's draws: what the stand-alone kernel (dropout.cu) and the gated unit share.
#pragma once
#include "pbt_common.cuh"

namespace pbt {
namespace dropout {

// 0 or the error that pbt_last_error has a message for
int check_rule(const pbt_drop_rule* r, long long members, long long rows, long long width);

// columns that one block of the generator serves
constexpr int kGroup = 8;

// n / d for n < 2^31 in two instructions (the quotient of a product with a rounded reciprocal of 32 bits; the error stays below 1 / d there)
struct Divisor {
  uint32_t factor, shift;
};
inline Divisor divisor(uint32_t d) {
  uint32_t s = 0;
  while (s < 31 && (1u << s) < d) ++s;                          // 2^(s - 1) < d <= 2^s
  return {(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};     // (d = 1: 2^31)
}
// A rule as the kernels take it, with the keys of the generator's rounds: operands from constant memory instead of two additions a round.
struct Rule {
  pbt_drop_rule rule;
  uint32_t keys[20];
};
inline Rule rule_of(const pbt_drop_rule& r) {
  Rule k = {r, {}};
  for (int i = 0; i < 10; ++i) {
    k.keys[2 * i] = (uint32_t)r.seed + 0x9E3779B9u * i;
    k.keys[2 * i + 1] = (uint32_t)(r.seed >> 32) + 0xBB67AE85u * i;
  }
  return k;
}

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t quotient(uint32_t n, Divisor d) { return (uint32_t)(((uint64_t)n * d.factor) >> 31) >> d.shift; }

// What a thread has to know to draw for one member.
struct Draw {
  uint32_t member, step, stream;
  uint32_t limit;     // a 16-bit draw d is kept where d << 16 > limit; only for `on`
  float scale;        // of what is kept
  bool on;            // false: a rate that rounds to 0, nothing is drawn
};
__device__ __forceinline__ Draw draw_of(const Rule& rule, int m) {
  const pbt_drop_rule& r = rule.rule;
  Draw d;
  d.member = (uint32_t)(r.first_member + m);
  d.step = (uint32_t)(r.steps ? __ldg(reinterpret_cast<const long long*>(r.steps) + m) : (long long)r.step);
  d.stream = kStreamDropout + (uint32_t)r.site;
  const float rate = r.rate ? __ldg(r.rate + m) : r.rate_all;
  const uint32_t t = (uint32_t)rintf(fminf(fmaxf(rate, 0.f), 1.f) * 65536.f);
  d.on = t != 0;
  d.limit = (t << 16) - 1u;                               // (t = 65536: no draw is above it)
  d.scale = t < 65536u ? __fdiv_rn(65536.f, (float)(65536u - t)) : 0.f;
  return d;
}
// The draws of eight neighbouring columns, and whether column c of them is kept (an odd column has the upper half of its word; what the
// lower half adds below it changes no comparison with limit, whose lower half is all ones).
__device__ __forceinline__ U4 draw_group(const Rule& rule, const Draw& d, uint32_t block) {
  uint32_t c0 = d.member, c1 = d.step, c2 = d.stream, c3 = block;      // philox4x32_10
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ rule.keys[2 * i];
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ rule.keys[2 * i + 1];
    c3 = (uint32_t)p0;
  }
  return {{c0, c1, c2, c3}};
}
__device__ __forceinline__ bool kept(const U4& w, int c, uint32_t limit) { return ((c & 1) ? w.x[c >> 1] : w.x[c >> 1] << 16) > limit; }
// bit c: column c is kept
__device__ __forceinline__ uint32_t kept_bits(const Rule& rule, const Draw& d, uint32_t block) {
  if (!d.on) return 0xFFu;
  const U4 w = draw_group(rule, d, block);
  uint32_t bits = 0;
#pragma unroll
  for (int c = 0; c < kGroup; ++c) bits |= kept(w, c, d.limit) ? 1u << c : 0u;
  return bits;
}

// Eight neighbouring elements as 16-byte vectors
struct Eight {
  float v[kGroup];
};
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 q;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
  return q;
}
__device__ __forceinline__ Eight unpack(const uint4& a) {       // bf16
  Eight e;
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { e.v[2 * i] = __uint_as_float(w[i] << 16); e.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  return e;
}
__device__ __forceinline__ Eight unpack(const uint4& a, const uint4& b) {
  return {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
          __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
}
__device__ __forceinline__ void store8(bf16* p, const Eight& e) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(e.v[2 * i], e.v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&t);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const Eight& e) {
  reinterpret_cast<float4*>(p)[0] = make_float4(e.v[0], e.v[1], e.v[2], e.v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(e.v[4], e.v[5], e.v[6], e.v[7]);
}
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
#endif

}  // namespace dropout
}  // namespace pbt
