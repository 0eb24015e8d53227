// Dropout of activations, with masks that are drawn where they are needed: y = residual + keep x / (1 - rate).
//
// One pass over x (and residual): 4 or 6 bytes an element in bf16, 8 or 12 in fp32.  A group of eight neighbouring columns shares one
// block of the generator (20 32-bit multiplications with a 64-bit product), so that the draws cost less than the transfers.  80 x 512 x 2048 bf16: 78 us with a residual
// (6.5 TB/s, the measured copy rate), 58 without (5.8 TB/s); 24 x 1024 x 512 fp32 with a residual 25 (6.1).
#include <type_traits>

#include "dropout.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace dropout {
namespace {

int fail(int code, const char* msg) {
  set_last_error(msg);
  return code;
}

template <typename T>
struct Args {
  const T* x; long long x_member, x_row;
  const T* residual; long long residual_member, residual_row;
  T* y;
  uint32_t rows, width, groups;     // groups of a row
  Rule rule;
};

template <typename T>
struct Raw {      // eight elements as they lie in memory
  uint4 a, b;
};
template <typename T>
__device__ __forceinline__ Raw<T> load8(const T* p) {
  Raw<T> r;
  r.a = load16(p);
  if (sizeof(T) == 4) r.b = load16(p + 4);
  return r;
}
__device__ __forceinline__ Eight values(const Raw<bf16>& r) { return unpack(r.a); }
__device__ __forceinline__ Eight values(const Raw<float>& r) { return unpack(r.a, r.b); }

// the residual (or 0) and the element scaled, if it is kept; one rounding
__device__ __forceinline__ float drop(float x, bool in, float scale, float residual) { return fmaf(in ? x : 0.f, scale, residual); }

// Whole groups in 16-byte vectors, U of them a thread, 256 apart, so that all their loads are under way before the first draw.
// FLAT: rows follow one another without gaps, and a group's number in the member is its place, too.
template <typename T, bool RESIDUAL, bool FLAT, int U>
__global__ void __launch_bounds__(256) k_dropout(const Args<T> a) {
  pdl_prologue();
  const int m = blockIdx.y;
  const uint32_t total = a.rows * a.groups, first = blockIdx.x * (256 * U) + threadIdx.x;
  const T* x = a.x + m * a.x_member;
  const T* r = RESIDUAL ? a.residual + m * a.residual_member : nullptr;
  T* y = a.y + (long long)m * a.rows * a.width;
  const Draw d = draw_of(a.rule, m);
  Raw<T> vx[U], vr[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = first + u * 256;
    if (i >= total || i < first) continue;
    long long at_x = (long long)i * kGroup, at_r = at_x;
    if (!FLAT) {
      const uint32_t row = i / a.groups, c = (i - row * a.groups) * kGroup;
      at_x = row * a.x_row + c;
      at_r = row * a.residual_row + c;
    }
    vx[u] = load8(x + at_x);
    if (RESIDUAL) vr[u] = load8(r + at_r);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = first + u * 256;
    if (i >= total || i < first) continue;
    Eight e = values(vx[u]), q = {};
    if (RESIDUAL) q = values(vr[u]);
    if (d.on) {
      const U4 w = draw_group(a.rule, d, i);
#pragma unroll
      for (int c = 0; c < kGroup; ++c) e.v[c] = drop(e.v[c], kept(w, c, d.limit), d.scale, q.v[c]);
    } else if (RESIDUAL) {
#pragma unroll
      for (int c = 0; c < kGroup; ++c) e.v[c] += q.v[c];
    }
    store8(y + (long long)i * kGroup, e);
  }
}

// Any width from 8 on, all activations without gaps (less than 2^31 elements of them): a thread has U vectors of eight elements from a 16-byte boundary, 32
// apart, which belong to two or three groups and one or two rows (the second one perhaps of the next member).  Every lane draws the group that its vector begins
// in; the next vector, the next lane's, begins in the group that follows it, or in the first one of the next row, so that its bits come from there, the last
// lane's from one more draw of the warp.  Only a row's last vector, where it begins inside the last group but one, takes a draw of its own.
// Bound by issue (80 x 512 x 2047 bf16 with a residual 104 us, without 98; 2048 columns take 78 and 58).
template <typename T, bool RESIDUAL, int U>
__global__ void __launch_bounds__(256) k_dropout_odd(const Args<T> a, const uint32_t total, const Divisor by_width, const Divisor by_rows) {
  pdl_prologue();
  const int lane = threadIdx.x & 31;
  const uint32_t v0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * (32 * U) + lane;
  if ((v0 - lane) * kGroup >= total) return;
  Raw<T> vx[U], vr[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t at = (v0 + u * 32) * kGroup;
    if (at + kGroup > total) continue;
    vx[u] = load8(a.x + at);
    if (RESIDUAL) vr[u] = load8(a.residual + at);
  }
  struct Place {
    uint32_t at, row, col, member;
  };
  auto place = [&](int u) {
    Place q;
    q.at = (v0 + u * 32) * kGroup;
    const uint32_t line = quotient(q.at, by_width);
    q.member = quotient(line, by_rows);
    q.row = line - q.member * a.rows;
    q.col = q.at - line * a.width;
    return q;
  };
  uint32_t bits[U + 1], last = 0xFFFFFFFFu;
  float scale[U + 1];
  Draw d = {};
#pragma unroll
  for (int u = 0; u <= U; ++u) {
    const Place q = place(u);
    bits[u] = 0;
    if (q.at >= total) continue;
    if (q.member != last) d = draw_of(a.rule, q.member);
    last = q.member;
    bits[u] = kept_bits(a.rule, d, q.row * a.groups + q.col / kGroup);
    scale[u] = d.on ? d.scale : 1.f;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t across = __shfl_down_sync(0xFFFFFFFFu, bits[u], 1), around = __shfl_sync(0xFFFFFFFFu, bits[u + 1], 0), next = lane == 31 ? around : across;
    const Place q = place(u);
    const uint32_t at = q.at, shift = q.col % kGroup, left = a.width - q.col;
    if (at >= total) continue;
    uint32_t in = bits[u] >> shift;
    float next_scale = scale[u];
    if (left > kGroup) {
      in |= next << (kGroup - shift);               // (without a shift nothing of it is looked at)
    } else {
      if (shift && left > kGroup - shift) in |= kept_bits(a.rule, draw_of(a.rule, q.member), q.row * a.groups + q.col / kGroup + 1) << (kGroup - shift);
      if (left < kGroup) {
        in = (in & ((1u << left) - 1u)) | next << left;
        if (q.row + 1 == a.rows && at + left < total) {
          const Draw other = draw_of(a.rule, q.member + 1);
          next_scale = other.on ? other.scale : 1.f;
        }
      }
    }
    if (at + kGroup <= total) {
      Eight e = values(vx[u]), r = {};
      if (RESIDUAL) r = values(vr[u]);
      if (next_scale == scale[u]) {
#pragma unroll
        for (int c = 0; c < kGroup; ++c) e.v[c] = drop(e.v[c], in >> c & 1u, scale[u], r.v[c]);
      } else {
#pragma unroll
        for (int c = 0; c < kGroup; ++c) e.v[c] = drop(e.v[c], in >> c & 1u, c < left ? scale[u] : next_scale, r.v[c]);
      }
      store8(a.y + at, e);
    } else {
      for (uint32_t c = 0; at + c < total; ++c) {
        store(a.y + at + c, drop(as_float(a.x[at + c]), in >> c & 1u, c < left ? scale[u] : next_scale, RESIDUAL ? as_float(a.residual[at + c]) : 0.f));
      }
    }
  }
}

// Any width, strides and alignment: a thread has a group.
template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(256) k_dropout_strided(const Args<T> a) {
  pdl_prologue();
  const int m = blockIdx.y;
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (uint64_t)a.rows * a.groups) return;
  const uint32_t row = (uint32_t)i / a.groups, c0 = ((uint32_t)i - row * a.groups) * kGroup, n = min(a.width - c0, (uint32_t)kGroup);
  const T* x = a.x + m * a.x_member + row * a.x_row + c0;
  const T* r = RESIDUAL ? a.residual + m * a.residual_member + row * a.residual_row + c0 : nullptr;
  T* y = a.y + ((long long)m * a.rows + row) * a.width + c0;
  const Draw d = draw_of(a.rule, m);
  const uint32_t bits = kept_bits(a.rule, d, (uint32_t)i);
  const float scale = d.on ? d.scale : 1.f;
#pragma unroll
  for (int c = 0; c < kGroup; ++c) {
    if (c >= n) break;
    store(y + c, drop(as_float(x[c]), bits >> c & 1u, scale, RESIDUAL ? as_float(r[c]) : 0.f));
  }
}

template <typename T, bool RESIDUAL>
cudaError_t launch(const pbt_dropout_desc* d, cudaStream_t s) {
  const uint32_t groups = (uint32_t)((d->width + kGroup - 1) / kGroup);
  const Args<T> a = {(const T*)d->x, d->x_member, d->x_row, (const T*)d->residual, d->residual_member, d->residual_row, (T*)d->y,
                     (uint32_t)d->rows, (uint32_t)d->width, groups, rule_of(d->rule)};
  const uint64_t per_member = (uint64_t)d->rows * groups;
  const long long cells = (long long)d->rows * d->width, step = 16 / sizeof(T);
  const bool many = d->members > 1;
  auto whole = [&](const void* p, long long member, long long row) {       // vectors at every group
    return ((uintptr_t)p & 15) == 0 && (d->rows == 1 || row % step == 0) && (!many || member % step == 0);
  };
  auto gapless = [&](long long member, long long row) { return (d->rows == 1 || row == d->width) && (!many || member == cells); };
  const bool vectors = d->width % kGroup == 0 && ((uintptr_t)d->y & 15) == 0 && whole(d->x, d->x_member, d->x_row) &&
                       (!RESIDUAL || whole(d->residual, d->residual_member, d->residual_row));
  auto grid = [&](int per_block) { return dim3((unsigned)((per_member + per_block - 1) / per_block), (unsigned)d->members); };
  if (vectors) {
    const bool flat = d->rows == 1 || (d->x_row == d->width && (!RESIDUAL || d->residual_row == d->width));
    // Groups of a thread: bf16 takes two or four, which share the generator's first rounds (they go by the member and the step alone) and keep more
    // bytes under way; fp32, twice the bytes a group, one.  80 x 512 x 2048 bf16 with residual (without): one 92.1 us (70.8), two 83.1 (65.0), three 81.3
    // (62.4), four 77.7 (58.1), and a plain copy of 4 bytes an element 52.4; 16 x 256 x 1024: 5.4, 5.1, 5.5, 5.5; 80 x 512 x 2048 fp32 146.3 (100.1) to 146.6 (101.0).
    const uint64_t all = per_member * d->members, fill = 148ull * 2048;       // the GPU's threads
    const int each = sizeof(T) == 4 || all < fill ? 1 : all < 4 * fill ? 2 : 4;
    auto go = [&](auto is_flat) {
      constexpr bool F = decltype(is_flat)::value;
      if (each == 4) return launch_with(grid(1024), 256, 0, s)(k_dropout<T, RESIDUAL, F, 4>, a);
      if (each == 2) return launch_with(grid(512), 256, 0, s)(k_dropout<T, RESIDUAL, F, 2>, a);
      return launch_with(grid(256), 256, 0, s)(k_dropout<T, RESIDUAL, F, 1>, a);
    };
    return flat ? go(std::true_type()) : go(std::false_type());
  }
  const long long total = cells * d->members;
  const uintptr_t bases = (uintptr_t)d->x | (uintptr_t)d->y | (RESIDUAL ? (uintptr_t)d->residual : 0);
  if (d->width >= kGroup && (bases & 15) == 0 && total < 0x7FFF0000ll && gapless(d->x_member, d->x_row) &&
      (!RESIDUAL || gapless(d->residual_member, d->residual_row))) {
    // Vectors of a thread, once the GPU has its fill of threads with them: 80 x 512 x 2047 bf16 with residual (without) one 141 us (138), two 114 (109), three
    // 104 (98), four 105 (95); fp32 151 (135), 147 (112), 150 (105), 165 (111).
    constexpr int U = sizeof(T) == 4 && RESIDUAL ? 2 : 3;
    const Divisor by_width = divisor((uint32_t)d->width), by_rows = divisor((uint32_t)d->rows);
    auto blocks = [&](int each) { return (unsigned)((total + 256 * kGroup * each - 1) / (256 * kGroup * each)); };
    if (total >= 148ll * 2048 * kGroup * 2) return launch_with(blocks(U), 256, 0, s)(k_dropout_odd<T, RESIDUAL, U>, a, (uint32_t)total, by_width, by_rows);
    return launch_with(blocks(1), 256, 0, s)(k_dropout_odd<T, RESIDUAL, 1>, a, (uint32_t)total, by_width, by_rows);
  }
  return launch_with(grid(256), 256, 0, s)(k_dropout_strided<T, RESIDUAL>, a);
}
template <typename T>
cudaError_t launch(const pbt_dropout_desc* d, cudaStream_t s) { return d->residual ? launch<T, true>(d, s) : launch<T, false>(d, s); }

}  // namespace

int check_rule(const pbt_drop_rule* r, long long members, long long rows, long long width) {
  if (r->site < 0 || r->site > (1 << 30)) return fail(PBT_ERR_INVALID_ARG, "a dropout's site must lie in [0, 2^30]");
  if (r->first_member < 0 || (long long)r->first_member + members > 0x7FFFFFFFll)
    return fail(PBT_ERR_INVALID_ARG, "first_member must be >= 0, and every member's index below 2^31");
  if (!r->rate && !(r->rate_all >= 0.f && r->rate_all <= 1.f)) return fail(PBT_ERR_INVALID_ARG, "a dropout rate must lie in [0, 1]");
  if (rows * ((width + kGroup - 1) / kGroup) > 0xFFFFFFFFll) return fail(PBT_ERR_UNSUPPORTED, "rows times ceil(width / 8) must stay below 2^32 (the generator's block number)");
  return PBT_OK;
}

}  // namespace dropout
}  // namespace pbt

extern "C" int pbt_dropout(const pbt_dropout_desc* d, void* stream) {
  using namespace pbt;
  using namespace pbt::dropout;
  if (!d) return fail(PBT_ERR_INVALID_ARG, "desc is NULL");
  if (d->members < 1 || d->rows < 0 || d->width < 1) return fail(PBT_ERR_INVALID_ARG, "members and width must be positive, rows >= 0");
  if (d->members > 65535) return fail(PBT_ERR_UNSUPPORTED, "more than 65535 members");
  if (d->dtype != 0 && d->dtype != 1) return fail(PBT_ERR_UNSUPPORTED, "activations are float or bfloat16");
  const int rc = check_rule(&d->rule, d->members, d->rows, d->width);
  if (rc) return rc;
  if (!d->rows) return PBT_OK;
  if (!d->x || !d->y) return fail(PBT_ERR_INVALID_ARG, "x or y is NULL");
  const cudaError_t e = d->dtype ? launch<bf16>(d, (cudaStream_t)stream) : launch<float>(d, (cudaStream_t)stream);
  return e == cudaSuccess ? PBT_OK : fail(PBT_ERR_CUDA, cudaGetErrorString(e));
}
