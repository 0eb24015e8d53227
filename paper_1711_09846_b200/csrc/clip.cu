// Global gradient norm over many tensors, and clipping, per group (population member):
//   norm_g = sqrt(sum over the tensors of group g, all elements: e^2),   dst = src * min(1, limit_g / norm_g).
//
// Memory-bound; the floor is ONE read and one write of every element, which asks for the gradients to stay on the chip
// between the two.
//
// Groups that fit the shared memory of all SMs together (30 MB): one cooperative launch goes through them in waves of as many
// whole groups as fit.  In a wave every CTA reads its share of the elements, keeps it in shared memory, leaves its sums of
// squares, meets the others at a grid barrier, and scales what it kept.  What is kept comes by bulk copies, all of them asked
// for when the wave begins (208 KB per SM in flight); while a CTA waits at the barrier the first bytes of its next wave are
// on their way into L2.
//
// Larger groups are streamed twice, all of them together: sums of 64 KB chunks, the groups' factors, and the scaling.  Keeping
// half of a 58.7 MB group in shared memory and the rest in L2 saves a third of the traffic, but meeting after each group costs
// more (80 such groups: 2.57 ms, 12 us to read a group, 10.5 to write it and 9 to meet and to find the factor; with two teams of
// CTAs on alternate groups 2.90 ms, L2 does not hold both).
//
// Sums are added in a fixed order (no atomics on values), so a run is reproducible bit for bit.
#include <stdio.h>

#include <algorithm>
#include <new>
#include <vector>

#include "tc_common.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace {

constexpr int kClipThreads = 512;
constexpr int kClipUnroll = 8;             // 16-byte loads of a thread in flight: 64 KB per SM
constexpr int kClipCtas = 148;             // one per SM
constexpr int kClipKeep = 208 * 1024;      // bytes of gradients a CTA keeps in shared memory
constexpr long long kClipWave = (long long)kClipCtas * (kClipKeep - 4096);   // bytes of a wave of whole groups
constexpr int kClipShare = 4096;           // smallest share of a CTA in a wave
constexpr int kClipPieces = 64;            // table entries of a wave that are fetched ahead of it
constexpr int kClipRuns = 32;              // groups of a CTA's share that are worked on together
constexpr int kClipAhead = 96 * 1024;      // bytes of the next wave asked for at the barrier
constexpr unsigned int kClipPolls = 1u << 24;

// A run of elements of one tensor that one CTA handles in one wave.
struct __align__(16) ClipPiece {
  const char* src;
  char* dst;
  int count;       // elements
  int kept;        // where the elements are kept in shared memory (same alignment as src), or -1
  int group2;      // 2 * group + (1: bfloat16)
  int sum;         // where the CTA's sum of this group goes
  int sum_begin, sum_end;   // the group's sums
  int pad[2];
  __device__ bool bf() const { return group2 & 1; }
};

struct ClipArgs {
  const ClipPiece* pieces;
  const int* first;        // [waves * CTAs + 1] first piece of every (wave, CTA)
  const int* empty;        // [groups] 1: the group has no elements
  double* sums;
  unsigned int* barrier;   // arrivals, exits, status
  int n_waves, n_groups;
  float limit;
  const float* limits;
  float* norms;
};

__device__ __forceinline__ float clip_load(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float clip_load(const float* p) { return *p; }
__device__ __forceinline__ void clip_store(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void clip_store(float* p, float v) { *p = v; }

template <typename S>
__device__ __forceinline__ S clip_warp_sum(S v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// 16 bytes of gradients
template <typename T> struct Quad;
template <> struct Quad<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void get(const uint4& r, float* f) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 put(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <> struct Quad<bf16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void get(const uint4& r, float* f) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&t);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// A piece is its elements up to the first 16-byte boundary, 16-byte vectors, and the rest.
struct ClipSpan { int head, vectors, tail; };   // elements, vectors, first element of the rest
template <typename T>
__device__ __forceinline__ ClipSpan clip_span(const ClipPiece& p) {
  ClipSpan s;
  s.head = min(p.count, (int)((16 - ((uintptr_t)p.src & 15)) & 15) / (int)sizeof(T));
  s.vectors = (p.count - s.head) / Quad<T>::n;
  s.tail = s.head + s.vectors * Quad<T>::n;
  return s;
}

// Pieces of a few hundred elements go to one warp each, in turn, so that a CTA has many of them in flight: the thread's
// first vector and the distance to its next, or nothing for it to do.
__device__ __forceinline__ bool clip_lanes(const ClipPiece& p, int index, int& lane, int& lanes) {
  lane = threadIdx.x;
  lanes = kClipThreads;
  if (p.count > 1024) return true;
  lane &= 31;
  lanes = 32;
  return (int)(threadIdx.x >> 5) == (index & (kClipThreads / 32 - 1));
}

template <typename T>
__device__ __forceinline__ void clip_add(const uint4& v, float* sum) {
  float f[Quad<T>::n];
  Quad<T>::get(v, f);
#pragma unroll
  for (int e = 0; e < Quad<T>::n; ++e) sum[e & 3] = __fmaf_rn(f[e], f[e], sum[e & 3]);
}

// Pieces that a bulk copy brings (those of the table's fetched entries that are kept and not small): their vectors.
__device__ __forceinline__ bool clip_bulk(const ClipPiece& p, int index) { return index < kClipPieces && p.kept >= 0 && p.count > 1024; }
template <typename T>
__device__ __forceinline__ void clip_ask(const ClipPiece& p, char* keep, uint64_t* bar) {
  const ClipSpan s = clip_span<T>(p);
  const uint32_t bytes = (uint32_t)s.vectors * 16, to = tc::smem_u32(keep + p.kept + s.head * sizeof(T));
  tc::mbar_expect_tx(bar, bytes);
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(to), "l"(p.src + s.head * sizeof(T)), "r"(bytes), "r"(tc::smem_u32(bar)) : "memory");
}
template <typename T>
__device__ __forceinline__ float clip_sum_kept(const ClipPiece& p, char* keep) {
  const ClipSpan s = clip_span<T>(p);
  const T* g = reinterpret_cast<const T*>(p.src);
  T* k = reinterpret_cast<T*>(keep + p.kept);
  const uint4* kv = reinterpret_cast<const uint4*>(k + s.head);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const int i0 = threadIdx.x, loose = s.head + p.count - s.tail;
  if (i0 < loose) {
    const int at = i0 < s.head ? i0 : s.tail + i0 - s.head;
    const T v = g[at];
    k[at] = v;
    const float f = clip_load(&v);
    sum[0] = f * f;
  }
#pragma unroll 4
  for (int i = i0; i < s.vectors; i += kClipThreads) clip_add<T>(kv[i], sum);
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

template <typename T>
__device__ __forceinline__ float clip_read(const ClipPiece& p, int index, char* keep) {
  int i, lanes;
  if (!clip_lanes(p, index, i, lanes)) return 0.f;
  const ClipSpan s = clip_span<T>(p);
  const T* g = reinterpret_cast<const T*>(p.src);
  T* k = reinterpret_cast<T*>(keep + p.kept);
  const uint4* gv = reinterpret_cast<const uint4*>(g + s.head);
  uint4* kv = reinterpret_cast<uint4*>(k + s.head);
  const bool kept = p.kept >= 0;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const int loose = s.head + p.count - s.tail;      // fewer than 16 elements
  if (i < loose) {
    const int at = i < s.head ? i : s.tail + i - s.head;
    const T v = g[at];
    if (kept) k[at] = v;
    const float f = clip_load(&v);
    sum[0] = f * f;
  }
  if (lanes == kClipThreads)
    for (; i + (kClipUnroll - 1) * kClipThreads < s.vectors; i += kClipUnroll * kClipThreads) {
      uint4 v[kClipUnroll];
#pragma unroll
      for (int u = 0; u < kClipUnroll; ++u) v[u] = __ldcg(gv + i + u * kClipThreads);
#pragma unroll
      for (int u = 0; u < kClipUnroll; ++u) {
        if (kept) kv[i + u * kClipThreads] = v[u];
        clip_add<T>(v[u], sum);
      }
    }
#pragma unroll 4
  for (; i < s.vectors; i += lanes) {
    const uint4 v = __ldcg(gv + i);
    if (kept) kv[i] = v;
    clip_add<T>(v, sum);
  }
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

template <typename T>
__device__ __noinline__ double clip_read_wide(const ClipPiece& p) {      // by one warp
  const T* g = reinterpret_cast<const T*>(p.src);
  double sum = 0.0;
  for (int i = threadIdx.x & 31; i < p.count; i += 32) {
    const double v = clip_load(g + i);
    sum = fma(v, v, sum);
  }
  return sum;
}

template <typename T>
__device__ __forceinline__ uint4 clip_scaled(const uint4& v, float f) {
  float e[Quad<T>::n];
  Quad<T>::get(v, e);
#pragma unroll
  for (int j = 0; j < Quad<T>::n; ++j) e[j] *= f;
  return Quad<T>::put(e);
}

template <typename T>
__device__ __forceinline__ void clip_write(const ClipPiece& p, int index, const char* keep, float f) {
  int i, lanes;
  if (!clip_lanes(p, index, i, lanes)) return;
  const ClipSpan s = clip_span<T>(p);
  const T* g = p.kept >= 0 ? reinterpret_cast<const T*>(keep + p.kept) : reinterpret_cast<const T*>(p.src);
  T* o = reinterpret_cast<T*>(p.dst);
  const uint4* gv = reinterpret_cast<const uint4*>(g + s.head);
  const int loose = s.head + p.count - s.tail;
  if (i < loose) {
    const int at = i < s.head ? i : s.tail + i - s.head;
    clip_store(o + at, clip_load(g + at) * f);
  }
  uint4* ov = reinterpret_cast<uint4*>(o + s.head);
  if (((uintptr_t)ov & 15) != 0) {     // a destination of another alignment than its source: element by element
    for (; i < s.vectors; i += lanes) {
      float e[Quad<T>::n];
      Quad<T>::get(gv[i], e);
#pragma unroll
      for (int j = 0; j < Quad<T>::n; ++j) clip_store(o + s.head + i * Quad<T>::n + j, e[j] * f);
    }
    return;
  }
  if (lanes == kClipThreads)
    for (; i + (kClipUnroll - 1) * kClipThreads < s.vectors; i += kClipUnroll * kClipThreads) {
      uint4 v[kClipUnroll];
#pragma unroll
      for (int u = 0; u < kClipUnroll; ++u) v[u] = gv[i + u * kClipThreads];
#pragma unroll
      for (int u = 0; u < kClipUnroll; ++u) __stcs(ov + i + u * kClipThreads, clip_scaled<T>(v[u], f));
    }
#pragma unroll 4
  for (; i < s.vectors; i += lanes) __stcs(ov + i, clip_scaled<T>(gv[i], f));
}

// min(1, limit / norm); a NaN norm makes the factor NaN (a diverged member stays visible), an infinite limit never clips
__device__ __forceinline__ float clip_factor(float limit, float norm) {
  if (isinf(limit) && limit > 0.f) return 1.f;
  if (norm <= limit) return 1.f;
  return __fdiv_rn(limit, norm);
}

// Arrive at the grid barrier (thread 0, after the block's sums are written and fenced), and wait until `target` CTAs have arrived.
// The wait is bounded; on expiry the status word is set, everybody leaves, and the norms that are missing stay NaN.
__device__ __forceinline__ void clip_arrive(const ClipArgs& a) {
  __threadfence();
  atomicAdd(a.barrier, 1u);
}
__device__ __forceinline__ bool clip_wait(const ClipArgs& a, unsigned int target) {
  volatile unsigned int* count = a.barrier;
  volatile unsigned int* status = a.barrier + 2;
  for (unsigned int i = 0; *count < target; ++i) {
    if (i > kClipPolls || (i > 64 && *status)) {
      *status = PBT_ERR_TIMEOUT;
      return false;
    }
    __nanosleep(20);
  }
  __threadfence();
  return true;
}

constexpr int kClipWarps = kClipThreads / 32;

__global__ void __launch_bounds__(kClipThreads, 1) k_clip(const ClipArgs a) {
  pdl_prologue();
  extern __shared__ __align__(16) char keep[];
  __shared__ ClipPiece near[2][kClipPieces];
  __shared__ float warp_sums[kClipRuns][kClipWarps];
  __shared__ int run_first[kClipRuns + 1];
  __shared__ float factor[kClipRuns];
  __shared__ uint64_t arrived[kClipPieces];     // bulk copies of the fetched entries
  __shared__ int go, wide, gave_up;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, b = blockIdx.x, ctas = gridDim.x;
  if (b == 0)
    for (int g = tid; g < a.n_groups; g += kClipThreads) a.norms[g] = a.empty[g] ? 0.f : __int_as_float(0x7FC00000);
  auto fetch = [&](int w) {       // 16 bytes a thread
    if (w < a.n_waves) {
      const int first = a.first[w * ctas + b], n = min(a.first[w * ctas + b + 1] - first, kClipPieces) * (int)(sizeof(ClipPiece) / 16);
      for (int i = tid; i < n; i += kClipThreads) reinterpret_cast<uint4*>(near[w & 1])[i] = reinterpret_cast<const uint4*>(a.pieces + first)[i];
    }
  };
  fetch(0);
  if (tid < kClipPieces) tc::mbar_init(&arrived[tid], 1);
  if (tid == 0) gave_up = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  unsigned long long turns = 0;      // bit i: parity of the next use of arrived[i]
  __syncthreads();
  for (int w = 0; w < a.n_waves; ++w) {
    const int first = a.first[w * ctas + b], n = a.first[w * ctas + b + 1] - first;
    auto piece = [&](int i) -> const ClipPiece& { return i < kClipPieces ? near[w & 1][i] : a.pieces[first + i]; };
    const int asked = min(n, kClipPieces);
    if (tid < asked && clip_bulk(piece(tid), tid)) {
      tc::fence_async_smem();        // the wave before has read these bytes (and all threads have met since)
      if (piece(tid).bf()) clip_ask<bf16>(piece(tid), keep, &arrived[tid]);
      else clip_ask<float>(piece(tid), keep, &arrived[tid]);
    }
    // A run is the CTA's pieces of one group.  kClipRuns of them at a time: the warps add up squares on their own and meet
    // once, whatever the number of runs.
    for (int i = 0; i < n;) {
      int runs = 0;
      const int start = i;
      while (i < n) {
        const int group = piece(i).group2 >> 1;
        const int begin = i;
        float sum = 0.f;
        if (runs == kClipRuns) break;
        if (tid == 0) run_first[runs] = i;
        for (; i < n; ++i) {
          const ClipPiece& p = piece(i);
          if (p.group2 >> 1 != group) break;
          if (!clip_bulk(p, i)) sum += p.bf() ? clip_read<bf16>(p, i, keep) : clip_read<float>(p, i, keep);
        }
        for (int k = begin; k < min(i, asked); ++k) {      // what the bulk copies have brought meanwhile
          const ClipPiece& p = piece(k);
          if (!clip_bulk(p, k)) continue;
          if (!tc::mbar_wait(&arrived[k], (uint32_t)(turns >> k) & 1u, &gave_up)) gave_up = 1;
          sum += p.bf() ? clip_sum_kept<bf16>(p, keep) : clip_sum_kept<float>(p, keep);
        }
        sum = clip_warp_sum(sum);
        if (lane == 0) warp_sums[runs][warp] = sum;
        ++runs;
      }
      if (tid == 0) {
        run_first[runs] = i;
        wide = 0;
      }
      __syncthreads();
      if (tid < runs) {
        float t = warp_sums[tid][0];
        for (int k = 1; k < kClipWarps; ++k) t += warp_sums[tid][k];
        // Squares are fp32; where their sum leaves the range in which that is exact to rounding (elements beyond 1.8e19, or
        // all below 1e-15), the run is summed again in fp64 below, so that only the norm itself can overflow.
        if (t > 1e-30f && t < 3e38f) a.sums[piece(run_first[tid]).sum] = t;
        else wide = 1;
      }
      __syncthreads();
      if (wide)
        for (int q = warp; q < runs; q += kClipWarps) {
          float t = lane < kClipWarps ? warp_sums[q][lane] : 0.f;
          t = clip_warp_sum(t);
          if (t > 1e-30f && t < 3e38f) continue;
          double d = 0.0;
          for (int k = run_first[q]; k < run_first[q + 1]; ++k) d += piece(k).bf() ? clip_read_wide<bf16>(piece(k)) : clip_read_wide<float>(piece(k));
          d = clip_warp_sum(d);
          if (lane == 0) a.sums[piece(run_first[q]).sum] = d;
        }
      if (wide || i < n || start > 0) __syncthreads();     // before the tables are used again, and before thread 0 arrives
    }
    for (int k = 0; k < asked; ++k)
      if (clip_bulk(piece(k), k)) turns ^= 1ull << k;
    __threadfence();
    __syncthreads();
    if (tid == 0) clip_arrive(a);
    fetch(w + 1);
    __syncthreads();
    if (w + 1 < a.n_waves) {
      const int next = a.first[(w + 1) * ctas + b], m = a.first[(w + 1) * ctas + b + 1] - next;
      if (tid < min(m, kClipPieces)) {
        const ClipPiece& p = near[(w + 1) & 1][tid];
        const uintptr_t from = ((uintptr_t)p.src + 15) & ~(uintptr_t)15;
        long long bytes = (long long)((uintptr_t)p.src + (long long)p.count * (p.bf() ? 2 : 4) - from) & ~15ll;
        if (bytes > kClipAhead) bytes = kClipAhead;
        if (bytes >= 16 && p.kept >= 0 && p.kept < kClipAhead)
          asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"((uint32_t)bytes) : "memory");
      }
    }
    if (tid == 0) {
      if (gave_up) a.barrier[2] = PBT_ERR_TIMEOUT;
      go = !gave_up && clip_wait(a, (unsigned int)(w + 1) * ctas);
    }
    __syncthreads();
    if (!go) break;
    for (int i = 0; i < n;) {
      // the runs' factors, a warp each, then all of their elements
      const int start = i;
      int runs = 0;
      for (int k = i; k < n;) {
        const int group = piece(k).group2 >> 1;
        if (runs == kClipRuns) break;
        if (runs % kClipWarps == warp) {
          const ClipPiece& p = piece(k);
          const float limit = a.limits ? __ldg(a.limits + group) : a.limit;
          double s = 0.0;
#pragma unroll 8
          for (int q = p.sum_begin + lane; q < p.sum_end; q += 32) s += __ldcg(a.sums + q);
          s = clip_warp_sum(s);
          const float norm = (float)sqrt(s);
          if (lane == 0) {
            factor[runs] = clip_factor(limit, norm);
            if (p.sum == p.sum_begin) a.norms[group] = norm;     // the CTA that holds the group's first sum
          }
        }
        ++runs;
        while (k < n && piece(k).group2 >> 1 == group) ++k;
      }
      __syncthreads();
      for (int q = 0; q < runs; ++q) {
        const int group = piece(i).group2 >> 1;
        const float f = factor[q];
        for (; i < n; ++i) {
          const ClipPiece& p = piece(i);
          if (p.group2 >> 1 != group) break;
          if (f == 1.f && p.src == p.dst) continue;
          if (p.bf()) clip_write<bf16>(p, i, keep, f);
          else clip_write<float>(p, i, keep, f);
        }
      }
      if (i < n || start > 0) __syncthreads();     // `factor` is written again
    }
    __syncthreads();     // `keep` and the tables are written again by the next wave
  }
  // the last CTA to leave puts the barrier back for the next run
  if (tid == 0) {
    __threadfence();
    if (atomicAdd(a.barrier + 1, 1u) == (unsigned int)ctas - 1) {
      a.barrier[0] = 0;
      a.barrier[1] = 0;
    }
  }
}

// ---- groups that do not fit: one block per chunk ----
constexpr int kStreamThreads = 256;
constexpr int kStreamChunk = 64 * 1024;      // bytes

struct StreamArgs {
  const ClipPiece* chunks;       // kept is -1, sum the chunk's own index
  const int* groups;             // the large groups, and for each its sums' range
  int n_chunks, n_groups;
  double* sums;
  float* factors;                // of every group of the call
  float limit;
  const float* limits;
  float* norms;
};

template <typename T>
__device__ __forceinline__ float stream_sum(const ClipPiece& p) {
  const ClipSpan s = clip_span<T>(p);
  const T* g = reinterpret_cast<const T*>(p.src);
  const uint4* gv = reinterpret_cast<const uint4*>(g + s.head);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  int i = threadIdx.x;
  for (; i + 7 * kStreamThreads < s.vectors; i += 8 * kStreamThreads) {
    uint4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = __ldcs(gv + i + u * kStreamThreads);
#pragma unroll
    for (int u = 0; u < 8; ++u) clip_add<T>(v[u], sum);
  }
  for (; i < s.vectors; i += kStreamThreads) clip_add<T>(gv[i], sum);
  const int loose = s.head + p.count - s.tail;
  if ((int)threadIdx.x < loose) {
    const float f = clip_load(g + ((int)threadIdx.x < s.head ? threadIdx.x : s.tail + threadIdx.x - s.head));
    sum[0] = __fmaf_rn(f, f, sum[0]);
  }
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}
template <typename T>
__device__ __noinline__ double stream_sum_wide(const ClipPiece& p) {
  const T* g = reinterpret_cast<const T*>(p.src);
  double sum = 0.0;
  for (int i = threadIdx.x; i < p.count; i += kStreamThreads) {
    const double v = clip_load(g + i);
    sum = fma(v, v, sum);
  }
  return sum;
}

__global__ void __launch_bounds__(kStreamThreads) k_clip_sums(const StreamArgs a) {
  pdl_prologue();
  __shared__ float part[kStreamThreads / 32];
  __shared__ double part_wide[kStreamThreads / 32];
  const ClipPiece p = a.chunks[blockIdx.x];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float s = clip_warp_sum(p.bf() ? stream_sum<bf16>(p) : stream_sum<float>(p));
  if (lane == 0) part[warp] = s;
  __syncthreads();
  float t = part[0];
#pragma unroll
  for (int k = 1; k < kStreamThreads / 32; ++k) t += part[k];
  if (t > 1e-30f && t < 3e38f) {      // (as in k_clip)
    if (threadIdx.x == 0) a.sums[blockIdx.x] = t;
    return;
  }
  const double d = clip_warp_sum(p.bf() ? stream_sum_wide<bf16>(p) : stream_sum_wide<float>(p));
  if (lane == 0) part_wide[warp] = d;
  __syncthreads();
  if (threadIdx.x == 0) {
    double all = part_wide[0];
    for (int k = 1; k < kStreamThreads / 32; ++k) all += part_wide[k];
    a.sums[blockIdx.x] = all;
  }
}

__global__ void __launch_bounds__(kStreamThreads) k_clip_factors(const StreamArgs a) {
  pdl_prologue();
  __shared__ double part[kStreamThreads / 32];
  const int group = a.groups[3 * blockIdx.x], begin = a.groups[3 * blockIdx.x + 1], end = a.groups[3 * blockIdx.x + 2];
  double s = 0.0;
  for (int q = begin + threadIdx.x; q < end; q += kStreamThreads) s += a.sums[q];
  s = clip_warp_sum(s);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < kStreamThreads / 32; ++k) s += part[k];
    const float norm = (float)sqrt(s);
    a.norms[group] = norm;
    a.factors[group] = clip_factor(a.limits ? a.limits[group] : a.limit, norm);
  }
}

template <typename T>
__device__ __forceinline__ void stream_scale(const ClipPiece& p, float f) {
  const ClipSpan s = clip_span<T>(p);
  const T* g = reinterpret_cast<const T*>(p.src);
  T* o = reinterpret_cast<T*>(p.dst);
  const uint4* gv = reinterpret_cast<const uint4*>(g + s.head);
  uint4* ov = reinterpret_cast<uint4*>(o + s.head);
  const int loose = s.head + p.count - s.tail;
  if ((int)threadIdx.x < loose) {
    const int at = (int)threadIdx.x < s.head ? threadIdx.x : s.tail + threadIdx.x - s.head;
    clip_store(o + at, clip_load(g + at) * f);
  }
  int i = threadIdx.x;
  if (((uintptr_t)ov & 15) != 0) {     // a destination of another alignment than its source: element by element
    for (; i < s.vectors; i += kStreamThreads) {
      float e[Quad<T>::n];
      Quad<T>::get(gv[i], e);
#pragma unroll
      for (int j = 0; j < Quad<T>::n; ++j) clip_store(o + s.head + i * Quad<T>::n + j, e[j] * f);
    }
    return;
  }
  for (; i + 3 * kStreamThreads < s.vectors; i += 4 * kStreamThreads) {
    uint4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = __ldcs(gv + i + u * kStreamThreads);
#pragma unroll
    for (int u = 0; u < 4; ++u) __stcs(ov + i + u * kStreamThreads, clip_scaled<T>(v[u], f));
  }
  for (; i < s.vectors; i += kStreamThreads) __stcs(ov + i, clip_scaled<T>(gv[i], f));
}

// from the last chunk to the first: the last ones that k_clip_sums has read are still in L2
__global__ void __launch_bounds__(kStreamThreads) k_clip_scale(const StreamArgs a) {
  pdl_prologue();
  const ClipPiece p = a.chunks[a.n_chunks - 1 - (int)blockIdx.x];
  const float f = __ldg(a.factors + (p.group2 >> 1));
  if (f == 1.f && p.src == p.dst) return;
  if (p.bf()) stream_scale<bf16>(p, f);
  else stream_scale<float>(p, f);
}

int clip_fail(int code, const char* msg) {
  set_last_error(msg);
  return code;
}

size_t clip_align(size_t n) { return (n + 255) & ~(size_t)255; }

int clip_check(const pbt_clip_tensor* t, int n, int n_groups) {
  if (n < 0 || n_groups < 1 || n_groups > (1 << 20)) return clip_fail(PBT_ERR_INVALID_ARG, "n_tensors must be >= 0 and n_groups in [1, 2^20]");
  if (n > 0 && !t) return clip_fail(PBT_ERR_INVALID_ARG, "tensors is NULL");
  for (int i = 0; i < n; ++i) {
    if (t[i].numel < 0 || (t[i].numel > 0 && (!t[i].src || !t[i].dst)))
      return clip_fail(PBT_ERR_INVALID_ARG, "a gradient tensor has a negative size or a NULL pointer");
    if (t[i].numel > (1ll << 46)) return clip_fail(PBT_ERR_INVALID_ARG, "a gradient tensor is larger than any memory");
    if (t[i].dtype != 0 && t[i].dtype != 1) return clip_fail(PBT_ERR_UNSUPPORTED, "gradient tensors are float or bfloat16");
    if (t[i].group < 0 || t[i].group >= n_groups) return clip_fail(PBT_ERR_INVALID_ARG, "a tensor's group is out of range");
    const uintptr_t esz = t[i].dtype ? 2 : 4;
    if (((uintptr_t)t[i].src % esz) || ((uintptr_t)t[i].dst % esz))
      return clip_fail(PBT_ERR_INVALID_ARG, "a gradient tensor is not aligned to its element size");
  }
  return PBT_OK;
}

// Who handles what: waves of whole groups, every wave's bytes dealt to the CTAs in equal consecutive shares.
struct ClipTable {
  std::vector<ClipPiece> pieces, chunks;      // of the waves, of the streamed groups
  std::vector<int> first, empty, large;       // large: (group, first sum, end) of every streamed group
  int n_sums = 0;
  int n_waves = 0, ctas = 1;
};
bool clip_table(const pbt_clip_tensor* t, int n_tensors, int n_groups, ClipTable* out) {
  std::vector<int> order;
  std::vector<long long> group_bytes(n_groups, 0);
  long long total = 0;
  for (int i = 0; i < n_tensors; ++i)
    if (t[i].numel) {
      order.push_back(i);
      group_bytes[t[i].group] += t[i].numel * (t[i].dtype ? 2 : 4);
      total += t[i].numel * (t[i].dtype ? 2 : 4);
    }
  if (total > (1ll << 40)) return false;
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return t[a].group < t[b].group; });
  for (int i : order) {
    const pbt_clip_tensor& x = t[i];
    if (group_bytes[x.group] <= kClipWave) continue;
    const long long esz = x.dtype ? 2 : 4;
    if (out->large.empty() || out->large[out->large.size() - 3] != x.group) {
      const int at = (int)out->chunks.size();
      out->large.insert(out->large.end(), {x.group, at, at});
    }
    for (long long done = 0; done < x.numel;) {
      const char* src = (const char*)x.src + done * esz;
      const long long take = std::min(x.numel - done, (kStreamChunk - (long long)((uintptr_t)src & 15)) / esz);   // chunks end on 16-byte boundaries
      const int at = (int)out->chunks.size();
      out->chunks.push_back({src, (char*)x.dst + done * esz, (int)take, -1, x.group * 2 + x.dtype, at, 0, 0, {0, 0}});
      done += take;
    }
    out->large.back() = (int)out->chunks.size();
  }
  order.erase(std::remove_if(order.begin(), order.end(), [&](int i) { return group_bytes[t[i].group] > kClipWave; }), order.end());
  std::vector<long long> wave_bytes;
  std::vector<size_t> wave_end;          // in `order`
  for (size_t i = 0; i < order.size();) {
    const int g = t[order[i]].group;
    size_t e = i;
    while (e < order.size() && t[order[e]].group == g) ++e;
    if (wave_bytes.empty() || wave_bytes.back() + group_bytes[g] > kClipWave) {
      wave_bytes.push_back(0);
      wave_end.push_back(i);
    }
    wave_bytes.back() += group_bytes[g];
    wave_end.back() = e;
    i = e;
  }
  out->n_waves = (int)wave_bytes.size();
  long long most = 0;
  for (long long b : wave_bytes) most = std::max(most, b);
  out->ctas = (int)std::max<long long>(1, std::min<long long>(kClipCtas, (most + kClipShare - 1) / kClipShare));
  std::vector<int> begin(n_groups, 0), end(n_groups, 0);      // sums of every group
  size_t at = 0;
  int sums = 0;
  for (int w = 0; w < out->n_waves; ++w) {
    const long long share = std::max<long long>(kClipShare, ((wave_bytes[w] + out->ctas - 1) / out->ctas + 15) / 16 * 16);
    long long done = 0;                  // elements of tensor order[at] that are dealt
    for (int c = 0; c < out->ctas; ++c) {
      out->first.push_back((int)out->pieces.size());
      long long room = share;
      int kept = 0, group = -1;
      while (at < wave_end[w] && (room > 0 || c == out->ctas - 1)) {
        const pbt_clip_tensor& x = t[order[at]];
        const long long esz = x.dtype ? 2 : 4, left = x.numel - done;
        const char* src = (const char*)x.src + done * esz;
        const int phase = (int)((uintptr_t)src & 15);
        long long take = left;
        const long long space = (kClipKeep - kept - 16) / 16 * 16;   // for a piece that keeps its alignment
        bool keeps = space >= 1024;
        auto cut = [&](long long bytes) { take = std::min(take, std::max<long long>(1, (bytes - phase) / esz)); };
        if (c < out->ctas - 1 && left * esz > room) cut((room + 15) / 16 * 16 + 16);   // pieces end on 16-byte boundaries
        if (keeps) cut(space);
        cut(1ll << 30);
        if (x.group != group) {
          group = x.group;
          if (begin[group] == end[group]) begin[group] = sums;
          end[group] = ++sums;
        }
        out->pieces.push_back({src, (char*)x.dst + done * esz, (int)take, keeps ? kept + phase : -1, x.group * 2 + x.dtype, sums - 1, 0, 0, {0, 0}});
        if (keeps) kept += (int)((phase + take * esz + 15) / 16 * 16);
        room -= take * esz;
        done += take;
        if (done == x.numel) { ++at; done = 0; }
      }
      if (out->pieces.size() > (1u << 30)) return false;
    }
  }
  out->first.push_back((int)out->pieces.size());
  for (ClipPiece& p : out->pieces) {
    p.sum_begin = begin[p.group2 >> 1];
    p.sum_end = end[p.group2 >> 1];
  }
  for (int g = 0; g < n_groups; ++g) out->empty.push_back(group_bytes[g] == 0);
  out->n_sums = sums;
  return true;
}

struct ClipLayout {
  size_t barrier, sums, empty, first, pieces, large, factors, chunk_sums, chunks, total;
};
ClipLayout clip_layout(const ClipTable& t) {
  ClipLayout l;
  l.barrier = 0;
  l.sums = 256;
  l.empty = l.sums + clip_align((size_t)t.n_sums * sizeof(double));
  l.first = l.empty + clip_align(t.empty.size() * sizeof(int));
  l.pieces = l.first + clip_align(t.first.size() * sizeof(int));
  l.large = l.pieces + clip_align(t.pieces.size() * sizeof(ClipPiece));
  l.factors = l.large + clip_align(t.large.size() * sizeof(int));
  l.chunk_sums = l.factors + clip_align(t.large.empty() ? 0 : t.empty.size() * sizeof(float));
  l.chunks = l.chunk_sums + clip_align(t.chunks.size() * sizeof(double));
  l.total = l.chunks + clip_align(t.chunks.size() * sizeof(ClipPiece));
  return l;
}

// A destination may be its own source (in place) and nothing else that this call reads or writes.
bool clip_overlap(const pbt_clip_tensor* t, int n) {
  struct Range { uintptr_t lo, hi; int tensor, is_dst; };
  std::vector<Range> r;
  for (int i = 0; i < n; ++i) {
    if (!t[i].numel) continue;
    const uintptr_t bytes = (uintptr_t)t[i].numel * (t[i].dtype ? 2 : 4);
    r.push_back({(uintptr_t)t[i].dst, (uintptr_t)t[i].dst + bytes, i, 1});
    if (t[i].src != t[i].dst) r.push_back({(uintptr_t)t[i].src, (uintptr_t)t[i].src + bytes, i, 0});
  }
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
  uintptr_t dst_end = 0, any_end = 0;
  for (const Range& x : r) {
    if (x.lo < dst_end || (x.is_dst && x.lo < any_end)) return true;
    any_end = std::max(any_end, x.hi);
    if (x.is_dst) dst_end = std::max(dst_end, x.hi);
  }
  return false;
}

}  // namespace
}  // namespace pbt

struct pbt_clip {
  pbt::ClipArgs args;
  pbt::StreamArgs stream;
  int ctas;
  bool some_empty;      // groups without elements: their norms are k_clip's to write
};

extern "C" int pbt_clip_query_workspace(const pbt_clip_tensor* tensors, int32_t n_tensors, int32_t n_groups, size_t* bytes) {
  using namespace pbt;
  if (!bytes) return clip_fail(PBT_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = clip_check(tensors, n_tensors, n_groups);
  if (rc) return rc;
  try {
    ClipTable t;
    if (!clip_table(tensors, n_tensors, n_groups, &t)) return clip_fail(PBT_ERR_UNSUPPORTED, "too many gradient elements for one call");
    *bytes = clip_layout(t).total;
  } catch (const std::bad_alloc&) {
    return clip_fail(PBT_ERR_STATE, "out of host memory");
  }
  return PBT_OK;
}

extern "C" int pbt_clip_create(pbt_clip_t** out, const pbt_clip_tensor* tensors, int32_t n_tensors, int32_t n_groups,
                               void* workspace, size_t workspace_bytes, void* stream) {
  using namespace pbt;
  if (!out) return clip_fail(PBT_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  const int rc = clip_check(tensors, n_tensors, n_groups);
  if (rc) return rc;
  try {
    ClipTable t;
    if (!clip_table(tensors, n_tensors, n_groups, &t)) return clip_fail(PBT_ERR_UNSUPPORTED, "too many gradient elements for one call");
    const ClipLayout l = clip_layout(t);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < l.total)
      return clip_fail(PBT_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than pbt_clip_query_workspace says");
    if (clip_overlap(tensors, n_tensors))
      return clip_fail(PBT_ERR_INVALID_ARG, "a destination overlaps another tensor of the call (only dst == src is allowed)");
    char* base = (char*)workspace;
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e = cudaMemsetAsync(base + l.barrier, 0, 256, s);
    auto upload = [&](size_t at, const void* from, size_t bytes) {
      if (e == cudaSuccess && bytes) e = cudaMemcpyAsync(base + at, from, bytes, cudaMemcpyHostToDevice, s);
    };
    upload(l.empty, t.empty.data(), t.empty.size() * sizeof(int));
    upload(l.first, t.first.data(), t.first.size() * sizeof(int));
    upload(l.pieces, t.pieces.data(), t.pieces.size() * sizeof(ClipPiece));
    upload(l.large, t.large.data(), t.large.size() * sizeof(int));
    upload(l.chunks, t.chunks.data(), t.chunks.size() * sizeof(ClipPiece));
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);   // the tables above are this function's own
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_clip, cudaFuncAttributeMaxDynamicSharedMemorySize, kClipKeep);
    if (e != cudaSuccess) return clip_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
    pbt_clip* p = new pbt_clip;
    memset(&p->args, 0, sizeof(p->args));
    p->args.pieces = (const ClipPiece*)(base + l.pieces);
    p->args.first = (const int*)(base + l.first);
    p->args.empty = (const int*)(base + l.empty);
    p->args.sums = (double*)(base + l.sums);
    p->args.barrier = (unsigned int*)(base + l.barrier);
    p->args.n_waves = t.n_waves;
    p->args.n_groups = n_groups;
    p->ctas = t.ctas;
    p->some_empty = std::find(t.empty.begin(), t.empty.end(), 1) != t.empty.end();
    memset(&p->stream, 0, sizeof(p->stream));
    p->stream.chunks = (const ClipPiece*)(base + l.chunks);
    p->stream.groups = (const int*)(base + l.large);
    p->stream.n_chunks = (int)t.chunks.size();
    p->stream.n_groups = (int)t.large.size() / 3;
    p->stream.sums = (double*)(base + l.chunk_sums);
    p->stream.factors = (float*)(base + l.factors);
    *out = p;
  } catch (const std::bad_alloc&) {
    return clip_fail(PBT_ERR_STATE, "out of host memory");
  }
  return PBT_OK;
}

extern "C" int pbt_clip_destroy(pbt_clip_t* p) {
  delete p;
  return PBT_OK;
}

extern "C" int pbt_clip_run(pbt_clip_t* p, float limit, const float* limits_device, float* norms_out_device, void* stream) {
  using namespace pbt;
  if (!p || !norms_out_device) return clip_fail(PBT_ERR_INVALID_ARG, "handle or norms_out_device is NULL");
  if (!limits_device && !(limit >= 0.f)) return clip_fail(PBT_ERR_INVALID_ARG, "the norm limit must be >= 0");
  ClipArgs a = p->args;
  a.limit = limit;
  a.limits = limits_device;
  a.norms = norms_out_device;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = cudaSuccess;
  if (a.n_waves || p->some_empty) {
    void* args[] = {&a};
    // cooperative: every CTA is resident, which the grid barrier relies on
    e = cudaLaunchCooperativeKernel((const void*)k_clip, dim3(p->ctas), dim3(kClipThreads), args, kClipKeep, st);
  }
  if (p->stream.n_chunks) {
    StreamArgs q = p->stream;
    q.limit = limit;
    q.limits = limits_device;
    q.norms = norms_out_device;
    if (e == cudaSuccess) e = launch_with(q.n_chunks, kStreamThreads, 0, st)(k_clip_sums, q);
    if (e == cudaSuccess) e = launch_with(q.n_groups, kStreamThreads, 0, st)(k_clip_factors, q);
    if (e == cudaSuccess) e = launch_with(q.n_chunks, kStreamThreads, 0, st)(k_clip_scale, q);
  }
  if (e != cudaSuccess) return clip_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
  return PBT_OK;
}

extern "C" int pbt_clip_status(pbt_clip_t* p, void* stream) {
  using namespace pbt;
  if (!p) return clip_fail(PBT_ERR_INVALID_ARG, "handle is NULL");
  unsigned int status = 0;
  cudaError_t e = cudaMemcpyAsync(&status, p->args.barrier + 2, sizeof(status), cudaMemcpyDeviceToHost, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e != cudaSuccess) return clip_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
  if (status) return clip_fail((int)status, "the grid barrier of a clipping run timed out; its norms are NaN");
  return PBT_OK;
}
