// Global gradient norm over many tensors, and clipping, per group (population member):
//   norm_g = sqrt(sum over the tensors of group g, all elements: e^2),   dst = src * min(1, limit_g / norm_g).
//
// Memory-bound.  One table of 32 KB chunks, sorted by group, a block to a chunk.  The first pass leaves the chunks' sums of squares; the
// block that brings a group's last sum adds the group's sums in their order and leaves norm and factor (so the order of
// arrival decides who adds, not what: a run is reproducible bit for bit).  The second pass scales.  The passes alternate over
// waves of whole groups, so that the second finds its gradients in L2; a launch scales one wave and sums the next, its
// blocks start while the launch before drains, load their chunk, and wait for the factors before they store.
//
// Floor: one read and one write of every element.  16 x 394,753 fp32 elements (7.7 us at the copy rate) take 15.7 us, two launches
// and the latencies of a load, a sum and a store each; 80 x 14.7 M (1.44 ms) 1.96 ms: 125 MB of DRAM traffic for each member's
// 118 MB, at 4.9 TB/s, since blocks start, load, wait and end instead of streaming.  Tried instead: gradients kept in the SMs' shared memory over a grid barrier, 21.2 us and
// 2.57 ms (the CTAs' meeting and the factor cost 9 us a wave); persistent CTAs with cp.async rings, 22 to 31 us and 2.42 to 2.96 ms.
#include <stdio.h>

#include <algorithm>
#include <new>
#include <vector>

#include "pbt_common.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace {

constexpr int kClipThreads = 256;
constexpr int kClipChunk = 32 * 1024;      // bytes (one wave of 80 x 14.7 M: 16 KB 2.10 ms, 32 KB 2.04, 64 KB 2.12)
// Bytes of the groups of a wave, at most (a larger group is a wave by itself).  200 x 2 M fp32 elements: 16 MB 711 us, 32 MB 640, 48 MB
// 647, 96 MB 665, all at once 707; 100 x 6 M: 1041, 1041, 989, 999, 1051.
constexpr long long kClipWave = 48 << 20;
constexpr int kClipVectors = kClipChunk / 16 / kClipThreads;      // 16-byte vectors of a thread

struct __align__(16) ClipPiece {
  const char* src;
  char* dst;
  int count;       // elements
  int group2;      // 2 * group + (1: bfloat16)
  int pad[2];
  __device__ bool bf() const { return group2 & 1; }
};

// A tensor of the call.  Its chunks end on 16-byte boundaries of the source, but for the last one.
struct ClipTensor {
  const char* src;
  char* dst;
  long long numel;
  int group2;
  int first;       // its first chunk
  __host__ __device__ long long per() const { return kClipChunk / (group2 & 1 ? 2 : 4); }
  __host__ __device__ long long head() const { return (kClipChunk - (long long)((uintptr_t)src & 15)) / (group2 & 1 ? 2 : 4); }
  __host__ __device__ long long chunks() const { return 1 + (numel > head() ? (numel - head() + per() - 1) / per() : 0); }
  __host__ __device__ ClipPiece chunk(int k) const {
    const long long from = k ? head() + (k - 1) * per() : 0, to = head() + k * per(), end = to < numel ? to : numel, esz = group2 & 1 ? 2 : 4;
    return {src + from * esz, dst + from * esz, (int)(end - from), group2, {0, 0}};
  }
};

// The table of chunks, when a handle is made: 140 thousand chunks of 80 tensors would take the host milliseconds.
__global__ void k_clip_table(const ClipTensor* tensors, int n_tensors, ClipPiece* chunks, int n_chunks) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= n_chunks) return;
  int lo = 0, hi = n_tensors;      // the last tensor whose first chunk is not behind c
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (tensors[mid].first <= c) lo = mid;
    else hi = mid;
  }
  chunks[c] = tensors[lo].chunk(c - tensors[lo].first);
}

struct ClipArgs {
  const ClipPiece* chunks;
  const int* begin;              // [groups + 1] first chunk of every group
  const int* empty;              // groups without elements
  int n_empty;
  double* sums;                  // of every chunk
  unsigned int* done;            // of every group: chunks summed (zero between runs)
  float* factors;                // of every group
  float limit;
  const float* limits;
  float* norms;
};

__device__ __forceinline__ float clip_load(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float clip_load(const float* p) { return *p; }
__device__ __forceinline__ void clip_store(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void clip_store(float* p, float v) { *p = v; }

// Sum over the block, the same for every thread.
template <typename S>
__device__ __forceinline__ S clip_block_sum(S v, S* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  S t = scratch[0];
#pragma unroll
  for (int w = 1; w < kClipThreads / 32; ++w) t += scratch[w];
  return t;
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

// A chunk is its elements up to the first 16-byte boundary, 16-byte vectors (at most kClipVectors a thread), and the rest; a
// thread has at most one of the loose elements.
template <typename T>
struct ClipSpan {
  const T* src;
  const uint4* from;
  int head, vectors, loose;
  __device__ __forceinline__ explicit ClipSpan(const ClipPiece& p) {
    src = reinterpret_cast<const T*>(p.src);
    head = min(p.count, (int)((16 - ((uintptr_t)p.src & 15)) & 15) / (int)sizeof(T));
    vectors = (p.count - head) / Quad<T>::n;
    loose = p.count - vectors * Quad<T>::n;
    from = reinterpret_cast<const uint4*>(src + head);
  }
  __device__ __forceinline__ int at(int i) const { return i < head ? i : i + vectors * Quad<T>::n; }   // place of loose element i
  // LAST: the last use of the gradients, after which L2 may drop them
  template <bool LAST>
  __device__ __forceinline__ void load(uint4* v) const {
#pragma unroll
    for (int u = 0; u < kClipVectors; ++u) {
      const int i = u * kClipThreads + threadIdx.x;
      if (i < vectors) v[u] = LAST ? __ldcs(from + i) : __ldg(from + i);
    }
  }
};

template <typename T>
__device__ __forceinline__ float clip_sum(const ClipPiece& p) {
  const ClipSpan<T> s(p);
  uint4 v[kClipVectors];
  s.load<false>(v);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  if ((int)threadIdx.x < s.loose) {
    const float f = clip_load(s.src + s.at(threadIdx.x));
    sum[0] = f * f;
  }
#pragma unroll
  for (int u = 0; u < kClipVectors; ++u)
    if (u * kClipThreads + (int)threadIdx.x < s.vectors) {
      float f[Quad<T>::n];
      Quad<T>::get(v[u], f);
#pragma unroll
      for (int e = 0; e < Quad<T>::n; ++e) sum[e & 3] = __fmaf_rn(f[e], f[e], sum[e & 3]);
    }
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}
template <typename T>
__device__ __noinline__ double clip_sum_wide(const ClipPiece& p) {
  const T* g = reinterpret_cast<const T*>(p.src);
  double sum = 0.0;
  for (int i = threadIdx.x; i < p.count; i += kClipThreads) {
    const double v = clip_load(g + i);
    sum = ::fma(v, v, sum);
  }
  return sum;
}

// min(1, limit / norm); a NaN norm makes the factor NaN (a diverged member stays visible), an infinite limit never clips
__device__ __forceinline__ float clip_factor(float limit, float norm) {
  if (isinf(limit) && limit > 0.f) return 1.f;
  if (norm <= limit) return 1.f;
  return __fdiv_rn(limit, norm);
}

__device__ __forceinline__ void clip_norm(const ClipArgs& a, int chunk) {
  __shared__ float scratch[kClipThreads / 32];
  __shared__ double scratch_wide[kClipThreads / 32];
  __shared__ bool last;
  const ClipPiece p = a.chunks[chunk];
  const int group = p.group2 >> 1;
  const float t = clip_block_sum(p.bf() ? clip_sum<bf16>(p) : clip_sum<float>(p), scratch);
  double sum = t;
  // Squares are fp32; where their sum leaves the range in which that is exact to rounding (elements beyond 1.8e19, or all
  // below 1e-15), the chunk is summed again in fp64, so that only the norm itself can overflow.
  if (!(t > 1e-30f && t < 3e38f)) sum = clip_block_sum(p.bf() ? clip_sum_wide<bf16>(p) : clip_sum_wide<float>(p), scratch_wide);
  const int begin = a.begin[group], end = a.begin[group + 1];
  if (threadIdx.x == 0) {
    a.sums[chunk] = sum;
    __threadfence();
    last = atomicAdd(a.done + group, 1u) == (unsigned int)(end - begin) - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double s = 0.0;
#pragma unroll 4
  for (int q = begin + threadIdx.x; q < end; q += kClipThreads) s += __ldcg(a.sums + q);
  const float norm = (float)sqrt(clip_block_sum(s, scratch_wide));
  if (threadIdx.x == 0) {
    const float limit = a.limits ? a.limits[group] : a.limit;      // (before the norm, which may take its place)
    a.norms[group] = norm;
    a.factors[group] = clip_factor(limit, norm);
    a.done[group] = 0;
  }
}

template <typename T>
__device__ __forceinline__ void clip_scale(const ClipArgs& a, const ClipPiece& p) {
  const ClipSpan<T> s(p);
  uint4 v[kClipVectors];
  s.load<true>(v);
  const int mine = (int)threadIdx.x < s.loose ? s.at(threadIdx.x) : -1;
  const float one = mine >= 0 ? clip_load(s.src + mine) : 0.f;
  asm volatile("griddepcontrol.wait;" ::: "memory");      // the factors are there, and every gradient has been summed
  const float f = __ldcg(a.factors + (p.group2 >> 1));
  if (f == 1.f && p.src == p.dst) return;
  T* o = reinterpret_cast<T*>(p.dst);
  if (mine >= 0) clip_store(o + mine, one * f);
  o += s.head;
  const bool whole = ((uintptr_t)o & 15) == 0;      // the destination has the source's alignment
#pragma unroll
  for (int u = 0; u < kClipVectors; ++u) {
    const int i = u * kClipThreads + threadIdx.x;
    if (i >= s.vectors) continue;
    float e[Quad<T>::n];
    Quad<T>::get(v[u], e);
#pragma unroll
    for (int j = 0; j < Quad<T>::n; ++j) e[j] *= f;
    if (whole) {
      __stcs(reinterpret_cast<uint4*>(o) + i, Quad<T>::put(e));
    } else {
#pragma unroll
      for (int j = 0; j < Quad<T>::n; ++j) clip_store(o + i * Quad<T>::n + j, e[j]);
    }
  }
}

// One step: scales the chunks of a wave, [scale, scale + scale_n), and sums those of the next one, [sum, sum + sum_n), by turns, so
// that DRAM reads and writes all the time.  Scaling begins with the last chunk, which is the most likely to be in L2 still.  The
// first step also leaves the norms of groups without elements.
// Five blocks to an SM: 1.96 ms for 80 x 14.7 M; four 2.02, six (which spill) 2.08.
__global__ void __launch_bounds__(kClipThreads, 5) k_clip(const ClipArgs a, int scale, int scale_n, int sum, int sum_n) {
  if (!scale_n) pdl_prologue();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int b = blockIdx.x, both = 2 * min(scale_n, sum_n), k = b < both ? b >> 1 : b - both / 2;
  if (b >= scale_n + sum_n) {
    const int i = (b - scale_n - sum_n) * kClipThreads + threadIdx.x;
    if (i < a.n_empty) a.norms[a.empty[i]] = 0.f;
  } else if (b < both ? b & 1 : scale_n > sum_n) {
    const ClipPiece p = a.chunks[scale + scale_n - 1 - k];
    if (p.bf()) clip_scale<bf16>(a, p);
    else clip_scale<float>(a, p);
  } else {
    clip_norm(a, sum + k);
  }
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

struct ClipTable {
  std::vector<ClipTensor> tensors;     // that have elements, by group
  std::vector<int> begin, empty;
  std::vector<int> waves;              // first chunk of every wave, and the number of chunks
  int chunks;
};
bool clip_table(const pbt_clip_tensor* t, int n_tensors, int n_groups, ClipTable* out) {
  std::vector<int> order;
  std::vector<long long> size(n_groups, 0);
  for (int i = 0; i < n_tensors; ++i)
    if (t[i].numel) {
      order.push_back(i);
      size[t[i].group] += t[i].numel * (t[i].dtype ? 2 : 4);
    }
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return t[a].group < t[b].group; });
  out->begin.assign(n_groups + 1, 0);
  long long chunks = 0;
  for (int i : order) {
    const ClipTensor x = {(const char*)t[i].src, (char*)t[i].dst, t[i].numel, t[i].group * 2 + t[i].dtype, (int)chunks};
    out->tensors.push_back(x);
    chunks += x.chunks();
    if (chunks > (1 << 30)) return false;
    out->begin[t[i].group + 1] = (int)chunks;
  }
  out->chunks = (int)chunks;
  long long wave = 0;
  out->waves.assign(1, 0);
  for (int g = 0; g < n_groups; ++g) {
    out->begin[g + 1] = std::max(out->begin[g], out->begin[g + 1]);
    if (out->begin[g] == out->begin[g + 1]) out->empty.push_back(g);
    if (size[g] && wave && wave + size[g] > kClipWave) {
      out->waves.push_back(out->begin[g]);
      wave = 0;
    }
    wave += size[g];
  }
  out->waves.push_back(out->chunks);
  return true;
}

struct ClipLayout {
  size_t done, sums, factors, begin, empty, tensors, chunks, total;
};
ClipLayout clip_layout(const ClipTable& t) {
  const size_t groups = t.begin.size() - 1;
  ClipLayout l;
  l.done = 0;
  l.sums = clip_align(groups * sizeof(unsigned int));
  l.factors = l.sums + clip_align((size_t)t.chunks * sizeof(double));
  l.begin = l.factors + clip_align(groups * sizeof(float));
  l.empty = l.begin + clip_align(t.begin.size() * sizeof(int));
  l.tensors = l.empty + clip_align(t.empty.size() * sizeof(int));
  l.chunks = l.tensors + clip_align(t.tensors.size() * sizeof(ClipTensor));
  l.total = l.chunks + clip_align((size_t)t.chunks * sizeof(ClipPiece));
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
  std::vector<int> waves;
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
    cudaError_t e = cudaMemsetAsync(base + l.done, 0, (size_t)n_groups * sizeof(unsigned int), s);
    auto upload = [&](size_t at, const void* from, size_t bytes) {
      if (e == cudaSuccess && bytes) e = cudaMemcpyAsync(base + at, from, bytes, cudaMemcpyHostToDevice, s);
    };
    upload(l.begin, t.begin.data(), t.begin.size() * sizeof(int));
    upload(l.empty, t.empty.data(), t.empty.size() * sizeof(int));
    upload(l.tensors, t.tensors.data(), t.tensors.size() * sizeof(ClipTensor));
    if (e == cudaSuccess && t.chunks) {
      k_clip_table<<<(t.chunks + 255) / 256, 256, 0, s>>>((const ClipTensor*)(base + l.tensors), (int)t.tensors.size(), (ClipPiece*)(base + l.chunks), t.chunks);
      e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);   // the host's tables are this function's own, and runs may be on any stream
    if (e != cudaSuccess) return clip_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
    pbt_clip* p = new pbt_clip();
    p->args.chunks = (const ClipPiece*)(base + l.chunks);
    p->args.begin = (const int*)(base + l.begin);
    p->args.empty = (const int*)(base + l.empty);
    p->waves = t.waves;
    p->args.n_empty = (int)t.empty.size();
    p->args.sums = (double*)(base + l.sums);
    p->args.done = (unsigned int*)(base + l.done);
    p->args.factors = (float*)(base + l.factors);
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
  cudaStream_t s = (cudaStream_t)stream;
  const std::vector<int>& w = p->waves;
  const int empty = (a.n_empty + kClipThreads - 1) / kClipThreads;
  cudaError_t e = cudaSuccess;
  if (w[1] || empty) e = launch_with(w[1] + empty, kClipThreads, 0, s)(k_clip, a, 0, 0, 0, w[1]);
  for (size_t i = 1; i < w.size() && e == cudaSuccess && w[1]; ++i) {
    const int scale_n = w[i] - w[i - 1], sum_n = i + 1 < w.size() ? w[i + 1] - w[i] : 0;
    e = launch_after(scale_n + sum_n, kClipThreads, 0, s, k_clip, a, w[i - 1], scale_n, w[i], sum_n);
  }
  if (e != cudaSuccess) return clip_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
  return PBT_OK;
}
