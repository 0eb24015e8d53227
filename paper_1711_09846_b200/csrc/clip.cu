// Global gradient norm over many tensors, and clipping, per group (population member):
//   norm_g = sqrt(sum over the tensors of group g, all elements: e^2),   dst = src * min(1, limit_g / norm_g).
//
// Two launches over one table of chunks, sorted by group: the first leaves one partial sum of squares per chunk, the
// second adds the partials of a chunk's group in a fixed order (no atomics: a run is reproducible bit for bit) and
// scales.  Memory-bound: the floor is one read and one write of every element.
#include <stdio.h>

#include <algorithm>
#include <new>
#include <vector>

#include "pbt_common.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace {

constexpr int kClipThreads = 256;
constexpr int kClipChunk = 16384;   // elements

struct ClipChunk {
  const char* src;
  char* dst;
  int count;
  int group_and_type;   // group * 2 + (1: bfloat16)
};

__device__ __forceinline__ float clip_load(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float clip_load(const float* p) { return *p; }
__device__ __forceinline__ void clip_store(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void clip_store(float* p, float v) { *p = v; }

template <typename S>
__device__ __forceinline__ S clip_block_sum(S v, S* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  S t = scratch[0];
  for (int w = 1; w < kClipThreads / 32; ++w) t += scratch[w];
  return t;
}

// Squares in fp32; where their sum leaves the range in which fp32 squares are exact to rounding (elements beyond
// 1.8e19 or all below 1e-15), the chunk is summed again in fp64, so that only the norm itself can overflow.
template <typename T>
__device__ double clip_sum_squares(const T* g, int n, double* scratch) {
  float s = 0.f;
  for (int i = threadIdx.x; i < n; i += kClipThreads) {
    const float v = clip_load(g + i);
    s = __fmaf_rn(v, v, s);
  }
  const float t = clip_block_sum(s, reinterpret_cast<float*>(scratch));
  if (t > 1e-30f && t < 3e38f) return t;
  double d = 0.0;
  for (int i = threadIdx.x; i < n; i += kClipThreads) {
    const double v = clip_load(g + i);
    d = fma(v, v, d);
  }
  return clip_block_sum(d, scratch);
}

__global__ void __launch_bounds__(kClipThreads) k_clip_norm(const ClipChunk* __restrict__ chunks, double* __restrict__ partial) {
  pdl_prologue();
  __shared__ double scratch[kClipThreads / 32];
  const ClipChunk c = chunks[blockIdx.x];
  const double s = (c.group_and_type & 1) ? clip_sum_squares(reinterpret_cast<const bf16*>(c.src), c.count, scratch)
                                          : clip_sum_squares(reinterpret_cast<const float*>(c.src), c.count, scratch);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// min(1, limit / norm); a NaN norm makes the factor NaN (a diverged member stays visible), an infinite limit never clips
__device__ __forceinline__ float clip_factor(float limit, float norm) {
  if (isinf(limit) && limit > 0.f) return 1.f;
  if (norm <= limit) return 1.f;
  return __fdiv_rn(limit, norm);
}

template <typename T>
__device__ void clip_scale(const ClipChunk& c, float f) {
  const T* g = reinterpret_cast<const T*>(c.src);
  T* o = reinterpret_cast<T*>(c.dst);
  for (int i = threadIdx.x; i < c.count; i += kClipThreads) clip_store(o + i, clip_load(g + i) * f);
}

__global__ void __launch_bounds__(kClipThreads) k_clip_scale(const ClipChunk* __restrict__ chunks, int n_chunks,
                                                             const double* __restrict__ partial,
                                                             const int* __restrict__ group_begin, float limit,
                                                             const float* __restrict__ limits, float* __restrict__ norms) {
  pdl_prologue();
  __shared__ double scratch[kClipThreads / 32];
  ClipChunk c;
  c.count = 0;
  int group = (int)blockIdx.x - n_chunks;   // the blocks behind the chunks write the norms
  if (group < 0) {
    c = chunks[blockIdx.x];
    group = c.group_and_type >> 1;
  }
  double s = 0.0;
  for (int i = group_begin[group] + threadIdx.x; i < group_begin[group + 1]; i += kClipThreads) s += partial[i];
  const float norm = (float)sqrt(clip_block_sum(s, scratch));
  if ((int)blockIdx.x >= n_chunks) {
    if (threadIdx.x == 0) norms[group] = norm;
    return;
  }
  const float f = clip_factor(limits ? limits[group] : limit, norm);
  if (f == 1.f && c.src == c.dst) return;
  if (c.group_and_type & 1) clip_scale<bf16>(c, f);
  else clip_scale<float>(c, f);
}

int clip_fail(int code, const char* msg) {
  set_last_error(msg);
  return code;
}

size_t clip_align(size_t n) { return (n + 255) & ~(size_t)255; }

struct ClipLayout {
  size_t partial, begin, chunks, total;
};
ClipLayout clip_layout(long long n_chunks, int n_groups) {
  ClipLayout l;
  l.partial = 0;
  l.begin = clip_align((size_t)n_chunks * sizeof(double));
  l.chunks = l.begin + clip_align((size_t)(n_groups + 1) * sizeof(int));
  l.total = l.chunks + clip_align((size_t)n_chunks * sizeof(ClipChunk));
  return l;
}

int clip_check(const pbt_clip_tensor* t, int n, int n_groups, long long* n_chunks) {
  if (n < 0 || n_groups < 1 || n_groups > (1 << 20)) return clip_fail(PBT_ERR_INVALID_ARG, "n_tensors must be >= 0 and n_groups in [1, 2^20]");
  if (n > 0 && !t) return clip_fail(PBT_ERR_INVALID_ARG, "tensors is NULL");
  long long total = 0;
  for (int i = 0; i < n; ++i) {
    if (t[i].numel < 0 || (t[i].numel > 0 && (!t[i].src || !t[i].dst)))
      return clip_fail(PBT_ERR_INVALID_ARG, "a gradient tensor has a negative size or a NULL pointer");
    if (t[i].dtype != 0 && t[i].dtype != 1) return clip_fail(PBT_ERR_UNSUPPORTED, "gradient tensors are float or bfloat16");
    if (t[i].group < 0 || t[i].group >= n_groups) return clip_fail(PBT_ERR_INVALID_ARG, "a tensor's group is out of range");
    const uintptr_t esz = t[i].dtype ? 2 : 4;
    if (((uintptr_t)t[i].src % esz) || ((uintptr_t)t[i].dst % esz))
      return clip_fail(PBT_ERR_INVALID_ARG, "a gradient tensor is not aligned to its element size");
    total += (t[i].numel + kClipChunk - 1) / kClipChunk;
  }
  if (total > (1ll << 30)) return clip_fail(PBT_ERR_UNSUPPORTED, "too many gradient elements for one call");
  *n_chunks = total;
  return PBT_OK;
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
  const pbt::ClipChunk* chunks;
  double* partial;
  const int* group_begin;
  int n_chunks, n_groups;
};

extern "C" int pbt_clip_query_workspace(const pbt_clip_tensor* tensors, int32_t n_tensors, int32_t n_groups, size_t* bytes) {
  if (!bytes) return pbt::clip_fail(PBT_ERR_INVALID_ARG, "bytes is NULL");
  long long n_chunks = 0;
  const int rc = pbt::clip_check(tensors, n_tensors, n_groups, &n_chunks);
  if (rc) return rc;
  *bytes = pbt::clip_layout(n_chunks, n_groups).total;
  return PBT_OK;
}

extern "C" int pbt_clip_create(pbt_clip_t** out, const pbt_clip_tensor* tensors, int32_t n_tensors, int32_t n_groups,
                               void* workspace, size_t workspace_bytes, void* stream) {
  using namespace pbt;
  if (!out) return clip_fail(PBT_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  long long n_chunks = 0;
  const int rc = clip_check(tensors, n_tensors, n_groups, &n_chunks);
  if (rc) return rc;
  const ClipLayout l = clip_layout(n_chunks, n_groups);
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < l.total)
    return clip_fail(PBT_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than pbt_clip_query_workspace says");
  try {
    if (clip_overlap(tensors, n_tensors))
      return clip_fail(PBT_ERR_INVALID_ARG, "a destination overlaps another tensor of the call (only dst == src is allowed)");
    std::vector<int> order(n_tensors), begin(n_groups + 1, 0);
    for (int i = 0; i < n_tensors; ++i) order[i] = i;
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return tensors[a].group < tensors[b].group; });
    std::vector<ClipChunk> table;
    table.reserve((size_t)n_chunks);
    for (int i : order) {
      const pbt_clip_tensor& t = tensors[i];
      const long long esz = t.dtype ? 2 : 4;
      for (long long at = 0; at < t.numel; at += kClipChunk) {
        const long long left = t.numel - at;
        table.push_back({(const char*)t.src + at * esz, (char*)t.dst + at * esz, (int)(left < kClipChunk ? left : kClipChunk),
                         t.group * 2 + t.dtype});
      }
      begin[t.group + 1] = (int)table.size();
    }
    for (int g = 0; g < n_groups; ++g) begin[g + 1] = std::max(begin[g], begin[g + 1]);   // groups without elements
    char* base = (char*)workspace;
    cudaError_t e = cudaMemcpyAsync(base + l.begin, begin.data(), begin.size() * sizeof(int), cudaMemcpyHostToDevice, (cudaStream_t)stream);
    if (e == cudaSuccess && n_chunks)
      e = cudaMemcpyAsync(base + l.chunks, table.data(), table.size() * sizeof(ClipChunk), cudaMemcpyHostToDevice, (cudaStream_t)stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);   // the tables above are this function's own
    if (e != cudaSuccess) return clip_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
    pbt_clip* p = new pbt_clip;
    p->chunks = (const ClipChunk*)(base + l.chunks);
    p->partial = (double*)(base + l.partial);
    p->group_begin = (const int*)(base + l.begin);
    p->n_chunks = (int)n_chunks;
    p->n_groups = n_groups;
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
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e = cudaSuccess;
  if (p->n_chunks) e = launch_with(p->n_chunks, kClipThreads, 0, s)(k_clip_norm, p->chunks, p->partial);
  if (e == cudaSuccess)
    e = launch_with(p->n_chunks + p->n_groups, kClipThreads, 0, s)(k_clip_scale, p->chunks, p->n_chunks, p->partial, p->group_begin,
                                                              limit, limits_device, norms_out_device);
  if (e != cudaSuccess) return clip_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
  return PBT_OK;
}
