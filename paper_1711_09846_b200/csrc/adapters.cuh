// Low-rank adapters of many requests (or members) beside one shared projection: declarations shared by the entry points
// (adapters.cu) and the kernels.
#pragma once
#include "pbt_common.cuh"

namespace pbt {
namespace adapters {

constexpr int kMaxRank = 64;

// Which rows belong to which adapter: segment j holds rows [offsets[j], offsets[j + 1]) and uses adapter ids[j].  The
// arrays are the caller's device memory; every read is clamped (offsets to [0, rows], ids outside [0, n_adapters) mean
// "no adapter"), so that no content of theirs makes a kernel leave its buffers.
struct Segments {
  const int* offsets;
  const int* ids;
  int n, rows, n_adapters;
};

// bf16, on the tensor cores (adapters_tc.cu)
size_t tc_workspace(const pbt_adapter_desc* d, bool backward);
cudaError_t tc_forward(const pbt_adapter_desc* d, const Segments& segs, char* workspace, cudaStream_t s);
cudaError_t tc_backward(const pbt_adapter_desc* d, const Segments& segs, char* workspace, cudaStream_t s);

// dA and dB as the sums of their splits, in order (parts: [splits][size] each)
cudaError_t join_gradients(const float* parts_a, const float* parts_b, long long size_a, long long size_b, int splits, float* dA, float* dB, cudaStream_t s);

#ifdef __CUDACC__
__device__ __forceinline__ int segment_begin(const Segments& s, int j) { return min(max(__ldg(s.offsets + j), 0), s.rows); }
__device__ __forceinline__ int segment_adapter(const Segments& s, int j) {
  const int a = __ldg(s.ids + j);
  return a >= 0 && a < s.n_adapters ? a : -1;
}
// The last segment that begins at or before `row` (offsets ascend; empty segments are passed over), -1 if none does.
__device__ __forceinline__ int segment_of_row(const Segments& s, int row) {
  int lo = 0, hi = s.n;   // offsets[lo - 1] <= row < offsets[hi], as far as those exist
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (segment_begin(s, mid) <= row) lo = mid + 1;
    else hi = mid;
  }
  return lo - 1;
}
// The same for a whole warp, in one trip to memory instead of one per halving (offsets ascend: those at or before the row count).
__device__ __forceinline__ int segment_of_row_warp(const Segments& s, int row) {
  if (s.n > 1024) return segment_of_row(s, row);
  int count = 0;
  for (int i = threadIdx.x & 31; i < s.n; i += 32) count += segment_begin(s, i) <= row;
  count = __reduce_add_sync(0xFFFFFFFFu, count);
  return count - 1;
}
#endif

}  // namespace adapters
}  // namespace pbt
