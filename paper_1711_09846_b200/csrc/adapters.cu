// Low-rank adapters of many requests (or members) at once beside one shared, frozen projection:
//   S = x A_a^T,  y = x W^T + bias + c_a S B_a^T        (a: the adapter of the row's segment)
//   dS = c_a dy B_a,  dx = dy W + dS A_a,  dA_a = sum dS^T x,  dB_a = c_a sum dy^T S
// The entry points and the fp32 kernels.
//
// fp32: the shared product is the library's fp32-ALU GEMM; the low-rank parts are small beside it (r / K of its work)
// and each runs as one pass over the rows.
#include <algorithm>
#include <type_traits>

#include "adapters.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace adapters {
namespace {

// s[row][j] = f sum_k x[row][k] m_a(j, k), one warp per row; m_a is A_a [rank][K] or, TRANS, B_a [K][rank].
// f: the adapter's scale or 1.
template <bool TRANS>
__global__ void __launch_bounds__(256) k_adapter_shrink_f32(const float* __restrict__ x, long long ldx, int K, const float* __restrict__ mats,
                                                            int rank, const float* __restrict__ scale, Segments segs,
                                                            float* __restrict__ s) {
  pdl_prologue();
  const int row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (row >= segs.rows) return;
  const int j = segment_of_row(segs, row);
  if (j < 0 || row >= segment_begin(segs, j + 1)) return;
  const int a = segment_adapter(segs, j);
  if (a < 0) return;
  const float* xr = x + row * ldx;
  const float* m = mats + (long long)a * rank * K;
  const float f = scale ? scale[a] : 1.f;
  for (int r0 = 0; r0 < rank; r0 += 8) {
    float acc[8] = {};
#pragma unroll 4
    for (int k = lane; k < K; k += 32) {
      const float v = xr[k];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + i < rank) acc[i] = __fmaf_rn(v, TRANS ? m[(long long)k * rank + r0 + i] : m[(long long)(r0 + i) * K + k], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], o);
      if (lane == 0 && r0 + i < rank) s[(long long)row * rank + r0 + i] = f * acc[i];
    }
  }
}

constexpr int kExpandRows = 32;

// out[row][n] += f sum_j s[row][j] m_a(n, j); m_a is B_a [N][rank] or, TRANS, A_a [rank][N].  A block has 32 rows and 256
// columns; a thread keeps its column of the adapter's matrix in registers from row to row.
template <bool TRANS, int RANK>
__global__ void __launch_bounds__(256) k_adapter_expand_f32(float* out, long long ld_out, int N, const float* __restrict__ mats, int rank,
                                                            const float* __restrict__ scale, Segments segs, const float* __restrict__ s) {
  pdl_prologue();
  __shared__ float sr[kExpandRows][RANK];
  __shared__ int owner[kExpandRows];
  const int row0 = blockIdx.x * kExpandRows, rows = min(kExpandRows, segs.rows - row0), n = blockIdx.y * 256 + threadIdx.x;
  if (threadIdx.x < rows) {
    const int row = row0 + threadIdx.x, j = segment_of_row(segs, row);
    owner[threadIdx.x] = j >= 0 && row < segment_begin(segs, j + 1) ? segment_adapter(segs, j) : -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * rank; i += 256) {
    const int r = i / rank;
    sr[r][i % rank] = owner[r] >= 0 ? s[(long long)row0 * rank + i] * (scale ? scale[owner[r]] : 1.f) : 0.f;
  }
  __syncthreads();
  if (n >= N) return;
  float m[RANK];
  int have = -1;
  for (int r0 = 0; r0 < rows; r0 += 4) {
    float v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (r0 + u < rows && owner[r0 + u] >= 0) v[u] = out[(row0 + r0 + u) * ld_out + n];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = r0 + u;
      if (r >= rows || owner[r] < 0) continue;
      if (owner[r] != have) {
        have = owner[r];
        const float* p = mats + (long long)have * rank * N;
#pragma unroll
        for (int i = 0; i < RANK; ++i)
          if (i < rank) m[i] = TRANS ? p[(long long)i * N + n] : p[(long long)n * rank + i];
      }
      float acc = 0.f;
#pragma unroll
      for (int i = 0; i < RANK; ++i)
        if (i < rank) acc = __fmaf_rn(sr[r][i], m[i], acc);
      out[(row0 + r) * ld_out + n] = v[u] + acc;
    }
  }
}

struct GradSide {
  const float* v; long long ldv;
  const float* s;
  const float* scale;        // or null
  float* g;
  int N, blocks;
  bool columns_first;        // g is [N][rank], else [rank][N]
};

// g_a(j, n) = f_a sum over the rows of adapter a of s[row][j] v[row][n]: dA from (dS, x) and dB from (S, dy) in one launch.  A
// block owns 64 columns of one adapter and side; its 256 threads take every fourth row, four rows at a time, and add up in
// shared memory.
template <int RANK>
__global__ void __launch_bounds__(256) k_adapter_grad_f32(const GradSide x, const GradSide dy, int rank, Segments segs) {
  pdl_prologue();
  __shared__ float sum[3][RANK][64];
  const bool second = (int)blockIdx.x >= x.blocks;
  const GradSide& side = second ? dy : x;
  const int col = threadIdx.x & 63, part = threadIdx.x >> 6, n = ((int)blockIdx.x - (second ? x.blocks : 0)) * 64 + col, a = blockIdx.y;
  const float* v = side.v + min(n, side.N - 1);
  float acc[RANK] = {};
  for (int j = 0; j < segs.n; ++j) {
    if (segment_adapter(segs, j) != a) continue;
    const int end = segment_begin(segs, j + 1);
    for (int row = segment_begin(segs, j) + part; row < end; row += 16) {
      float y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = row + 4 * u < end ? v[(row + 4 * u) * side.ldv] : 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (row + 4 * u >= end) continue;
        const float* sr = side.s + (long long)(row + 4 * u) * rank;
#pragma unroll
        for (int i = 0; i < RANK; ++i) if (i < rank) acc[i] = __fmaf_rn(__ldg(sr + i), y[u], acc[i]);
      }
    }
  }
  if (part > 0)
#pragma unroll
    for (int i = 0; i < RANK; ++i) sum[part - 1][i][col] = acc[i];
  __syncthreads();
  if (part > 0 || n >= side.N) return;
  const float f = side.scale ? side.scale[a] : 1.f;
  float* out = side.g + (long long)a * rank * side.N;
#pragma unroll
  for (int i = 0; i < RANK; ++i)
    if (i < rank) out[side.columns_first ? (long long)n * rank + i : (long long)i * side.N + n] = f * (acc[i] + sum[0][i][col] + sum[1][i][col] + sum[2][i][col]);
}

// f(integral_constant) with the smallest of 4, 8, 16, 32, 64 that holds the rank
template <typename F>
cudaError_t with_rank(int rank, F f) {
  if (rank <= 4) return f(std::integral_constant<int, 4>());
  if (rank <= 8) return f(std::integral_constant<int, 8>());
  if (rank <= 16) return f(std::integral_constant<int, 16>());
  if (rank <= 32) return f(std::integral_constant<int, 32>());
  return f(std::integral_constant<int, 64>());
}

int fail(int code, const char* msg) {
  set_last_error(msg);
  return code;
}

int check(const pbt_adapter_desc* d) {
  if (!d) return fail(PBT_ERR_INVALID_ARG, "desc is NULL");
  if (d->rows < 0 || d->inputs < 1 || d->outputs < 1 || d->n_adapters < 1 || d->n_segments < 0)
    return fail(PBT_ERR_INVALID_ARG, "inputs, outputs and n_adapters must be positive, rows and n_segments >= 0");
  if (d->rank < 1 || d->rank > kMaxRank) return fail(PBT_ERR_UNSUPPORTED, "rank must be in [1, 64]");
  if (d->n_adapters > 65535) return fail(PBT_ERR_UNSUPPORTED, "more than 65535 adapters");
  if (d->dtype != 0 && d->dtype != 1) return fail(PBT_ERR_UNSUPPORTED, "operands are float or bfloat16");
  if (!d->weight || !d->A || !d->B || !d->scale || !d->row_offsets || (d->n_segments && !d->adapter_ids))
    return fail(PBT_ERR_INVALID_ARG, "weight, A, B, scale, row_offsets or adapter_ids is NULL");
  if (d->dtype == 1 && !d->status_device) return fail(PBT_ERR_INVALID_ARG, "status_device is required by the tensor-core kernels");
  if (d->ld_weight < d->inputs) return fail(PBT_ERR_INVALID_ARG, "ld_weight is smaller than inputs");
  return PBT_OK;
}

cudaError_t forward_f32(const pbt_adapter_desc* d, const Segments& segs, float* ws, cudaStream_t st) {
  float *s = d->s ? d->s : ws, *y = (float*)d->y;
  cudaError_t e = launch_with((d->rows + 7) / 8, 256, 0, st)(k_adapter_shrink_f32<false>, (const float*)d->x, d->ld_x, d->inputs, (const float*)d->A,
                                                         d->rank, nullptr, segs, s);
  if (e != cudaSuccess) return e;
  GemmArgs g;
  memset(&g, 0, sizeof(g));
  g.M = d->rows; g.N = d->outputs; g.K = d->inputs; g.batch = 1;
  g.in_dtype = g.out_dtype = kF32;
  g.A = d->x; g.lda = d->ld_x;
  g.B = d->weight; g.ldb = d->ld_weight;
  g.C = y; g.ldc = d->ld_y;
  g.bias = d->bias;
  e = launch_gemm_simt(g, st);
  if (e != cudaSuccess) return e;
  return with_rank(d->rank, [&](auto r) {
    return launch_with(dim3((d->rows + kExpandRows - 1) / kExpandRows, (d->outputs + 255) / 256), 256, 0, st)(
        k_adapter_expand_f32<false, decltype(r)::value>, y, d->ld_y, d->outputs, (const float*)d->B, d->rank, d->scale, segs, s);
  });
}

cudaError_t backward_f32(const pbt_adapter_desc* d, const Segments& segs, float* ds, cudaStream_t st) {
  const float *x = (const float*)d->x, *dy = (const float*)d->dy;
  float* dx = (float*)d->dx;
  cudaError_t e = launch_with((d->rows + 7) / 8, 256, 0, st)(k_adapter_shrink_f32<true>, dy, d->ld_dy, d->outputs, (const float*)d->B, d->rank, d->scale, segs, ds);
  if (e != cudaSuccess) return e;
  GemmArgs g;
  memset(&g, 0, sizeof(g));
  g.M = d->rows; g.N = d->inputs; g.K = d->outputs; g.batch = 1;
  g.in_dtype = g.out_dtype = kF32;
  g.A = dy; g.lda = d->ld_dy;
  g.B = d->weight; g.ldb = d->ld_weight; g.b_mn = 1;
  g.C = dx; g.ldc = d->ld_dx;
  e = launch_gemm_simt(g, st);
  if (e != cudaSuccess) return e;
  e = with_rank(d->rank, [&](auto r) {
    return launch_with(dim3((d->rows + kExpandRows - 1) / kExpandRows, (d->inputs + 255) / 256), 256, 0, st)(
        k_adapter_expand_f32<true, decltype(r)::value>, dx, d->ld_dx, d->inputs, (const float*)d->A, d->rank, nullptr, segs, ds);
  });
  if (e != cudaSuccess) return e;
  const GradSide a = {x, d->ld_x, ds, nullptr, d->dA, d->inputs, (d->inputs + 63) / 64, false};
  const GradSide b = {dy, d->ld_dy, d->s, d->scale, d->dB, d->outputs, (d->outputs + 63) / 64, true};
  return with_rank(d->rank, [&](auto r) {
    return launch_with(dim3(a.blocks + b.blocks, d->n_adapters), 256, 0, st)(k_adapter_grad_f32<decltype(r)::value>, a, b, d->rank, segs);
  });
}

// fp32: S of a forward pass that does not keep it, dS of a backward pass
size_t workspace_bytes(const pbt_adapter_desc* d, bool backward) {
  if (d->dtype) return tc_workspace(d, backward);
  return std::max<size_t>(256, ((size_t)d->rows * d->rank * sizeof(float) + 255) & ~(size_t)255);
}

int check_workspace(const pbt_adapter_desc* d, bool backward, const void* workspace, size_t bytes) {
  if (workspace && ((uintptr_t)workspace & 255) == 0 && bytes >= workspace_bytes(d, backward)) return PBT_OK;
  return fail(PBT_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than pbt_adapter_query_workspace says");
}

}  // namespace
}  // namespace adapters
}  // namespace pbt

extern "C" int pbt_adapter_query_workspace(const pbt_adapter_desc* d, int backward, size_t* bytes) {
  using namespace pbt::adapters;
  if (!bytes) return fail(PBT_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = check(d);
  if (rc) return rc;
  *bytes = workspace_bytes(d, backward != 0);
  return PBT_OK;
}

extern "C" int pbt_adapter_forward(const pbt_adapter_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace pbt;
  using namespace pbt::adapters;
  const int rc = check(d);
  if (rc) return rc;
  if (!d->rows) return PBT_OK;
  if (!d->x || !d->y || d->ld_x < d->inputs || d->ld_y < d->outputs)
    return fail(PBT_ERR_INVALID_ARG, "x or y is NULL, or its row stride is smaller than a row");
  const int ws = check_workspace(d, false, workspace, workspace_bytes);
  if (ws) return ws;
  const Segments segs = {d->row_offsets, d->adapter_ids, d->n_segments, d->rows, d->n_adapters};
  const cudaError_t e = d->dtype ? tc_forward(d, segs, (char*)workspace, (cudaStream_t)stream) : forward_f32(d, segs, (float*)workspace, (cudaStream_t)stream);
  return e == cudaSuccess ? PBT_OK : fail(PBT_ERR_CUDA, cudaGetErrorString(e));
}

extern "C" int pbt_adapter_backward(const pbt_adapter_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace pbt;
  using namespace pbt::adapters;
  const int rc = check(d);
  if (rc) return rc;
  if (!d->dA || !d->dB) return fail(PBT_ERR_INVALID_ARG, "dA or dB is NULL");
  if (d->rows && (!d->x || !d->dy || !d->dx || !d->s || d->ld_x < d->inputs || d->ld_dy < d->outputs || d->ld_dx < d->inputs))
    return fail(PBT_ERR_INVALID_ARG, "x, s, dy or dx is NULL, or a row stride is smaller than a row");
  const int ws = check_workspace(d, true, workspace, workspace_bytes);
  if (ws) return ws;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (!d->rows) {
    e = cudaMemsetAsync(d->dA, 0, (size_t)d->n_adapters * d->rank * d->inputs * sizeof(float), st);
    if (e == cudaSuccess) e = cudaMemsetAsync(d->dB, 0, (size_t)d->n_adapters * d->rank * d->outputs * sizeof(float), st);
  } else {
    const Segments segs = {d->row_offsets, d->adapter_ids, d->n_segments, d->rows, d->n_adapters};
    e = d->dtype ? tc_backward(d, segs, (char*)workspace, st) : backward_f32(d, segs, (float*)workspace, st);
  }
  return e == cudaSuccess ? PBT_OK : fail(PBT_ERR_CUDA, cudaGetErrorString(e));
}
