// Low-rank adapters of many requests (or members) at once beside one shared, frozen projection:
//   S = x A_a^T,  y = x W^T + bias + c_a S B_a^T        (a: the adapter of the row's segment)
//   dS = c_a dy B_a,  dx = dy W + dS A_a,  dA_a = sum dS^T x,  dB_a = c_a sum dy^T S
// The entry points and the fp32 kernels.
//
// fp32 runs on the ALUs: one pass over the rows for the low-rank operand, then the shared product with the low-rank one as
// further blocks of the same contraction.
#include <algorithm>
#include <type_traits>

#include "adapters.cuh"
#include "tc_common.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace adapters {
namespace {

// s[row][j] = f sum_k x[row][k] m_a(j, k); m_a is A_a [rank][K] or, TRANS, B_a [K][rank]; f: the adapter's scale or 1.  A warp has
// R rows and 8 ranks, its lanes every 32nd k; where the rows are of several segments, it goes over them once for each.
// A call's time is latency: 871 rows x 104, rank 64, 8.4 us; a warp for a row and all ranks one after the other took 45.
template <bool TRANS, int R>
__global__ void __launch_bounds__(256) k_adapter_shrink_f32(const float* __restrict__ x, long long ldx, int K, const float* __restrict__ mats,
                                                            int rank, const float* __restrict__ scale, Segments segs,
                                                            float* __restrict__ s) {
  pdl_prologue();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the product may begin with its own operands
  const int lane = threadIdx.x & 31, rank_groups = (rank + 7) / 8, w = blockIdx.x * 8 + (threadIdx.x >> 5);
  const int row0 = w / rank_groups * R, r0 = w % rank_groups * 8, rows = min(R, segs.rows - row0);
  if (rows <= 0) return;
  const int ranks = min(8, rank - r0);
  for (int j = max(segment_of_row_warp(segs, row0), 0); j < segs.n; ++j) {
    const int lo = max(segment_begin(segs, j), row0), hi = min(segment_begin(segs, j + 1), row0 + rows), a = segment_adapter(segs, j);
    if (segment_begin(segs, j) >= row0 + rows) return;
    if (a < 0 || lo >= hi) continue;
    const float* m = mats + (long long)a * rank * K + (TRANS ? r0 : (long long)r0 * K);
    float acc[R * 8] = {};
#pragma unroll (R == 1 ? 4 : 2)
    for (int k = lane; k < K; k += 32) {
      float v[R], f[8];
#pragma unroll
      for (int u = 0; u < R; ++u) v[u] = x[(row0 + min(u, rows - 1)) * ldx + k];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < ranks ? (TRANS ? m[(long long)k * rank + i] : m[(long long)i * K + k]) : 0.f;
#pragma unroll
      for (int u = 0; u < R; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[u * 8 + i] = __fmaf_rn(v[u], f[i], acc[u * 8 + i]);
    }
    // lane l ends with the sum of acc[l] over the lanes (R = 4): half of the values change hands in every step.  With one row
    // the lanes of a group of eight hold its eight sums of their group, which are added up first.
#pragma unroll
    for (int o = 16; o >= R * 8; o >>= 1)
#pragma unroll
      for (int i = 0; i < R * 8; ++i) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], o);
#pragma unroll
    for (int o = R * 4; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < o; ++i) {
        const bool up = lane & o;
        const float give = up ? acc[i] : acc[i + o], keep = up ? acc[i + o] : acc[i];
        acc[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, o);
      }
    const int row = R == 1 ? (lane < 8 ? row0 : -1) : row0 + (lane >> 3), i = lane & 7;
    if (row >= lo && row < hi && i < ranks) s[(long long)row * rank + r0 + i] = (scale ? scale[a] : 1.f) * acc[0];
  }
}

// C = X W^T + bias + f_a S m_a^T over tiles of BM rows and BN columns.  W is [N][K] and m_a [N][rank] or, TRANS, [K][N] and
// [rank][N]; S is [rows][rank].  The contraction runs in chunks of BK: X and W first, then, for every segment with rows in
// the tile, S and its adapter's matrix, whose products are added to the segment's rows alone (not multiplied by zero elsewhere: a
// diverged adapter reaches its own rows only).  The CTA's threads are KG groups that share a chunk's k, so that small tiles keep
// eight warps busy.  Chunks come by cp.async, 16 bytes at a time where the operand's rows allow it, else element by element.
// Bound by the ALUs' issue: 2048 x 256 -> 512, rank 4 takes 26 us, 0.28 of the fp32 rate; 8192 x 512 -> 512 about 140 us, 0.4.
// A narrow tile with more segments than 2 + rank / 16 leaves the low-rank part to its last step, where every thread multiplies out its own
// elements (60 single rows, 72 -> 200, rank 4: a whole call 11 us, with chunks 24; 871 rows in segments of 13, 104 -> 152, rank 64, which has
// chunks: 18.5 us, element by element 25).
// A thread's rows and columns are BM / TM and BN / TN apart (columns of a TRANS chunk adjacent): the vectors that a warp reads
// then lie in different banks.
template <int BM_, int BN_, int TM_, int TN_, int BK_, int STAGES_>
struct ProductShape {
  static constexpr int BM = BM_, BN = BN_, TM = TM_, TN = TN_, BK = BK_, STAGES = STAGES_;
  static constexpr int kRowThreads = BM / TM, kColThreads = BN / TN, kGroupThreads = kRowThreads * kColThreads, KG = 256 / kGroupThreads;
  static constexpr int kPerGroup = BK / KG;
  static constexpr int PK = BK + 4, PN = BN + 4;       // pitches of rows of k and of columns
  static constexpr int kA = BM * PK, kB = BN * PK > BK * PN ? BN * PK : BK * PN, kStage = kA + kB;
  static constexpr int kBytes = (STAGES * kStage > KG * BM * BN ? STAGES * kStage : KG * BM * BN) * 4;
  static_assert(BM <= 64 && TN == 4 && BK % 4 == 0 && kPerGroup % 4 == 0 && KG * kPerGroup == BK, "tile shape");
};
typedef ProductShape<64, 64, 8, 4, 32, 3> ProductWide;
typedef ProductShape<16, 32, 4, 4, 64, 3> ProductNarrow;
// Wide tiles from this many of them on: a whole call of 1024 rows, 256 -> 384, rank 16 (96 wide tiles) 24.7 us, narrow ones 28; 256 -> 256 (64)
// 22.6 both; 871 rows, 104 -> 152, rank 64 (42) 35 us, narrow ones 18.
constexpr long long kWideTiles = 64;

struct ProductArgs {
  const float* x; long long ldx;
  const float* w; long long ldw;
  const float* bias;
  float* y; long long ldy;
  int N, K;
  const float* s; const float* mats; int rank;
  const float* scale;              // or null: S is scaled already
  Segments segs;
  bool vec_x, vec_w, vec_s, vec_m; // rows of 16-byte vectors
};

// `bytes` of a vector or an element (the rest is filled with zeros)
template <int N>
__device__ __forceinline__ void copy_part(uint32_t to, const float* from, int bytes) {
  if (N == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
// A box of ROWS rows and COLS elements into rows of PITCH, `rows` and `cols` of which exist.
template <int ROWS, int COLS, int PITCH, int N>
__device__ __forceinline__ void copy_box(uint32_t to, const float* from, long long ld, int rows, int cols) {
#pragma unroll
  for (int i = 0; i < ROWS * COLS / N / 256; ++i) {
    const int q = i * 256 + threadIdx.x, row = q / (COLS / N), c = q % (COLS / N) * N;
    const int have = row < rows ? min(max(cols - c, 0), N) : 0;
    copy_part<N>(to + (row * PITCH + c) * 4, have ? from + row * ld + c : from, have * 4);
  }
}
template <int ROWS, int COLS, int PITCH>
__device__ __forceinline__ void copy_box(uint32_t to, const float* from, long long ld, int rows, int cols, bool vectors) {
  if (vectors) copy_box<ROWS, COLS, PITCH, 4>(to, from, ld, rows, cols);
  else copy_box<ROWS, COLS, PITCH, 1>(to, from, ld, rows, cols);
}

template <typename P, bool TRANS>
__global__ void __launch_bounds__(256, 2) k_adapter_product_f32(const ProductArgs a) {
  extern __shared__ __align__(16) float product_smem[];
  __shared__ int seg_lo[P::BM], seg_hi[P::BM], seg_adapter[P::BM], n_segs;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int tiles_n = (a.N + P::BN - 1) / P::BN, row0 = (int)(blockIdx.x / tiles_n) * P::BM, n0 = (int)(blockIdx.x % tiles_n) * P::BN;
  const int rows = min(P::BM, a.segs.rows - row0), cols = min(P::BN, a.N - n0);
  const int chunks = (a.K + P::BK - 1) / P::BK, low_chunks = (a.rank + P::BK - 1) / P::BK;
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(product_smem);

  auto load = [&](int t) {
    const uint32_t sa = base + (t % P::STAGES) * P::kStage * 4, sb = sa + P::kA * 4;
    const bool main = t < chunks;
    const int k0 = (main ? t : (t - chunks) % low_chunks) * P::BK, K = main ? a.K : a.rank;
    const float* B = main ? a.w : a.mats + (long long)seg_adapter[(t - chunks) / low_chunks] * a.rank * a.N;
    const long long lda = main ? a.ldx : a.rank, ldb = main ? a.ldw : TRANS ? a.N : a.rank;
    copy_box<P::BM, P::BK, P::PK>(sa, (main ? a.x : a.s) + row0 * lda + k0, lda, rows, K - k0, main ? a.vec_x : a.vec_s);
    if (TRANS) copy_box<P::BK, P::BN, P::PN>(sb, B + k0 * ldb + n0, ldb, K - k0, cols, main ? a.vec_w : a.vec_m);
    else copy_box<P::BN, P::BK, P::PK>(sb, B + n0 * ldb + k0, ldb, cols, K - k0, main ? a.vec_w : a.vec_m);
  };

  const int first = min(P::STAGES - 1, chunks);
  for (int t = 0; t < first; ++t) {
    load(t);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // the segments that have an adapter and rows in the tile, in order
  if (warp == 0) {
    int n = 0;
    for (int j0 = max(segment_of_row_warp(a.segs, row0), 0); j0 < a.segs.n; j0 += 32) {
      const int j = min(j0 + lane, a.segs.n - 1), begin = segment_begin(a.segs, j) - row0, end = segment_begin(a.segs, j + 1) - row0;
      const int adapter = segment_adapter(a.segs, j), lo = max(begin, 0), hi = min(end, rows);
      const bool counts = j0 + lane < a.segs.n && adapter >= 0 && lo < hi;
      const unsigned int all = __ballot_sync(0xFFFFFFFFu, counts);
      const int q = n + __popc(all & ((1u << lane) - 1u));
      if (counts && q < P::BM) { seg_lo[q] = lo; seg_hi[q] = hi; seg_adapter[q] = adapter; }
      n = min(n + __popc(all), P::BM);
      if (__any_sync(0xFFFFFFFFu, begin >= rows)) break;
    }
    if (lane == 0) n_segs = n;
  }
  __syncthreads();
  const bool direct = P::BM <= 16 && n_segs > 2 + a.rank / 16;
  const int turns = chunks + (direct ? 0 : n_segs * low_chunks);
  // S is there from here on; k_adapter_grad_f32 may begin, too: it needs dS and nothing of this kernel's
  bool waited = false;
  auto low_rank = [&]() {
    if (!waited) asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");
    waited = true;
  };
  for (int t = first; t < P::STAGES - 1; ++t) {
    low_rank();
    if (t < turns) load(t);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  const int group = tid / P::kGroupThreads, g = tid % P::kGroupThreads, tx = g % P::kColThreads, ty = g / P::kColThreads;
  float acc[P::TM][P::TN] = {};
  auto column = [&](int e) { return TRANS ? tx * P::TN + e : tx + e * P::kColThreads; };
#pragma unroll 1
  for (int t = 0; t < turns; ++t) {
    asm volatile("cp.async.wait_group %0;" ::"n"(P::STAGES - 2) : "memory");
    __syncthreads();
    if (t + P::STAGES - 1 >= chunks) low_rank();
    if (t + P::STAGES - 1 < turns) load(t + P::STAGES - 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const float *sa = product_smem + (t % P::STAGES) * P::kStage, *sb = sa + P::kA;
    auto multiply = [&](auto whole, int lo, int hi, float f) {
#pragma unroll
      for (int k = 0; k < P::kPerGroup; k += 4) {
        const int kk = group * P::kPerGroup + k;
        float v[4][P::TN];       // [k][column]
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 q = *reinterpret_cast<const float4*>(TRANS ? sb + (kk + i) * P::PN + column(0) : sb + column(i) * P::PK + kk);
          if (TRANS) { v[i][0] = q.x; v[i][1] = q.y; v[i][2] = q.z; v[i][3] = q.w; }
          else { v[0][i] = q.x; v[1][i] = q.y; v[2][i] = q.z; v[3][i] = q.w; }
        }
#pragma unroll
        for (int i = 0; i < P::TM; ++i) {
          const int row = ty + i * P::kRowThreads;
          if (!whole.value && (row < lo || row >= hi)) continue;
          const float4 q = *reinterpret_cast<const float4*>(sa + row * P::PK + kk);
          const float u[4] = {whole.value ? q.x : q.x * f, whole.value ? q.y : q.y * f, whole.value ? q.z : q.z * f, whole.value ? q.w : q.w * f};
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int e = 0; e < P::TN; ++e) acc[i][e] = __fmaf_rn(u[x], v[x][e], acc[i][e]);
        }
      }
    };
    if (t < chunks) {
      multiply(std::true_type(), 0, P::BM, 1.f);
    } else {
      const int q = (t - chunks) / low_chunks;
      multiply(std::false_type(), seg_lo[q], seg_hi[q], a.scale ? __ldg(a.scale + seg_adapter[q]) : 1.f);
    }
  }

  low_rank();
  // the groups' sums, in their order
  __syncthreads();
#pragma unroll
  for (int i = 0; i < P::TM; ++i)
#pragma unroll
    for (int e = 0; e < P::TN; ++e) product_smem[(group * P::BM + ty + i * P::kRowThreads) * P::BN + column(e)] = acc[i][e];
  __syncthreads();
  const int n = tid % P::BN;
  if (n >= cols) return;
  const float bias = a.bias ? a.bias[n0 + n] : 0.f;
  for (int row = tid / P::BN; row < rows; row += 256 / P::BN) {
    float v = product_smem[row * P::BN + n];
#pragma unroll
    for (int q = 1; q < P::KG; ++q) v += product_smem[(q * P::BM + row) * P::BN + n];
    if (direct)
      for (int q = 0; q < n_segs; ++q) {
        if (row < seg_lo[q] || row >= seg_hi[q]) continue;
        const int adapter = seg_adapter[q];
        const float* s = a.s + (long long)(row0 + row) * a.rank;      // (written while this kernel runs already: no read-only loads)
        const float* m = a.mats + (long long)adapter * a.rank * a.N + (TRANS ? n0 + n : (long long)(n0 + n) * a.rank);
        float low = 0.f;
        if (!TRANS && a.vec_s && a.vec_m) {
#pragma unroll 8
          for (int j = 0; j < a.rank; j += 4) {
            const float4 u = __ldcg(reinterpret_cast<const float4*>(s + j)), w = __ldg(reinterpret_cast<const float4*>(m + j));
            low = __fmaf_rn(u.x, w.x, __fmaf_rn(u.y, w.y, __fmaf_rn(u.z, w.z, __fmaf_rn(u.w, w.w, low))));
          }
        } else {
#pragma unroll 8
          for (int j = 0; j < a.rank; ++j) low = __fmaf_rn(__ldcg(s + j), __ldg(TRANS ? m + (long long)j * a.N : m + j), low);
        }
        v = __fmaf_rn(a.scale ? __ldg(a.scale + adapter) : 1.f, low, v);
        break;
      }
    a.y[(row0 + row) * a.ldy + n0 + n] = v + bias;
  }
}

template <typename P, bool TRANS>
cudaError_t launch_product(const ProductArgs& a, cudaStream_t st) {
  static tc::DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = tc::device_setup(&setup, k_adapter_product_f32<P, TRANS>, P::kBytes, &sms);
  if (e != cudaSuccess) return e;
  const unsigned tiles = (unsigned)(((a.segs.rows + P::BM - 1) / P::BM) * (long long)((a.N + P::BN - 1) / P::BN));
  // Narrow tiles begin while the shrink runs (64 single rows, 256 -> 256: 12.3 us, after it 14.5).  Wide ones would crowd on the SMs that it leaves
  // free, and a CTA that shares its SM takes twice its time (1024 rows 256 -> 256: 31 us, after it 22.6).
  if (P::BM <= 16) return launch_after(tiles, 256, P::kBytes, st, k_adapter_product_f32<P, TRANS>, a);
  return launch_with(tiles, 256, P::kBytes, st)(k_adapter_product_f32<P, TRANS>, a);
}
template <bool TRANS>
cudaError_t launch_product(ProductArgs a, cudaStream_t st) {
  auto vectors = [](const float* p, long long ld) { return ((uintptr_t)p & 15) == 0 && ld % 4 == 0; };
  a.vec_x = vectors(a.x, a.ldx);
  a.vec_w = vectors(a.w, a.ldw);
  a.vec_s = vectors(a.s, a.rank);
  a.vec_m = vectors(a.mats, TRANS ? a.N : a.rank);
  const long long wide = ((a.segs.rows + 63) / 64) * (long long)((a.N + 63) / 64);
  return wide >= kWideTiles ? launch_product<ProductWide, TRANS>(a, st) : launch_product<ProductNarrow, TRANS>(a, st);
}

struct GradSide {
  const float* v; long long ldv;
  const float* s;
  const float* scale;        // or null
  float* g; long long split; // result, and the distance from one split's partial result to the next one's
  int N, blocks;
  bool columns_first;        // g is [N][rank], else [rank][N]
};

// g_a(j, n) = f_a sum over the rows of adapter a of s[row][j] v[row][n]: dA from (dS, x) and dB from (S, dy) in one launch.  A
// block owns 64 columns of one adapter and side and one split of the rows; its 256 threads are four parts, which have a quarter
// of the ranks each (beyond rank 32: 64 accumulators a thread keep too few rows in flight; 2048 rows, 64 -> 512, rank 64: a whole pass
// 156 us, by rows 221), or every fourth row (added up in shared memory; 256 -> 512, rank 32: 118 us, by ranks, which read every row
// four times, 139).
template <int RANK>
__global__ void __launch_bounds__(256, RANK == 32 ? 3 : 4) k_adapter_grad_f32(const GradSide x, const GradSide dy, int rank, Segments segs) {
  constexpr bool kByRank = RANK >= 64;
  constexpr int R = kByRank ? RANK / 4 : RANK, kRowParts = kByRank ? 1 : 4;
  __shared__ float sum[kByRank ? 1 : 3][kByRank ? 1 : RANK][64];
  const bool second = (int)blockIdx.x >= x.blocks;
  const GradSide& side = second ? dy : x;
  const int col = threadIdx.x & 63, part = threadIdx.x >> 6, n = ((int)blockIdx.x - (second ? x.blocks : 0)) * 64 + col, a = blockIdx.y;
  const int r0 = kByRank ? part * R : 0, first = kByRank ? 0 : part, ranks = min(R, rank - r0);
  const int from = (int)((long long)segs.rows * blockIdx.z / gridDim.z), to = (int)((long long)segs.rows * (blockIdx.z + 1) / gridDim.z);
  const float* v = side.v + min(n, side.N - 1);
  const bool vectors = ranks == R && R % 4 == 0 && rank % 4 == 0 && ((uintptr_t)side.s & 15) == 0;
  float acc[R] = {};
  for (int j = 0; j < segs.n; ++j) {
    if (segment_adapter(segs, j) != a) continue;
    const int end = min(segment_begin(segs, j + 1), to);
    for (int row = max(segment_begin(segs, j), from) + first; row < end; row += 4 * kRowParts) {
      float y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = row + kRowParts * u < end ? v[(row + kRowParts * u) * side.ldv] : 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (row + kRowParts * u >= end) continue;
        const float* sr = side.s + (long long)(row + kRowParts * u) * rank + r0;
        if (vectors) {
#pragma unroll
          for (int i = 0; i < R / 4; ++i) {
            const float4 q = __ldg(reinterpret_cast<const float4*>(sr) + i);
            acc[4 * i] = __fmaf_rn(q.x, y[u], acc[4 * i]);
            acc[4 * i + 1] = __fmaf_rn(q.y, y[u], acc[4 * i + 1]);
            acc[4 * i + 2] = __fmaf_rn(q.z, y[u], acc[4 * i + 2]);
            acc[4 * i + 3] = __fmaf_rn(q.w, y[u], acc[4 * i + 3]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < R; ++i) if (i < ranks) acc[i] = __fmaf_rn(__ldg(sr + i), y[u], acc[i]);
        }
      }
    }
  }
  if (!kByRank) {
    if (part > 0)
#pragma unroll
      for (int i = 0; i < R; ++i) sum[part - 1][i][col] = acc[i];
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int i = 0; i < R; ++i) acc[i] += sum[0][i][col] + sum[kByRank ? 0 : 1][i][col] + sum[kByRank ? 0 : 2][i][col];
  }
  if (n >= side.N) return;
  const float f = side.scale ? side.scale[a] : 1.f;
  float* out = side.g + blockIdx.z * side.split + (long long)a * rank * side.N;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < ranks) out[side.columns_first ? (long long)n * rank + r0 + i : (long long)(r0 + i) * side.N + n] = f * acc[i];
  asm volatile("griddepcontrol.wait;" ::: "memory");     // what follows in the stream follows the product, too (every block has a thread here)
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
  // the kernels work out the ends of their tiles in 32 bits
  constexpr int kMost = 0x7FFFFFFF - 4096;
  if (d->rows > kMost || d->inputs > kMost || d->outputs > kMost || d->n_segments > (1 << 30))
    return fail(PBT_ERR_UNSUPPORTED, "more than 2^31 - 4097 rows, inputs or outputs, or more than 2^30 segments");
  if (d->rank < 1 || d->rank > kMaxRank) return fail(PBT_ERR_UNSUPPORTED, "rank must be in [1, 64]");
  if (d->n_adapters > 65535) return fail(PBT_ERR_UNSUPPORTED, "more than 65535 adapters");
  if (d->dtype != 0 && d->dtype != 1) return fail(PBT_ERR_UNSUPPORTED, "operands are float or bfloat16");
  if (!d->weight || !d->A || !d->B || !d->scale || !d->row_offsets || (d->n_segments && !d->adapter_ids))
    return fail(PBT_ERR_INVALID_ARG, "weight, A, B, scale, row_offsets or adapter_ids is NULL");
  if (d->dtype == 1 && !d->status_device) return fail(PBT_ERR_INVALID_ARG, "status_device is required by the tensor-core kernels");
  if (d->ld_weight < d->inputs) return fail(PBT_ERR_INVALID_ARG, "ld_weight is smaller than inputs");
  return PBT_OK;
}

size_t low_rank_bytes(const pbt_adapter_desc* d) { return ((size_t)d->rows * d->rank * sizeof(float) + 255) & ~(size_t)255; }

// Splits of the rows in the gradients' kernel: a block for every SM, 64 rows of the call at least.
int grad_splits_f32(const pbt_adapter_desc* d) {
  const long long blocks = ((d->inputs + 63) / 64 + (d->outputs + 63) / 64) * (long long)d->n_adapters;
  return (int)std::max<long long>(1, std::min<long long>((147 + blocks) / blocks, d->rows / 64));
}

// Up to two waves of warps with a row each, beyond that four rows to a warp, which read the adapter's matrix once for all (80 single rows,
// 512 -> 512, rank 64: a whole call 33 us with one row, 43 with four; 8192 rows in segments of 128, rank 16: 181 and 166).
constexpr long long kShrinkWarps = 148 * 16;
template <bool TRANS>
cudaError_t launch_shrink_f32(const float* x, long long ldx, int K, const float* mats, int rank, const float* scale, const Segments& segs, float* s,
                              cudaStream_t st) {
  const long long groups = (rank + 7) / 8;
  auto blocks = [&](int rows) { return (unsigned)(((long long)((segs.rows + rows - 1) / rows) * groups + 7) / 8); };
  if (segs.rows * groups <= kShrinkWarps) return launch_with(blocks(1), 256, 0, st)(k_adapter_shrink_f32<TRANS, 1>, x, ldx, K, mats, rank, scale, segs, s);
  return launch_with(blocks(4), 256, 0, st)(k_adapter_shrink_f32<TRANS, 4>, x, ldx, K, mats, rank, scale, segs, s);
}

cudaError_t forward_f32(const pbt_adapter_desc* d, const Segments& segs, float* ws, cudaStream_t st) {
  float *s = d->s ? d->s : ws, *y = (float*)d->y;
  const float *x = (const float*)d->x, *A = (const float*)d->A, *B = (const float*)d->B, *w = (const float*)d->weight;
  const cudaError_t e = launch_shrink_f32<false>(x, d->ld_x, d->inputs, A, d->rank, nullptr, segs, s, st);
  if (e != cudaSuccess) return e;
  return launch_product<false>({x, d->ld_x, w, d->ld_weight, d->bias, y, d->ld_y, d->outputs, d->inputs, s, B, d->rank, d->scale, segs}, st);
}

cudaError_t backward_f32(const pbt_adapter_desc* d, const Segments& segs, float* ds, cudaStream_t st) {
  const float *x = (const float*)d->x, *dy = (const float*)d->dy, *A = (const float*)d->A, *B = (const float*)d->B, *w = (const float*)d->weight;
  cudaError_t e = launch_shrink_f32<true>(dy, d->ld_dy, d->outputs, B, d->rank, d->scale, segs, ds, st);
  if (e != cudaSuccess) return e;
  e = launch_product<true>({dy, d->ld_dy, w, d->ld_weight, nullptr, (float*)d->dx, d->ld_dx, d->inputs, d->outputs, ds, A, d->rank, nullptr, segs}, st);
  if (e != cudaSuccess) return e;
  const int splits = grad_splits_f32(d);
  const long long size_a = (long long)d->n_adapters * d->rank * d->inputs, size_b = (long long)d->n_adapters * d->rank * d->outputs;
  float* parts = (float*)((char*)ds + low_rank_bytes(d));
  const GradSide a = {x, d->ld_x, ds, nullptr, splits > 1 ? parts : d->dA, size_a, d->inputs, (d->inputs + 63) / 64, false};
  const GradSide b = {dy, d->ld_dy, d->s, d->scale, splits > 1 ? parts + splits * size_a : d->dB, size_b, d->outputs, (d->outputs + 63) / 64, true};
  e = with_rank(d->rank, [&](auto r) {
    return launch_after(dim3(a.blocks + b.blocks, d->n_adapters, splits), 256, 0, st, k_adapter_grad_f32<decltype(r)::value>, a, b, d->rank, segs);
  });
  return e == cudaSuccess && splits > 1 ? join_gradients(a.g, b.g, size_a, size_b, splits, d->dA, d->dB, st) : e;
}

// fp32: S of a forward pass that does not keep it; dS of a backward pass and the splits' partial gradients
size_t workspace_bytes(const pbt_adapter_desc* d, bool backward) {
  if (d->dtype) return tc_workspace(d, backward);
  const int splits = backward ? grad_splits_f32(d) : 1;
  const size_t parts = splits > 1 ? (size_t)splits * d->n_adapters * d->rank * ((size_t)d->inputs + d->outputs) * sizeof(float) : 0;
  return std::max<size_t>(256, low_rank_bytes(d) + parts);
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
