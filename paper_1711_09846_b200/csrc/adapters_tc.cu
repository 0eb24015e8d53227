// bf16 adapters on the tensor cores.  Three kernels carry both directions:
//
//   k_adapter_shrink   S = x A_a^T (or dS = c dy B_a): a product with r <= 64 columns, bound by reading x once; rows of
//                      one (tile of at most 64 rows, segment) pair per CTA, mma.sync fed by 16-byte loads straight from global memory
//   k_adapter_gemm     y = x W^T + bias + c S B_a^T (or dx = dy W + dS A_a): the shared product on tcgen05, with the
//                      low-rank product as one more block of the same contraction in the same TMEM accumulator
//   k_adapter_rows     the same product for a few rows (one token of many requests): bound by reading W once, mma.sync
//                      with W's rows as the tall operand, low-rank part in fp32 at the end
//   k_adapter_grad     dA_a = dS^T x, dB_a = dy^T (c S): contractions over an adapter's rows on tcgen05, r columns wide
//
// Segments and tiles.  Output tiles are 128 consecutive rows whatever the segments; for every segment that reaches into
// a tile the low-rank block is issued once with that adapter's matrix and with the other segments' rows switched off in
// the instruction (the disable-output-lane mask: a TMEM lane is a row).  Rows are therefore independent of one another's
// adapters exactly, not up to a multiplication with zero: an adapter that has diverged to NaN reaches only its own rows.
//
// Precision.  S and dS are fp32, the tensor cores take bf16.  The low-rank operand of a bf16 result is S (dS) as the sum of two bf16
// numbers, which leaves out less than 2^-16 of it, 2^-7 of what the result's own rounding does; one number (2^-9) raised the error of
// y on 3001 ragged rows, rank 8, from 0.00166 to 0.00181.  dA and dB are fp32 results, so their operand is the sum of
// three (24 bits), whose three products land in separate accumulator columns and are added in fp32.  The tensor
// cores' accumulation truncates (about 2^-24 of the accumulator per instruction), so chains are kept short: the shrink
// folds its accumulators into fp32 registers every 64 columns, the gradients every 128 rows.
#include <algorithm>
#include <type_traits>

#include "adapters.cuh"
#include "tc_epilogue.cuh"

namespace pbt {
namespace adapters {
namespace {

using namespace tc;

// ------------------------------------------------------------------------------------------------------------------
// Operands whose rows are not multiples of 16 bytes are copied once into rows that are.
// ------------------------------------------------------------------------------------------------------------------
struct PackJob {
  const bf16* src; long long ld;
  bf16* dst;
  long long rows;
  int cols, to;                // elements of a row, and rounded up to 8
  unsigned block0;             // its first block
};
struct PackJobs {
  PackJob job[5];
  int n;
};
// All operands of a call in one launch; a thread has 8 elements.
__global__ void __launch_bounds__(256) k_pack_rows(const PackJobs a) {
  pdl_prologue();
  int q = 0;
  while (q + 1 < a.n && blockIdx.x >= a.job[q + 1].block0) ++q;
  const PackJob j = a.job[q];
  const long long i = (long long)(blockIdx.x - j.block0) * 256 + threadIdx.x;
  const int per_row = j.to / 8;
  const long long row = i / per_row;
  if (row >= j.rows) return;
  const int c = (int)(i - row * per_row) * 8;
  const bf16* from = j.src + row * j.ld + c;
  __align__(16) bf16 v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c + e < j.cols ? from[e] : __float2bfloat16_rn(0.f);
  *reinterpret_cast<uint4*>(j.dst + row * j.to + c) = *reinterpret_cast<const uint4*>(v);
}

// ------------------------------------------------------------------------------------------------------------------
// Shrink
// ------------------------------------------------------------------------------------------------------------------

struct ShrinkArgs {
  const bf16* x; long long ldx; int K;
  const bf16* mats; int pitch;        // A_a [rank][pitch] (K of them used), or B_a [K][pitch] (rank of them used)
  int rank, rp;                       // rp: columns of a plane, the rank rounded up to 16
  const float* scale;
  Segments segs;
  int tile, n_tiles;                  // rows of a tile
  float* s;                           // fp32 result, not scaled (may be null)
  float* scaled;                      // scaled fp32 result [rows][rank], for k_adapter_rows (null: planes instead)
  int* row_adapter;                   // adapter of every row or -1, for k_adapter_rows
  bf16* planes; int terms;            // scaled result as `terms` bf16 summands side by side, [rows][terms * rp]
  const float* kept; bf16* kept_planes;   // a second fp32 matrix [rows][rank], split into three summands the same way
  int* tile_seg; int tile_rows, n_table;  // first segment of every output tile of the product that follows
};

__device__ __forceinline__ void copy16(void* slot, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(slot)), "l"(from) : "memory");
}
__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// The next bf16 summand of v, which becomes the rest.  Nothing is left of an infinite v (inf - inf would make its row NaN); a finite
// one beyond the largest bf16 is cut instead of rounded, so that it stays finite.
__device__ __forceinline__ float next_term(float& v) {
  float h = __bfloat162float(__float2bfloat16_rn(v));
  if (isinf(h)) h = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);
  v = isinf(h) ? 0.f : v - h;
  return h;
}
// two neighbouring columns (col is even), as two summands or three
__device__ __forceinline__ void store_terms(bf16* row, int rp, int col, float v0, float v1, bool three) {
#pragma unroll
  for (int t = 0; t < 3; ++t) {
    if (t == 2 && !three) return;
    const float h0 = next_term(v0), h1 = next_term(v1);
    *reinterpret_cast<__nv_bfloat162*>(row + t * rp + col) = __floats2bfloat162_rn(h0, h1);
  }
}

// A warp multiplies 32 rows by the adapter's matrix over every `parts`-th block of 64 columns.  The columns of a block are
// dealt to the fragments in the order in which 16-byte loads deliver them (lane t of a quad holds columns 8t .. 8t+7 of
// each half block); the sum over k does not mind, as long as both operands use the same order.  B_a lies with its ranks
// contiguous, so its fragments are transposed on the way: 64 rows of it lie in shared memory in an order in which the
// eight rows one ldmatrix takes are 128 consecutive bytes.
// What bounds it is the bytes in flight: the blocks come through shared memory (cp.async, a warp's own ring of kShrinkStages
// blocks, every lane reading back what it copied itself), 2 x 96 KB per SM at rank 16.
template <int NT> struct ShrinkRing {
  static constexpr int kStages = NT <= 2 ? 2 : NT == 4 ? 3 : 2;    // two CTAs of an SM share 227 KB up to rank 16, one beyond
  static constexpr int kBytes = 4096 + NT * 1024;                  // a block of a warp: 32 rows of x, 8 NT rows of the matrix
  static constexpr int kTotal = 8 * kStages * kBytes;
};
template <bool TRANS, int NT>
__global__ void __launch_bounds__(256, NT <= 2 ? 2 : 1) k_adapter_shrink(const ShrinkArgs a) {
  pdl_prologue();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (k_adapter_rows may begin with its own operand)
  extern __shared__ __align__(16) uint8_t shrink_smem[];
  typedef ShrinkRing<NT> Ring;
  const int q = blockIdx.x, tid = threadIdx.x;
  const Segments& g = a.segs;
  if (q >= a.n_tiles + g.n) {
    const int i = (q - a.n_tiles - g.n) * 256 + tid;
    if (i >= a.n_table) return;
    const int row = i * a.tile_rows, j = segment_of_row(g, row);
    if (a.row_adapter) a.row_adapter[i] = j >= 0 && row < segment_begin(g, j + 1) ? segment_adapter(g, j) : -1;
    else a.tile_seg[i] = max(j, 0);
    return;
  }
  // The pairs (tile t, segment j) that meet ascend in t + j by at least one, so q = t + j names at most one of them: j is
  // the last segment whose first pair is not behind q.
  int j = -1;
  for (int base = 0; base < g.n; base += 256) {
    const int i = base + tid;
    j += __syncthreads_count(i < g.n && segment_begin(g, i) / a.tile + i <= q);
  }
  if (j < 0) return;
  const int t = q - j;
  const int adapter = segment_adapter(g, j);
  const int lo = max(segment_begin(g, j), t * a.tile), hi = min(segment_begin(g, j + 1), min((t + 1) * a.tile, g.rows));
  if (lo >= hi || adapter < 0) return;

  const int warp = tid >> 5, lane = tid & 31, gr = lane >> 2, tq = lane & 3;
  const int groups = hi - lo > 32 ? 2 : 1, parts = 8 / groups;     // few rows: more warps share the columns
  const int group = warp / parts, part = warp % parts;
  const bool both = hi - lo > 16;     // rows for the second fragment of 16
  const int nt8 = TRANS ? a.pitch / 8 : (a.rank + 7) / 8;
  const bf16* mat = a.mats + (long long)adapter * (TRANS ? (long long)a.K : (long long)a.rank) * a.pitch;
  const bf16* xrow[4];
  bool in[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = lo + group * 32 + gr + 8 * i;
    in[i] = row < hi;
    xrow[i] = a.x + (long long)row * a.ldx;
  }
  uint8_t* ring = shrink_smem + warp * (Ring::kStages * Ring::kBytes);
  // rows behind the tile are never copied: zero
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int s = 0; s < Ring::kStages; ++s)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint8_t* to = ring + s * Ring::kBytes + h * 512 + lane * 16;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!in[i]) *reinterpret_cast<uint4*>(to + i * 1024) = zero;
    }
  auto ask = [&](int k0, int s) {
    uint8_t* to = ring + s * Ring::kBytes;
    if (k0 < a.K) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + h * 32 + tq * 8;
        if (k < a.K) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (in[i]) copy16(to + (2 * i + h) * 512 + lane * 16, xrow[i] + k);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(to + (2 * i + h) * 512 + lane * 16) = zero;     // behind the last column
        }
        if constexpr (!TRANS) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const int r = n * 8 + gr;
            uint8_t* slot = to + 4096 + (2 * n + h) * 512 + lane * 16;
            if (r < a.rank && k < a.K) copy16(slot, mat + (long long)r * a.pitch + k);
            else *reinterpret_cast<uint4*>(slot) = zero;
          }
        }
      }
      if constexpr (TRANS) {
        auto row_piece = [&](int k, int n) {
          uint8_t* slot = to + 4096 + n * 1024 + ((k & 32) + (k & 7) * 4 + ((k & 31) >> 3)) * 16;
          if (k0 + k < a.K) copy16(slot, mat + (long long)(k0 + k) * a.pitch + n * 8);
          else *reinterpret_cast<uint4*>(slot) = zero;
        };
        if (nt8 == NT) {
#pragma unroll
          for (int p = 0; p < 2 * NT; ++p) row_piece((p * 32 + lane) / NT, (p * 32 + lane) % NT);
        } else {
          for (int p = lane; p < 64 * nt8; p += 32) row_piece(p / nt8, p % nt8);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < Ring::kStages; ++s) ask(part * 64 + s * parts * 64, s);
  // the second matrix's elements that this thread splits at the end: a pair of columns each
  constexpr int kPairs = NT < 2 ? 2 : NT;
  const int half = a.rp / 2;
  const float f = __ldg(a.scale + adapter);
  float second[kPairs][2] = {};
  if (a.kept)
#pragma unroll
    for (int u = 0; u < kPairs; ++u) {
      const int i = tid + u * 256, r = i / half, c = i % half * 2;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (r < hi - lo && c + e < a.rank) second[u][e] = __ldg(a.kept + (long long)(lo + r) * a.rank + c + e);
    }
  float acc[2][NT][4] = {};
  int stage = 0;
  for (int k0 = part * 64; k0 < a.K; k0 += parts * 64) {
    asm volatile("cp.async.wait_group %0;" ::"n"(Ring::kStages - 1) : "memory");
    if constexpr (TRANS) __syncwarp();   // the other lanes' part of the matrix
    const uint8_t* from = ring + stage * Ring::kBytes;
    float sum[2][NT][4] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 xv[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) xv[i] = *reinterpret_cast<const uint4*>(from + (2 * i + h) * 512 + lane * 16);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (n >= nt8) continue;
        uint32_t b[4];   // two steps of 16 columns, two registers each
        if constexpr (TRANS) {
          // matrix m = lane / 8 holds, for step m / 2 and half m % 2, row 2t + e: column 8t + 4 (m / 2) + 2 (m % 2) + e of the block
          const int m = lane >> 3, c = lane & 7;
          ldmatrix4_trans(b, smem_u32(from) + 4096 + n * 1024 + (h * 32 + (4 * (m >> 1) + 2 * (m & 1) + (c & 1)) * 4 + (c >> 1)) * 16);
        } else {
          const uint4 bv = *reinterpret_cast<const uint4*>(from + 4096 + (2 * n + h) * 512 + lane * 16);
          b[0] = bv.x; b[1] = bv.y; b[2] = bv.z; b[3] = bv.w;
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int m = 0; m < 2; ++m)
            if (m == 0 || both) mma16816(sum[m][n], word(xv[2 * m], 2 * s), word(xv[2 * m + 1], 2 * s), word(xv[2 * m], 2 * s + 1), word(xv[2 * m + 1], 2 * s + 1),
                     b[2 * s], b[2 * s + 1]);
      }
    }
    if constexpr (TRANS) __syncwarp();   // every lane has read the block
    ask(k0 + Ring::kStages * parts * 64, stage);
    if (++stage == Ring::kStages) stage = 0;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[m][n][e] += sum[m][n][e];
  }
  __syncthreads();   // the rings' memory becomes the parts' sums: [warp][32 rows][8 NT]
  float* red = reinterpret_cast<float*>(shrink_smem);
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<float2*>(&red[(warp * 32 + m * 16 + gr + 8 * e) * (NT * 8) + n * 8 + tq * 2]) = make_float2(acc[m][n][2 * e], acc[m][n][2 * e + 1]);
  __syncthreads();
  const int width = a.terms * a.rp;
#pragma unroll
  for (int u = 0; u < kPairs; ++u) {
    const int i = tid + u * 256, r = i / half, c = i % half * 2;
    if (r >= hi - lo) break;
    const long long row = lo + r;
    float v[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (c + e < a.rank) {
        for (int p = 0; p < parts; ++p) v[e] += red[(((r >> 5) * parts + p) * 32 + (r & 31)) * (NT * 8) + c + e];
        if (a.s) a.s[row * a.rank + c + e] = v[e];
        if (a.scaled) a.scaled[row * a.rank + c + e] = f * v[e];
      }
    if (!a.planes) continue;
    store_terms(a.planes + row * width, a.rp, c, f * v[0], f * v[1], a.terms == 3);
    if (a.kept) store_terms(a.kept_planes + row * 3 * a.rp, a.rp, c, f * second[u][0], f * second[u][1], true);
  }
}

template <bool TRANS, int NT>
cudaError_t launch_shrink(const ShrinkArgs& a, unsigned grid, cudaStream_t s) {
  static DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = device_setup(&setup, k_adapter_shrink<TRANS, NT>, ShrinkRing<NT>::kTotal, &sms);
  if (e != cudaSuccess) return e;
  return launch_with(grid, 256, ShrinkRing<NT>::kTotal, s)(k_adapter_shrink<TRANS, NT>, a);
}
template <bool TRANS>
cudaError_t launch_shrink(ShrinkArgs a, cudaStream_t s) {
  // A CTA's time is its matrix instructions: smaller tiles, whose warps share the columns, while there are SMs for them (242 rows x 1496 -> 1096
  // in two segments, rank 64: a training step 72 us, with tiles of 64 rows 94)
  a.tile = 64;
  while (a.tile > 16 && a.segs.rows / a.tile + a.segs.n < 148) a.tile /= 2;
  a.n_tiles = (a.segs.rows + a.tile - 1) / a.tile;
  const unsigned grid = (unsigned)(a.n_tiles + a.segs.n + (a.n_table + 255) / 256);
  if (a.rank <= 8) return launch_shrink<TRANS, 1>(a, grid, s);
  if (a.rank <= 16) return launch_shrink<TRANS, 2>(a, grid, s);
  if (a.rank <= 32) return launch_shrink<TRANS, 4>(a, grid, s);
  return launch_shrink<TRANS, 8>(a, grid, s);
}

// ------------------------------------------------------------------------------------------------------------------
// Shared product with the low-rank block
// ------------------------------------------------------------------------------------------------------------------
// The wide tiles have four epilogue warps and a fourth stage where a CTA has several tiles (a training step of 40960 x 2048 -> 2048: 691 us,
// with eight warps and three stages 715; 10240 x 1024 -> 1024: 115 and 126), eight where its only tile's epilogue is not hidden behind
// the next one (3001 x 784 -> 1024, one wave: 19.1 us, with four warps 22.5).

// A segment's low-rank block is its two summands of S against the same matrix.  Up to rank 32 both lie in one stage of 64 columns,
// beyond it each has a stage, which brings the matrix again.
struct LowRank {
  Segments segs;
  const int* tile_seg;
  int rp;           // columns of a summand
  int stages;       // of a segment
  int steps;        // MMA steps of 16 ranks for a summand
};

// The segments that reach into rows [m0, m0 + tile_rows): walked in the same order by the roles of a CTA.
struct SegmentWalk {
  const Segments& g;
  int j, m0, m1;
  __device__ SegmentWalk(const Segments& segs, int first, int row0, int tile_rows) : g(segs), j(first), m0(row0), m1(min(row0 + tile_rows, segs.rows)) {}
  // next segment with an adapter and rows in the tile; false at the end
  __device__ bool next(int& adapter, int& lo, int& hi) {
    while (j < g.n) {
      const int b = segment_begin(g, j), e = segment_begin(g, j + 1);
      if (b >= m1) return false;
      adapter = segment_adapter(g, j);
      ++j;
      lo = max(b, m0);
      hi = min(e, m1);
      if (adapter >= 0 && lo < hi) return true;
    }
    return false;
  }
};

// bits of the rows of a 32-row group that starts at `base` and are NOT in [lo, hi)
__device__ __forceinline__ uint32_t rows_off(int base, int lo, int hi) {
  const int b = min(max(lo - base, 0), 32), e = min(max(hi - base, 0), 32);
  const uint32_t below_e = e >= 32 ? 0xFFFFFFFFu : (1u << e) - 1u, below_b = b >= 32 ? 0xFFFFFFFFu : (1u << b) - 1u;
  return ~(below_e & ~below_b);
}

// the lanes whose bit is set keep their accumulator
__device__ __forceinline__ void umma_bf16_rows(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, const uint32_t* off) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.eq.b32 p, 1, 1;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%4, %5, %6, %7}, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3])
      : "memory");
}

template <int BN, int STAGES, int EPI>
struct GemmSmem {
  static constexpr int kABytes = kBM * kBK * 2;
  static constexpr int kBBytes = BN * kBK * 2;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kEpiOffset = STAGES * kStageBytes;
  static constexpr int kEpiBytesPerWarp = 32 * kEpiPitch * 4;
  static constexpr int kBarOffset = kEpiOffset + EPI * kEpiBytesPerWarp;
  static constexpr int kTotal = kBarOffset + 256 + 1024;
  static_assert(kTotal <= 232448, "shared memory budget of one CTA");
};

// Roles as in the member-batched GEMM: warp 0 TMA producer, warp 1 MMA issuer, EPI epilogue warps, double-buffered
// accumulator.  After a tile's k-blocks both walk its segments: one more stage each (two beyond rank 32), 128 rows of the low-rank operand
// and the adapter's matrix (columns past the rank are out of the tensor map and arrive as zeros).  Launched while the shrink
// runs; the two threads that read what it leaves (the tiles' first segments, the planes through TMA) wait for its end
// after the k-blocks of their first tile.  From then on k_adapter_grad may begin beside it: it needs the shrink's results and none of
// this kernel's (training steps of 112 rows 87 -> 203: 45 us one after the other, 35 so; 1500 rows 1001 -> 603: 69 and 58).
template <int BN, int STAGES, int EPI, bool B_MN>
__global__ void __launch_bounds__(64 + 32 * EPI, 1)
k_adapter_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmP,
               const __grid_constant__ CUtensorMap tmL, const TcParams p, const LowRank low) {
  using L = GemmSmem<BN, STAGES, EPI>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBarOffset);
  uint64_t* empty = full + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint64_t* tempty = tfull + 2;
  uint64_t* idle = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(idle + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  constexpr uint32_t kTmemCols = 2 * BN;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(&tfull[a], 1); mbar_init(&tempty[a], EPI); }
    mbar_init(idle, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(tmem_slot, kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < p.num_tiles && ok; tile += gridDim.x) {
        const int tm = tile / p.tiles_n, m0 = tm * kBM, n0 = (tile % p.tiles_n) * BN;
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) { ok = false; break; }
          uint8_t* sa = smem + stage * L::kStageBytes;
          uint8_t* sb = sa + L::kABytes;
          mbar_expect_tx(&full[stage], L::kStageBytes);
          const int k0 = kb * kBK;
          tma_load_3d(sa, &tmA, &full[stage], k0, m0, 0);
          if constexpr (!B_MN) {
            tma_load_3d(sb, &tmB, &full[stage], k0, n0, 0);
          } else {
#pragma unroll
            for (int j = 0; j < BN / 64; ++j) tma_load_3d(sb + j * 8192, &tmB, &full[stage], n0 + j * 64, k0, 0);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (tile == blockIdx.x) asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");
        SegmentWalk walk(low.segs, __ldcg(low.tile_seg + tm), m0, kBM);
        int adapter, lo, hi;
        while (ok && walk.next(adapter, lo, hi))
          for (int part = 0; part < low.stages; ++part) {
            if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) { ok = false; break; }
            uint8_t* sa = smem + stage * L::kStageBytes;
            uint8_t* sb = sa + L::kABytes;
            mbar_expect_tx(&full[stage], L::kStageBytes);
            tma_load_3d(sa, &tmP, &full[stage], part * low.rp, m0, 0);
            if constexpr (!B_MN) {
              tma_load_3d(sb, &tmL, &full[stage], 0, n0, adapter);
            } else {
#pragma unroll
              for (int j = 0; j < BN / 64; ++j) tma_load_3d(sb + j * 8192, &tmL, &full[stage], n0 + j * 64, 0, adapter);
            }
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
          }
      }
      if (!ok) {
        *abort_flag = 1;
        atomicCAS(&p.counters->status, 0, PBT_ERR_TIMEOUT);
        p.counters->status_info = 31;
      }
      // every stage this thread armed has landed before the CTA exits, and been read unless a wait ran out
      for (int s = 0; s < STAGES; ++s) mbar_wait_out(&full[s], s < (int)stage ? phase : phase ^ 1);
      for (int s = 0; s < STAGES && ok; ++s) {
        if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) break;
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)B_MN << 16) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(kBM >> 4) << 24);
      uint32_t stage = 0, phase = 0;
      int it = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < p.num_tiles && ok; tile += gridDim.x, ++it) {
        const int tm = tile / p.tiles_n, m0 = tm * kBM;
        const int acc = it & 1;
        if (!mbar_wait(&tempty[acc], ((it >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t tmem_d = tmem_base + acc * BN;
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!mbar_wait(&full[stage], phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = smem_u32(smem + stage * L::kStageBytes), sb = sa + L::kABytes;
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k)
            umma_bf16(tmem_d, smem_desc(sa + k * 32, 16, 1024), B_MN ? smem_desc(sb + k * 2048, 8192, 1024) : smem_desc(sb + k * 32, 16, 1024), idesc,
                      (kb | k) != 0 ? 1u : 0u);
          umma_commit(&empty[stage]);
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (tile == blockIdx.x) asm volatile("griddepcontrol.wait;" ::: "memory");
        SegmentWalk walk(low.segs, __ldcg(low.tile_seg + tm), m0, kBM);
        int adapter, lo, hi;
        while (ok && walk.next(adapter, lo, hi)) {
          uint32_t off[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) off[w] = rows_off(m0 + 32 * w, lo, hi);
          for (int part = 0; part < low.stages; ++part) {
            if (!mbar_wait(&full[stage], phase, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t sa = smem_u32(smem + stage * L::kStageBytes), sb = sa + L::kABytes;
            for (int term = part; term < 2; term += low.stages)
              for (int k = 0; k < low.steps; ++k)
                umma_bf16_rows(tmem_d, smem_desc(sa + (term - part) * low.rp * 2 + k * 32, 16, 1024),
                               B_MN ? smem_desc(sb + k * 2048, 8192, 1024) : smem_desc(sb + k * 32, 16, 1024), idesc, off);
            umma_commit(&empty[stage]);
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
          }
        }
        if (ok) umma_commit(&tfull[acc]);
      }
      if (!ok) {
        *abort_flag = 1;
        atomicCAS(&p.counters->status, 0, PBT_ERR_TIMEOUT);
        p.counters->status_info = 32;
      }
      umma_commit(idle);        // no instruction reads shared memory or writes the accumulators when they are given back
      mbar_wait_out(idle, 0);
    }
  } else {
    const int q = warp & 3, e = warp - 2, half = e >> 2;
    float* buf = reinterpret_cast<float*>(smem + L::kEpiOffset + e * L::kEpiBytesPerWarp);
    int it = 0;
    bool ok = true;
    const bool vec_ok = (((uintptr_t)p.C & 15) == 0) && ((p.ldc * 2) % 16 == 0) && (!p.bias || (((uintptr_t)p.bias & 15) == 0));
    for (int tile = blockIdx.x; tile < p.num_tiles && ok; tile += gridDim.x, ++it) {
      const int m0 = (tile / p.tiles_n) * kBM, n0 = (tile % p.tiles_n) * BN;
      const int acc = it & 1;
      if (!mbar_wait(&tfull[acc], (it >> 1) & 1, abort_flag)) { ok = false; break; }
      tc_fence_after();
      epilogue_tile<BN, EPI>(p, buf, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN), 0, m0, n0, q, half, lane, vec_ok);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&tempty[acc]);
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      atomicCAS(&p.counters->status, 0, PBT_ERR_TIMEOUT);
      p.counters->status_info = 33;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem_base, kTmemCols);
}

template <int BN, int STAGES, int EPI, bool B_MN>
cudaError_t launch_gemm(const CUtensorMap* maps, TcParams& p, const LowRank& low, cudaStream_t s) {
  using L = GemmSmem<BN, STAGES, EPI>;
  static DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = device_setup(&setup, k_adapter_gemm<BN, STAGES, EPI, B_MN>, L::kTotal, &sms);
  if (e != cudaSuccess) return e;
  p.tiles_n = (p.N + BN - 1) / BN;
  p.num_tiles = p.tiles_m * p.tiles_n;
  return launch_after(p.num_tiles < sms ? p.num_tiles : sms, 64 + 32 * EPI, L::kTotal, s, k_adapter_gemm<BN, STAGES, EPI, B_MN>, maps[0], maps[1], maps[2],
                      maps[3], p, low);
}

// C[rows][N] = X[rows][K] B^T + bias + low-rank; B is [N][K], or [K][N] when b_mn; the low-rank matrices alike over ranks.
struct GemmCall {
  const bf16* x; long long ldx;
  const bf16* b; long long ldb; int b_mn;
  const bf16* planes; long long ld_planes; int rp;
  const bf16* mats; int mat_pitch, rank;
  void* c; long long ldc;
  const float* bias;
  int N, K;
};
cudaError_t launch_gemm(const GemmCall& c, const Segments& segs, const int* tile_seg, Counters* counters, cudaStream_t s) {
  TcParams p;
  memset(&p, 0, sizeof(p));
  p.M = segs.rows; p.N = c.N; p.K = c.K; p.batch = 1;
  p.tiles_m = (segs.rows + kBM - 1) / kBM;
  p.k_blocks = (c.K + kBK - 1) / kBK;
  p.C = c.c; p.ldc = c.ldc; p.out_dtype = kBF16;
  p.bias = c.bias;
  p.counters = counters;
  const LowRank low = {segs, tile_seg, c.rp, 2 * c.rp <= kBK ? 1 : 2, c.rp / 16};
  // 128-wide tiles when the 256-wide ones would leave most of their last wave idle; a wave of narrow ones counts 1.35 times half a wave of
  // wide ones (1024 x 1024 -> 1024, one wave of either: 12.4 us, wide 14.5; 6400 rows, three narrow or two wide: 31 and 27; 4096 rows, two or one:
  // 22.7 and 20.5; 4096 x 2048 -> 2048: 56 and 39).
  const long long wide_tiles = (long long)p.tiles_m * ((c.N + 255) / 256), narrow_tiles = (long long)p.tiles_m * ((c.N + 127) / 128);
  const bool wide = 1.35 * (double)((narrow_tiles + 147) / 148) >= 2.0 * (double)((wide_tiles + 147) / 148);
  CUtensorMap maps[4];
  bool ok = make_map(&maps[0], c.x, c.K, segs.rows, c.ldx, 1, 0, kBM) && make_map(&maps[2], c.planes, 2 * c.rp, segs.rows, c.ld_planes, 1, 0, kBM);
  if (!c.b_mn) {
    ok = ok && make_map(&maps[1], c.b, c.K, c.N, c.ldb, 1, 0, wide ? 256 : 128);
    ok = ok && make_map(&maps[3], c.mats, c.mat_pitch, c.N, c.mat_pitch, segs.n_adapters, (long long)c.N * c.mat_pitch, wide ? 256 : 128);
  } else {
    ok = ok && make_map(&maps[1], c.b, c.N, c.K, c.ldb, 1, 0, kBK);
    ok = ok && make_map(&maps[3], c.mats, c.N, c.rank, c.mat_pitch, segs.n_adapters, (long long)c.rank * c.mat_pitch, kBK);
  }
  if (!ok) return cudaErrorInvalidValue;
  const bool one_wave = wide_tiles <= 148;
  auto launch = [&](auto b_mn) {
    if (!wide) return launch_gemm<128, 4, 8, decltype(b_mn)::value>(maps, p, low, s);
    return one_wave ? launch_gemm<256, 3, 8, decltype(b_mn)::value>(maps, p, low, s) : launch_gemm<256, 4, 4, decltype(b_mn)::value>(maps, p, low, s);
  };
  return c.b_mn ? launch(std::true_type()) : launch(std::false_type());
}

// ------------------------------------------------------------------------------------------------------------------
// Few rows
// ------------------------------------------------------------------------------------------------------------------
// Rows of a CTA, and the rows up to which the kernel takes every call: 64 rows of one segment, 2048 -> 2048, rank 16 12.4 us, by the product 18.6;
// 8 rows, 1024 -> 1024 8.3 and 12.4.
constexpr int kRowsMost = 64;
constexpr int kRowsOut = 16;      // output columns of a CTA

struct RowsArgs {
  const bf16* x; long long ldx;
  const bf16* w; long long ldw;
  const bf16* B; int pitch;       // [adapters][N][pitch]
  const float* bias; const float* scaled; const int* row_adapter;
  bf16* y; long long ldy;
  int T, N, K, rank;
};

// y[t][n] for 16 columns n and all rows t: the eight warps take every eighth block of 64 inputs, W's rows are the tall
// operand of mma.sync (16 x 16), eight rows of x the narrow one, in the order of the contraction index that 16-byte loads
// deliver (as in the shrink) and through the same kind of ring: a warp's own, every lane reading back what it copied.  With
// plain loads the kernel waited for one group of rows of x after the other (64 rows, 2048 x 2048: 20 us against 8 us).
// The warps' sums meet in shared memory, where the low-rank part is added in fp32.  Launched while the shrink runs: only that
// last part waits for it.
template <int GROUPS> struct RowsRing {
  static constexpr int kStages = GROUPS == 8 ? 2 : GROUPS == 4 ? 3 : 4;
  static constexpr int kVectors = 4 + 2 * GROUPS;                   // 16-byte vectors of a lane in a block of 64 inputs
  static constexpr int kBytes = kVectors * 512;
  static constexpr int kPitch = GROUPS * 8 + 1;                     // of the sums [8 warps][16 columns][rows]
  static constexpr int kSums = 8 * kRowsOut * kPitch * 4 + GROUPS * 8 * (kMaxRank + 1) * 4;   // and the rows' S and adapters
  static constexpr int kTotal = 8 * kStages * kBytes > kSums ? 8 * kStages * kBytes : kSums;
};
template <int GROUPS>
__global__ void __launch_bounds__(256) k_adapter_rows(const RowsArgs a) {
  extern __shared__ __align__(16) uint8_t rows_smem[];
  typedef RowsRing<GROUPS> Ring;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, tq = lane & 3;
  const int n0 = blockIdx.x * kRowsOut, t0 = blockIdx.y * kRowsMost, T = min(a.T - t0, kRowsMost);
  uint8_t* ring = rows_smem + warp * (Ring::kStages * Ring::kBytes) + lane * 16;
  const bf16* w0 = a.w + (long long)(n0 + gr) * a.ldw;
  const bf16* w1 = w0 + 8 * a.ldw;
  const bf16* x = a.x + (t0 + gr) * a.ldx;
  const bool in0 = n0 + gr < a.N, in1 = n0 + gr + 8 < a.N;
  auto put = [&](uint8_t* slot, const bf16* from, bool in) {
    if (in) copy16(slot, from);
    else *reinterpret_cast<uint4*>(slot) = make_uint4(0u, 0u, 0u, 0u);
  };
  auto ask = [&](int k0, int s) {
    if (k0 < a.K) {
      uint8_t* to = ring + s * Ring::kBytes;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + h * 32 + tq * 8;
        const bool in = k < a.K;
        put(to + h * 512, w0 + k, in && in0);
        put(to + (2 + h) * 512, w1 + k, in && in1);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) put(to + (4 + 2 * g + h) * 512, x + g * 8 * a.ldx + k, in && g * 8 + gr < T);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < Ring::kStages; ++s) ask(warp * 64 + s * 512, s);
  float acc[GROUPS][4] = {};
  int stage = 0;
  for (int k0 = warp * 64; k0 < a.K; k0 += 512) {
    asm volatile("cp.async.wait_group %0;" ::"n"(Ring::kStages - 1) : "memory");
    const uint4* from = reinterpret_cast<const uint4*>(ring + stage * Ring::kBytes);
    uint4 wv[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) { wv[0][h] = from[h * 32]; wv[1][h] = from[(2 + h) * 32]; }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      float sum[4] = {};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 xv = from[(4 + 2 * g + h) * 32];
        mma16816(sum, wv[0][h].x, wv[1][h].x, wv[0][h].y, wv[1][h].y, xv.x, xv.y);
        mma16816(sum, wv[0][h].z, wv[1][h].z, wv[0][h].w, wv[1][h].w, xv.z, xv.w);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[g][e] += sum[e];
    }
    ask(k0 + Ring::kStages * 512, stage);
    if (++stage == Ring::kStages) stage = 0;
  }
  __syncthreads();     // the rings' memory becomes the warps' sums
  float* red = reinterpret_cast<float*>(rows_smem);
#pragma unroll
  for (int g = 0; g < GROUPS; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[(warp * kRowsOut + gr + 8 * (e >> 1)) * Ring::kPitch + g * 8 + tq * 2 + (e & 1)] = acc[g][e];
  float* low = red + 8 * kRowsOut * Ring::kPitch;          // scaled S of the rows
  int* owner = reinterpret_cast<int*>(low + GROUPS * 8 * kMaxRank);
  asm volatile("griddepcontrol.wait;" ::: "memory");     // the shrink is complete and its results are visible
  for (int i = threadIdx.x; i < T * a.rank; i += 256) low[(i / a.rank) * a.pitch + i % a.rank] = __ldcg(a.scaled + (long long)t0 * a.rank + i);
  if (threadIdx.x < T) owner[threadIdx.x] = __ldcg(a.row_adapter + t0 + threadIdx.x);
  __syncthreads();
  // a thread has one column and every 16th row, whose adapters' matrices it asks for together
  const int n = threadIdx.x % kRowsOut, col = n0 + n;
  if (col >= a.N) return;
  const float bias = a.bias ? __ldg(a.bias + col) : 0.f;
  constexpr int kMine = (GROUPS * 8 + 15) / 16;
  float v[kMine];
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    const int t = threadIdx.x / kRowsOut + 16 * u;
    v[u] = bias;
    if (t < T)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[u] += red[(k * kRowsOut + n) * Ring::kPitch + t];
  }
  for (int j = 0; j < a.rank; j += 8) {
    uint4 bv[kMine];
#pragma unroll
    for (int u = 0; u < kMine; ++u) {
      const int t = threadIdx.x / kRowsOut + 16 * u, adapter = t < T ? owner[t] : -1;
      bv[u] = adapter >= 0 ? __ldg(reinterpret_cast<const uint4*>(a.B + ((long long)adapter * a.N + col) * a.pitch + j)) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < kMine; ++u) {
      const int t = threadIdx.x / kRowsOut + 16 * u;
      if (t < T && owner[t] >= 0)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t pairs = word(bv[u], e >> 1);
          if (j + e < a.rank) v[u] = __fmaf_rn(__uint_as_float((e & 1) ? pairs & 0xFFFF0000u : pairs << 16), low[t * a.pitch + j + e], v[u]);
        }
    }
  }
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    const int t = threadIdx.x / kRowsOut + 16 * u;
    if (t < T) a.y[(t0 + t) * a.ldy + col] = __float2bfloat16_rn(v[u]);
  }
}

template <int GROUPS>
cudaError_t launch_rows(const RowsArgs& a, cudaStream_t s) {
  static DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = device_setup(&setup, k_adapter_rows<GROUPS>, RowsRing<GROUPS>::kTotal, &sms);
  if (e != cudaSuccess) return e;
  return launch_after(dim3((a.N + kRowsOut - 1) / kRowsOut, (a.T + kRowsMost - 1) / kRowsMost), 256, RowsRing<GROUPS>::kTotal, s, k_adapter_rows<GROUPS>, a);
}
cudaError_t launch_rows(const RowsArgs& a, cudaStream_t s) {
  if (a.T <= 8) return launch_rows<1>(a, s);
  if (a.T <= 16) return launch_rows<2>(a, s);
  if (a.T <= 32) return launch_rows<4>(a, s);
  return launch_rows<8>(a, s);
}

// ------------------------------------------------------------------------------------------------------------------
// Gradients of the adapters
// ------------------------------------------------------------------------------------------------------------------
constexpr int kGradStages = 4, kGradChunk = 512, kGradList = 1024;

struct GradArgs {
  Segments segs;
  int rank;
  int K, N, blocks_k, blocks_n;        // column blocks of dA come first, those of dB after them
  int splits;
  float *dA, *dB;                      // [splits][adapters][...]: the results themselves when splits == 1
  long long stride_a, stride_b;        // elements of one split
  uint32_t tmem_cols;
  Counters* counters;
};

// a bounded wait of a whole warp: every lane gives up if one does
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag));
}

// Work items are (adapter, split, column block): an adapter's gradient in 128 columns, over all its rows or, when there are
// splits, over every splits-th chunk of 512 of them.  A CTA takes an equal share of consecutive items.  128 columns of v (x for dA, dy for dB) are the accumulator's lanes, its columns the three summands of the
// r ranks.  Both operands are read as they lie (rows = contraction index: MN-major).  Where a block of 64 rows ends
// inside a box, the rows behind the end (another member's) are cleared in shared memory in both operands before the MMA
// reads them.  The producer runs ahead into the next column block while the last one is drained, so that two CTAs per SM
// keep 4 x 24 KB each on their way throughout (with a CTA per column block, 136 us at 80 members x 512 rows x 2048: the
// pipeline filled and drained 2560 times).
template <int RP>
__global__ void __launch_bounds__(192, 2) k_adapter_grad(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmDS,
                                                      const __grid_constant__ CUtensorMap tmDY, const __grid_constant__ CUtensorMap tmS, const GradArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  constexpr int kBoxes = (3 * RP + 63) / 64, stage_bytes = 16384 + kBoxes * 8192;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + kGradStages * stage_bytes);
  uint64_t* empty = full + kGradStages;
  uint64_t* tfull = empty + kGradStages;
  uint64_t* tempty = tfull + 2;
  uint64_t* idle = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(idle + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int2* list = reinterpret_cast<int2*>(idle + 2);
  __shared__ int list_n;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kGradStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&tfull[i], 1); mbar_init(&tempty[i], 4); }
    mbar_init(idle, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(tmem_slot, a.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  uint32_t stage = 0, phase = 0;   // producer, MMA warp
  int folds = 0;                   // MMA warp, epilogue: accumulators handed over so far
  bool ok = true;
  const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)((3 * RP) >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);

  const int columns = a.blocks_k + a.blocks_n;
  const long long items = (long long)a.segs.n_adapters * a.splits * columns;
  const long long item_end = items * (blockIdx.x + 1) / gridDim.x;
  for (long long item = items * blockIdx.x / gridDim.x; item < item_end;) {
    const int owner = (int)(item / columns), adapter = owner / a.splits, z = owner % a.splits;
    const int first = (int)(item % columns), last = (int)min((long long)columns, first + item_end - item);   // columns of this adapter and split
    item += last - first;
    // The adapter's segments, kGradList table entries at a time, as a list of row ranges in shared memory.  One pass does for
    // up to 1024 segments; later passes add to what the earlier ones left in dA and dB.
    for (int base = 0; base == 0 || base < a.segs.n; base += kGradList) {
      __syncthreads();
      if (warp == 0) {
        int n = 0;
        for (int i0 = base; i0 < min(a.segs.n, base + kGradList); i0 += 32) {   // (kGradList is a multiple of 32)
          const int i = i0 + lane;
          const bool have = i < a.segs.n && segment_adapter(a.segs, i) == adapter;
          const int2 r = have ? make_int2(segment_begin(a.segs, i), segment_begin(a.segs, i + 1)) : make_int2(0, 0);
          const bool keep = have && r.x < r.y;
          const uint32_t votes = __ballot_sync(0xFFFFFFFFu, keep);
          if (keep) list[n + __popc(votes & ((1u << lane) - 1u))] = r;
          n += __popc(votes);
        }
        if (lane == 0) list_n = n;
      }
      __syncthreads();
      const int n = list_n;
      int blocks = 0;   // blocks of 64 rows in this list that belong to this split
      for (int i = 0; i < n; ++i)
        for (int t = list[i].x / kGradChunk; t * kGradChunk < list[i].y; ++t)
          if (t % a.splits == z) blocks += (min(list[i].y, (t + 1) * kGradChunk) - max(list[i].x, t * kGradChunk) + 63) / 64;
      if (base > 0 && !blocks) continue;

      for (int column = first; column < last && ok; ++column) {
        const bool is_b = column >= a.blocks_k;
        const int c0 = (column - (is_b ? a.blocks_k : 0)) * 128;
        if (warp == 0) {
          if (lane == 0) {
            const CUtensorMap* tmV = is_b ? &tmDY : &tmX;
            const CUtensorMap* tmT = is_b ? &tmS : &tmDS;
            for (int i = 0; i < n && ok; ++i)
              for (int t = list[i].x / kGradChunk; t * kGradChunk < list[i].y && ok; ++t) {
                if (t % a.splits != z) continue;
                const int end = min(list[i].y, (t + 1) * kGradChunk);
                for (int row = max(list[i].x, t * kGradChunk); row < end; row += 64) {
                  if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) { ok = false; break; }
                  uint8_t* sv = smem + stage * stage_bytes;
                  mbar_expect_tx(&full[stage], stage_bytes);
                  tma_load_3d(sv, tmV, &full[stage], c0, row, 0);
                  tma_load_3d(sv + 8192, tmV, &full[stage], c0 + 64, row, 0);
                  for (int b = 0; b < kBoxes; ++b) tma_load_3d(sv + 16384 + b * 8192, tmT, &full[stage], b * 64, row, 0);
                  if (++stage == kGradStages) { stage = 0; phase ^= 1; }
                }
              }
          }
          ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
        } else if (warp == 1) {
          int done = 0;
          for (int i = 0; i < n && ok; ++i)
            for (int t = list[i].x / kGradChunk; t * kGradChunk < list[i].y && ok; ++t) {
              if (t % a.splits != z) continue;
              const int end = min(list[i].y, (t + 1) * kGradChunk);
              for (int row = max(list[i].x, t * kGradChunk); row < end; row += 64, ++done) {
                const int acc_buf = folds & 1;
                if ((done & 1) == 0) {
                  if (!warp_wait(&tempty[acc_buf], ((folds >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
                }
                if (!warp_wait(&full[stage], phase, abort_flag)) { ok = false; break; }
                uint8_t* sv = smem + stage * stage_bytes;
                const int valid = end - row;
                if (valid < 64) {   // rows are 128-byte lines of each box
                  for (int b = 0; b < 2 + kBoxes; ++b)
                    for (int o = valid * 8 + lane; o < 64 * 8; o += 32) reinterpret_cast<uint4*>(sv + b * 8192)[o] = make_uint4(0u, 0u, 0u, 0u);
                  fence_async_smem();
                  __syncwarp();
                }
                if (lane == 0) {
                  tc_fence_after();
                  const uint32_t sa = smem_u32(sv), sb = sa + 16384;
                  const uint32_t tmem_d = tmem_base + (uint32_t)(acc_buf * (3 * RP));
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    umma_bf16(tmem_d, smem_desc(sa + k * 2048, 8192, 1024), smem_desc(sb + k * 2048, 8192, 1024), idesc, ((done & 1) | k) != 0 ? 1u : 0u);
                  umma_commit(&empty[stage]);
                  if ((done & 1) == 1 || done + 1 == blocks) umma_commit(&tfull[acc_buf]);
                }
                __syncwarp();
                if ((done & 1) == 1 || done + 1 == blocks) ++folds;
                if (++stage == kGradStages) { stage = 0; phase ^= 1; }
              }
            }
        } else {
          const int q = warp & 3;
          float acc[RP];
#pragma unroll
          for (int i = 0; i < RP; ++i) acc[i] = 0.f;
          for (int f = 0; f < (blocks + 1) / 2 && ok; ++f, ++folds) {
            const int acc_buf = folds & 1;
            if (!warp_wait(&tfull[acc_buf], (folds >> 1) & 1, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t t0 = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc_buf * (3 * RP));
#pragma unroll
            for (int c = 0; c < RP; c += 16) {
              uint32_t h[16], m[16], l[16];
              tmem_ld16(t0 + c, h);
              tmem_ld16(t0 + RP + c, m);
              tmem_ld16(t0 + 2 * RP + c, l);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) acc[c + i] += __uint_as_float(h[i]) + (__uint_as_float(m[i]) + __uint_as_float(l[i]));
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&tempty[acc_buf]);
          }
          const int col = c0 + q * 32 + lane;
          if (ok && col < (is_b ? a.N : a.K)) {
            // dA [rank][K]: a warp's lanes are neighbours; dB [N][rank]: a lane's ranks are
            float* o = is_b ? a.dB + z * a.stride_b + ((long long)adapter * a.N + col) * a.rank
                            : a.dA + z * a.stride_a + (long long)adapter * a.rank * a.K + col;
            const long long step = is_b ? 1 : a.K;
#pragma unroll
            for (int i = 0; i < RP; ++i)
              if (i < a.rank) o[i * step] = base > 0 ? o[i * step] + acc[i] : acc[i];
          }
        }
      }
    }
  }
  if (!ok && lane == 0) {
    *abort_flag = 1;
    atomicCAS(&a.counters->status, 0, PBT_ERR_TIMEOUT);
    a.counters->status_info = 40 + min(warp, 2);
  }
  // as in k_adapter_gemm: what was asked for has landed, the last commits into `empty` too unless a wait ran out, and the tensor cores are idle
  if (warp == 0 && lane == 0) {
    for (int s = 0; s < kGradStages; ++s) mbar_wait_out(&full[s], s < (int)stage ? phase : phase ^ 1);
    for (int s = 0; s < kGradStages && ok; ++s) {
      if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) break;
      if (++stage == kGradStages) { stage = 0; phase ^= 1; }
    }
  } else if (warp == 1 && lane == 0) {
    umma_commit(idle);
    mbar_wait_out(idle, 0);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem_base, a.tmem_cols);
  asm volatile("griddepcontrol.wait;" ::: "memory");     // what follows in the stream follows the product, too
}

template <int RP>
cudaError_t launch_grad(const CUtensorMap& x, const CUtensorMap& ds, const CUtensorMap& dy, const CUtensorMap& kept, const GradArgs& g, cudaStream_t st) {
  constexpr int kSmem = kGradStages * (16384 + (3 * RP + 63) / 64 * 8192) + 256 + kGradList * 8 + 1024;
  static_assert(kSmem <= 232448, "shared memory budget of one CTA");
  static DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = device_setup(&setup, k_adapter_grad<RP>, kSmem, &sms);
  if (e != cudaSuccess) return e;
  const long long items = (long long)g.segs.n_adapters * g.splits * (g.blocks_k + g.blocks_n);
  const int resident = (RP == 16 ? 2 : 1) * sms;      // two CTAs per SM where shared memory allows it
  return launch_after((unsigned)std::min<long long>(resident, items), 192, kSmem, st, k_adapter_grad<RP>, x, ds, dy, kept, g);
}

// out = the splits' partial results, added in order
__global__ void __launch_bounds__(256) k_adapter_grad_join(const float* __restrict__ pa, const float* __restrict__ pb, long long na, long long nb, int splits,
                                                           float* __restrict__ dA, float* __restrict__ dB) {
  pdl_prologue();
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < na + nb; i += (long long)gridDim.x * 256) {
    const bool is_b = i >= na;
    const float* p = is_b ? pb + (i - na) : pa + i;
    const long long stride = is_b ? nb : na;
    float t = 0.f;
    for (int z = 0; z < splits; ++z) t += p[z * stride];
    (is_b ? dB[i - na] : dA[i]) = t;
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------------------------------
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
int round_up(int n, int m) { return (n + m - 1) / m * m; }
bool aligned(const void* p, long long ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

struct Plan {
  int rp, splits;
  bool few;      // rows that k_adapter_rows takes
  bool pack_x, pack_w, pack_a, pack_b, pack_dy;
  size_t x, w, a, b, dy, planes, kept, table, parts, total;
};
Plan plan(const pbt_adapter_desc* d, bool backward) {
  Plan p;
  memset(&p, 0, sizeof(p));
  const size_t rows = (size_t)d->rows;
  p.rp = round_up(d->rank, 16);
  p.pack_x = !aligned(d->x, d->ld_x) || d->inputs % 8;     // (vector loads end with the row)
  // Few rows, or many short segments: the product has a low-rank block for every segment of a 128-row tile (12 us and 0.5 for each), k_adapter_rows
  // a wave of CTAs for every 148 of its 64 rows x 16 columns (6 us and 8.5 for each, less below 1024 inputs).  1024 -> 1024, rank 16: 128 single rows 12 us,
  // as a product 80; 64 segments of four rows 18 and 30; 2048 -> 2048, 80 segments of four rows 49 and 35;
  // 512 -> 512, rank 8 the same 12 and 27.  (Beyond rank 32 both take about twice that.)
  const long long waves = ((long long)((d->rows + kRowsMost - 1) / kRowsMost) * ((d->outputs + kRowsOut - 1) / kRowsOut) + 147) / 148;
  const int tile_segments = std::min(kBM, d->n_segments / ((d->rows + kBM - 1) / kBM + (d->rows == 0)));
  p.few = !backward && (d->rows <= kRowsMost || std::min(21, 1 + d->inputs / 48) * waves < 15 + tile_segments * 4 / 3);
  p.pack_w = !aligned(d->weight, d->ld_weight) || (p.few && d->inputs % 8);
  p.pack_a = !aligned(d->A, d->inputs);
  p.pack_b = !aligned(d->B, d->rank);
  p.pack_dy = backward && (!aligned(d->dy, d->ld_dy) || d->outputs % 8);
  // Splits of the adapters' rows in the gradients: enough CTAs for two per SM, at most one for every chunk of an adapter's share of the rows
  // (a training step of 4096 x 1024 -> 1024 with one adapter: 53 us, without splits 76; 2048 x 512 -> 512 with sixteen: 36 with three, 31 without).
  const long long blocks = ((d->inputs + 127ll) / 128 + (d->outputs + 127ll) / 128) * d->n_adapters, chunk = (long long)d->n_adapters * kGradChunk;
  p.splits = (int)std::max(1ll, std::min((2 * 148 + blocks - 1) / blocks, (d->rows + chunk - 1) / chunk));
  size_t at = 0;
  auto take = [&](bool want, size_t bytes) {
    const size_t here = at;
    if (want) at += align256(bytes);
    return here;
  };
  p.x = take(p.pack_x, rows * round_up(d->inputs, 8) * 2);
  p.w = take(p.pack_w, (size_t)d->outputs * round_up(d->inputs, 8) * 2);
  p.a = take(p.pack_a, (size_t)d->n_adapters * d->rank * round_up(d->inputs, 8) * 2);
  p.b = take(p.pack_b, (size_t)d->n_adapters * d->outputs * round_up(d->rank, 8) * 2);
  p.dy = take(p.pack_dy, rows * round_up(d->outputs, 8) * 2);
  p.planes = take(true, p.few ? rows * d->rank * sizeof(float) : rows * p.rp * 2 * (backward ? 3 : 2));
  p.kept = take(backward, rows * p.rp * 2 * 3);
  p.table = take(true, (p.few ? rows : (rows + kBM - 1) / kBM) * sizeof(int));
  p.parts = take(backward && p.splits > 1, (size_t)p.splits * d->n_adapters * d->rank * ((size_t)d->inputs + d->outputs) * sizeof(float));
  p.total = std::max<size_t>(at, 256);
  return p;
}

// collects an operand to pack, and stands for the packed one from then on
struct Packer {
  PackJobs jobs;
  unsigned blocks;
  Packer() : blocks(0) { jobs.n = 0; }
  void add(bool want, const void*& src, long long& ld, long long rows, int cols, char* dst) {
    if (!want) return;
    const int to = round_up(cols, 8);
    jobs.job[jobs.n++] = {(const bf16*)src, ld, (bf16*)dst, rows, cols, to, blocks};
    blocks += (unsigned)((rows * (to / 8) + 255) / 256);
    src = dst;
    ld = to;
  }
  cudaError_t run(cudaStream_t s) const { return blocks ? launch_with(blocks, 256, 0, s)(k_pack_rows, jobs) : cudaSuccess; }
};

}  // namespace

cudaError_t join_gradients(const float* parts_a, const float* parts_b, long long size_a, long long size_b, int splits, float* dA, float* dB, cudaStream_t s) {
  const long long n = size_a + size_b;
  return launch_with((unsigned)std::min<long long>((n + 255) / 256, 148 * 16), 256, 0, s)(k_adapter_grad_join, parts_a, parts_b, size_a, size_b, splits, dA, dB);
}

size_t tc_workspace(const pbt_adapter_desc* d, bool backward) { return plan(d, backward).total; }

#define STEP(call) do { const cudaError_t e_ = (call); if (e_ != cudaSuccess) return e_; } while (0)

cudaError_t tc_forward(const pbt_adapter_desc* d, const Segments& segs, char* ws, cudaStream_t st) {
  const Plan p = plan(d, false);
  const void *x = d->x, *w = d->weight, *A = d->A, *B = d->B;
  long long ldx = d->ld_x, ldw = d->ld_weight, lda = d->inputs, ldb = d->rank;
  Packer pk;
  pk.add(p.pack_x, x, ldx, d->rows, d->inputs, ws + p.x);
  pk.add(p.pack_w, w, ldw, d->outputs, d->inputs, ws + p.w);
  pk.add(p.pack_a, A, lda, (long long)d->n_adapters * d->rank, d->inputs, ws + p.a);
  pk.add(p.pack_b, B, ldb, (long long)d->n_adapters * d->outputs, d->rank, ws + p.b);
  STEP(pk.run(st));
  ShrinkArgs a;
  memset(&a, 0, sizeof(a));
  a.x = (const bf16*)x; a.ldx = ldx; a.K = d->inputs;
  a.mats = (const bf16*)A; a.pitch = (int)lda; a.rank = d->rank; a.rp = p.rp;
  a.scale = d->scale; a.segs = segs;
  a.s = d->s;
  if (p.few) {
    a.scaled = (float*)(ws + p.planes);
    a.row_adapter = (int*)(ws + p.table); a.tile_rows = 1; a.n_table = d->rows;
    STEP(launch_shrink<false>(a, st));
    const RowsArgs r = {(const bf16*)x, ldx, (const bf16*)w, ldw, (const bf16*)B, (int)ldb, d->bias, a.scaled, a.row_adapter, (bf16*)d->y, d->ld_y,
                        d->rows, d->outputs, d->inputs, d->rank};
    return launch_rows(r, st);
  }
  a.planes = (bf16*)(ws + p.planes); a.terms = 2;
  a.tile_seg = (int*)(ws + p.table); a.tile_rows = kBM; a.n_table = (d->rows + kBM - 1) / kBM;
  STEP(launch_shrink<false>(a, st));
  const GemmCall c = {(const bf16*)x, ldx, (const bf16*)w, ldw, 0, a.planes, 2 * p.rp, p.rp, (const bf16*)B, (int)ldb, d->rank, d->y, d->ld_y, d->bias, d->outputs, d->inputs};
  return launch_gemm(c, segs, a.tile_seg, (Counters*)d->status_device, st);
}

cudaError_t tc_backward(const pbt_adapter_desc* d, const Segments& segs, char* ws, cudaStream_t st) {
  const Plan p = plan(d, true);
  const void *x = d->x, *w = d->weight, *A = d->A, *B = d->B, *dy = d->dy;
  long long ldx = d->ld_x, ldw = d->ld_weight, lda = d->inputs, ldb = d->rank, lddy = d->ld_dy;
  Packer pk;
  pk.add(p.pack_x, x, ldx, d->rows, d->inputs, ws + p.x);
  pk.add(p.pack_w, w, ldw, d->outputs, d->inputs, ws + p.w);
  pk.add(p.pack_a, A, lda, (long long)d->n_adapters * d->rank, d->inputs, ws + p.a);
  pk.add(p.pack_b, B, ldb, (long long)d->n_adapters * d->outputs, d->rank, ws + p.b);
  pk.add(p.pack_dy, dy, lddy, d->rows, d->outputs, ws + p.dy);
  STEP(pk.run(st));
  const int width = 3 * p.rp;
  ShrinkArgs a;
  memset(&a, 0, sizeof(a));
  a.x = (const bf16*)dy; a.ldx = lddy; a.K = d->outputs;
  a.mats = (const bf16*)B; a.pitch = (int)ldb; a.rank = d->rank; a.rp = p.rp;
  a.scale = d->scale; a.segs = segs;
  a.planes = (bf16*)(ws + p.planes); a.terms = 3;
  a.kept = d->s; a.kept_planes = (bf16*)(ws + p.kept);
  a.tile_seg = (int*)(ws + p.table); a.tile_rows = kBM; a.n_table = (d->rows + kBM - 1) / kBM;
  STEP(launch_shrink<true>(a, st));
  const GemmCall c = {(const bf16*)dy, lddy, (const bf16*)w, ldw, 1, a.planes, width, p.rp, (const bf16*)A, (int)lda, d->rank, d->dx, d->ld_dx, nullptr, d->inputs, d->outputs};
  STEP(launch_gemm(c, segs, a.tile_seg, (Counters*)d->status_device, st));

  GradArgs g;
  memset(&g, 0, sizeof(g));
  g.segs = segs; g.rank = d->rank;
  g.K = d->inputs; g.N = d->outputs; g.blocks_k = (d->inputs + 127) / 128; g.blocks_n = (d->outputs + 127) / 128;
  g.splits = p.splits;
  g.stride_a = (long long)d->n_adapters * d->rank * d->inputs;
  g.stride_b = (long long)d->n_adapters * d->rank * d->outputs;
  g.dA = p.splits > 1 ? (float*)(ws + p.parts) : d->dA;
  g.dB = p.splits > 1 ? g.dA + p.splits * g.stride_a : d->dB;
  g.tmem_cols = 32;
  while (g.tmem_cols < (uint32_t)(2 * width)) g.tmem_cols *= 2;
  g.counters = (Counters*)d->status_device;
  CUtensorMap mx, mds, mdy, ms;
  if (!make_map(&mx, x, d->inputs, d->rows, ldx, 1, 0, 64) || !make_map(&mdy, dy, d->outputs, d->rows, lddy, 1, 0, 64) ||
      !make_map(&mds, a.planes, width, d->rows, width, 1, 0, 64) || !make_map(&ms, a.kept_planes, width, d->rows, width, 1, 0, 64))
    return cudaErrorInvalidValue;
  const cudaError_t launched = p.rp == 16 ? launch_grad<16>(mx, mds, mdy, ms, g, st) : p.rp == 32 ? launch_grad<32>(mx, mds, mdy, ms, g, st)
                             : p.rp == 48 ? launch_grad<48>(mx, mds, mdy, ms, g, st) : launch_grad<64>(mx, mds, mdy, ms, g, st);
  STEP(launched);
  if (p.splits > 1) {
    STEP(join_gradients(g.dA, g.dB, g.stride_a, g.stride_b, p.splits, d->dA, d->dB, st));
  }
  return cudaSuccess;
}

}  // namespace adapters
}  // namespace pbt
