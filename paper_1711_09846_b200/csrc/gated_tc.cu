// bf16 gated units on the tensor cores: both projections, the activation, the product and dropout in one kernel.
//
//   k_gated_tc_pair / k_gated_tc   tiles of 256 (128) rows and 128 (64) hidden units: the B operand of one tcgen05 product is the gate's weight
//                                  rows and the up-projection's for the same hidden units, so that g and u of a hidden unit meet in one TMEM lane
//   k_gated_rows                   a few rows (single tokens): bound by reading the weight once, which is the tall operand there; clusters of CTAs
//                                  share a contraction
//
// h is rounded once, from fp32 g and u.
#include <algorithm>
#include <type_traits>

#include "gated.cuh"
#include "tc_epilogue.cuh"

namespace pbt {
namespace gated {
namespace {

using namespace tc;
using dropout::Divisor;
using dropout::divisor;
using dropout::Eight;
using dropout::quotient;
using dropout::store8;

// ------------------------------------------------------------------------------------------------------------------
// Tiles
// ------------------------------------------------------------------------------------------------------------------
constexpr int kEpiW = 8;                      // epilogue warps of a CTA: two for each quarter of the TMEM lanes
constexpr int kTcThreads = 64 + 32 * kEpiW;
constexpr int kBoxBytes = 4096;               // a staging box: 32 rows of 32 fp32 values, or of 32 bf16 ones (half of it)

struct TileParams {
  int rows, hidden, tiles_m, tiles_n, num_tiles, k_blocks;
  int x_batched, w_batched;
  int activation, drop, h_tma;
  bf16* h;                                     // or null: only g and u
  int want_z;
  dropout::Rule rule;
  Counters* counters;
};
struct TileMaps {
  CUtensorMap x, w, h, g, u;
};

// HN: hidden units of a tile.  A pair of CTAs shares a tile of 256 rows: each loads 128 rows of x, the first the gate's rows of the weight
// and the second the up-projection's, and each has the accumulator of its own 128 rows.  Alone, a CTA loads both.
template <bool PAIR, int HN, int STAGES>
struct Tile {
  static constexpr int kRows = PAIR ? 256 : 128;
  static constexpr int kABytes = kBM * kBK * 2, kBBytes = (PAIR ? HN : 2 * HN) * kBK * 2, kStage = kABytes + kBBytes;
  static constexpr int kEpi = STAGES * kStage;
  static constexpr int kBars = kEpi + kEpiW * 2 * kBoxBytes;
  static constexpr int kTotal = kBars + 256 + 1024;
  static_assert(kTotal <= 232448 && kEpi % 1024 == 0, "shared memory of one CTA; staging boxes are 1024-byte aligned");
  static constexpr uint32_t kCols = 4 * HN;    // two accumulators of g and u
};

// brings a tensor map into the cache of descriptors, ahead of the first load
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// a bounded wait of a whole warp: every lane gives up if one does
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag));
}

// h of 32 hidden units of a row, in the place of u
template <int KIND>
__device__ __forceinline__ void apply(const uint32_t* g, uint32_t* u) {
#pragma unroll
  for (int c = 0; c < 32; ++c) u[c] = __float_as_uint(activation_bf16(KIND, __uint_as_float(g[c])) * __uint_as_float(u[c]));
}
__device__ __forceinline__ void apply(int kind, const uint32_t* g, uint32_t* u) {
  switch (kind) {
    case kSilu: apply<kSilu>(g, u); break;
    case kGelu: apply<kGelu>(g, u); break;
    case kRelu: apply<kRelu>(g, u); break;
    default: apply<kSigmoid>(g, u);
  }
}

// One warp's part of a tile: 32 rows (a lane has one) and HN / 2 hidden units, in chunks of 32.  g and u leave as they are (want_z), h after
// the activation and dropout, each through a staging box of the warp's (two, used in turn) and a bulk store that the tensor map clips at the
// last row and hidden unit.  Rows of h that are no multiples of 16 bytes go from the box by ordinary stores, 32 hidden units of a row at a time.
template <int HN>
__device__ __forceinline__ void drain(const TileParams& p, const TileMaps& maps, uint8_t* stage, uint32_t tacc, int member, int row0, int n0, int half,
                                      int lane, const dropout::Draw& d, uint32_t handback, bool pair, uint64_t* tempty, uint32_t& boxes) {
  constexpr int kChunks = HN / 64;
  const int row = row0 + lane;
  const uint32_t groups = (uint32_t)(p.hidden + dropout::kGroup - 1) / dropout::kGroup;
  auto box = [&]() {
    if (lane == 0) tma_store_wait_read_but_one();
    __syncwarp();
    return stage + (boxes++ & 1u) * kBoxBytes;
  };
  auto send = [&](const CUtensorMap* map, const uint8_t* from, int c) {
    fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_3d(map, from, c, row0, member);
      tma_store_commit();
    }
  };
#pragma unroll 1
  for (int q = 0; q < kChunks; ++q) {
    const int c0 = (half * kChunks + q) * 32, col = n0 + c0;
    uint32_t g[32], u[32];
    tmem_ld32(tacc + c0, g);
    tmem_ld32(tacc + HN + c0, u);
    tmem_ld_wait();
    if (q + 1 == kChunks) {                     // the accumulator is empty
      if (pair) release_accumulator(handback, lane);
      else {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty);
      }
    }
    if (row0 >= p.rows || col >= p.hidden) continue;      // (uniform in the warp)
    if (p.want_z) {
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        uint8_t* to = box();
        const uint32_t* v = side ? u : g;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *reinterpret_cast<uint4*>(to + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        send(side ? &maps.u : &maps.g, to, col);
      }
    }
    if (!p.h) continue;
    apply(p.activation, g, u);
    if (d.on) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const U4 w = dropout::draw_group(p.rule, d, (uint32_t)row * groups + (uint32_t)(col / dropout::kGroup + j));
#pragma unroll
        for (int c = 0; c < 8; ++c) u[8 * j + c] = dropout::kept(w, c, d.limit) ? __float_as_uint(__uint_as_float(u[8 * j + c]) * d.scale) : 0u;
      }
    }
    uint32_t o[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(__uint_as_float(u[2 * c]), __uint_as_float(u[2 * c + 1]));
      o[c] = *reinterpret_cast<const uint32_t*>(&t);
    }
    uint8_t* to = box();
    // (64-byte swizzle: conflict-free 16-byte stores)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint4*>(to + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
    if (p.h_tma) {
      send(&maps.h, to, col);
    } else {
      --boxes;                                   // no bulk store reads this box: it is the next one, too
      __syncwarp();
      bf16* out = p.h + ((long long)member * p.rows + row0) * p.hidden + col + lane;
      const int rows = min(32, p.rows - row0);
      if (col + lane < p.hidden)
        for (int r = 0; r < rows; ++r)
          out[(long long)r * p.hidden] = *reinterpret_cast<const bf16*>(to + r * 64 + (((lane >> 3) ^ ((r >> 1) & 3)) << 4) + (lane & 7) * 2);
      __syncwarp();
    }
  }
}

// A pair in which a wait ran out: the leader's barriers count what both CTAs load, and one of the two may be up to a ring of loads ahead.  Of these,
// the leader's were announced for both, and the partner's part never comes; the partner's are under way and were not announced.  With both put right, every
// load's phase ends when its copies have landed.  (The counts are far from wrapping: 2^32 loads are 140 TB through one pair.)
template <int STAGES, int BYTES>
__device__ __forceinline__ void settle(uint64_t* full, uint32_t leader, uint32_t partner) {
  const uint32_t less = min(leader, partner), more = max(leader, partner);
  for (uint32_t i = less; i < more; ++i) {
    if (i >= partner) mbar_complete_tx(&full[i % STAGES], BYTES);
    else mbar_expect_tx(&full[i % STAGES], BYTES);
  }
  for (uint32_t i = more - min(more, (uint32_t)STAGES); i < more; ++i) mbar_wait_out(&full[i % STAGES], i / STAGES & 1);
}

template <bool PAIR, int HN, int STAGES>
__device__ __forceinline__ void gated_tiles(const TileMaps& maps, const TileParams& p) {
  pdl_prologue();
  typedef Tile<PAIR, HN, STAGES> L;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);       // of a pair: used in the leader only
  uint64_t* empty = full + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint64_t* tempty = tfull + 2;                                          // of a pair: used in the leader only
  uint64_t* idle = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(idle + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile uint32_t* told = tmem_slot + 2;                               // of a pair: the partner's loads, and whether it gave up
  uint32_t issued = 0;                                                   // loads of this CTA (thread 0)

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0;
  const int first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;
  if (threadIdx.x == 64) { prefetch_map(&maps.x); prefetch_map(&maps.w); }
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(&tfull[a], 1); mbar_init(&tempty[a], (PAIR ? 2 : 1) * kEpiW); }
    mbar_init(idle, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) tmem_alloc_pair(tmem_slot, L::kCols);
    else tmem_alloc(tmem_slot, L::kCols);
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();   // both CTAs' barriers exist before anyone signals across the pair
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int per_member = p.tiles_m * p.tiles_n;
  auto give_up = [&](int where) {
    *abort_flag = 1;
    atomicCAS(&p.counters->status, 0, PBT_ERR_TIMEOUT);
    p.counters->status_info = where;
  };

  if (warp == 0) {
    // ------------------------------ TMA producer ------------------------------
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      for (int tile = first; tile < p.num_tiles && ok; tile += step) {
        const int member = tile / per_member, rem = tile % per_member;
        const int m0 = (rem / p.tiles_n) * L::kRows + (int)rank * kBM, n0 = (rem % p.tiles_n) * HN;
        const int cx = p.x_batched ? member : 0, cw = p.w_batched ? member : 0;
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) { ok = false; break; }
          uint8_t *sa = smem + stage * L::kStage, *sb = sa + L::kABytes;
          const int k0 = kb * kBK;
          if (PAIR) {
            // the leader announces the bytes of both CTAs (its partner cannot run a phase ahead: its stage is handed back by the
            // leader's commit for the previous phase)
            const uint32_t lbar = map_to_cta(smem_u32(&full[stage]), 0);
            if (rank == 0) mbar_expect_tx(&full[stage], 2 * L::kStage);
            tma_load_3d_pair(sa, &maps.x, lbar, k0, m0, cx);
            tma_load_3d_pair(sb, &maps.w, lbar, k0, (int)rank * p.hidden + n0, cw);
          } else {
            mbar_expect_tx(&full[stage], L::kStage);
            tma_load_3d(sa, &maps.x, &full[stage], k0, m0, cx);
            tma_load_3d(sb, &maps.w, &full[stage], k0, n0, cw);
            tma_load_3d(sb + HN * kBK * 2, &maps.w, &full[stage], k0, p.hidden + n0, cw);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
          ++issued;
        }
      }
      if (!ok) give_up(31);
      // every stage that was armed has landed before the CTA ends (of a pair: below, if a wait ran out; else the products have read them)
      for (int s = 0; s < STAGES && !PAIR; ++s) mbar_wait_out(&full[s], s < (int)stage ? phase : phase ^ 1);
      for (int s = 0; s < STAGES && ok; ++s) {
        if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) break;
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------ MMA issuer (of a pair: the leader's) ------------------------------
    if (lane == 0 && rank == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(2 * HN >> 3) << 17) | ((uint32_t)(L::kRows >> 4) << 24);
      uint32_t stage = 0, phase = 0;
      int it = 0;
      bool ok = true;
      auto commit = [&](uint64_t* bar) {
        if (PAIR) {
          umma_commit_pair(map_to_cta(smem_u32(bar), 0));
          umma_commit_pair(map_to_cta(smem_u32(bar), 1));
        } else {
          umma_commit(bar);
        }
      };
      for (int tile = first; tile < p.num_tiles && ok; tile += step, ++it) {
        const int acc = it & 1;
        if (!mbar_wait(&tempty[acc], ((it >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t tmem_d = tmem_base + acc * 2 * HN;
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!mbar_wait(&full[stage], phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = smem_u32(smem + stage * L::kStage), sb = sa + L::kABytes;
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k) {
            const uint64_t ad = smem_desc(sa + k * 32, 16, 1024), bd = smem_desc(sb + k * 32, 16, 1024);
            if (PAIR) umma_bf16_pair(tmem_d, ad, bd, idesc, (kb | k) != 0 ? 1u : 0u);
            else umma_bf16(tmem_d, ad, bd, idesc, (kb | k) != 0 ? 1u : 0u);
          }
          commit(&empty[stage]);
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (ok) commit(&tfull[acc]);
      }
      if (!ok) give_up(32);
      // no instruction reads shared memory or writes the accumulators when they are given back
      if (PAIR) umma_commit_pair(map_to_cta(smem_u32(idle), 0));
      else umma_commit(idle);
      mbar_wait_out(idle, 0);
    }
  } else {
    // ------------------------------ epilogue (a CTA's own 128 rows) ------------------------------
    const int q = warp & 3, e = warp - 2, half = e >> 2;
    uint8_t* stage = smem + L::kEpi + e * 2 * kBoxBytes;
    uint32_t boxes = 0;
    int it = 0, drawn_for = -1;
    bool ok = true;
    dropout::Draw d = {};
    for (int tile = first; tile < p.num_tiles && ok; tile += step, ++it) {
      const int member = tile / per_member, rem = tile % per_member;
      const int row0 = (rem / p.tiles_n) * L::kRows + (int)rank * kBM + q * 32, n0 = (rem % p.tiles_n) * HN;
      const int acc = it & 1;
      if (p.drop && member != drawn_for) {
        d = dropout::draw_of(p.rule, member);
        drawn_for = member;
      }
      if (!warp_wait(&tfull[acc], (it >> 1) & 1, abort_flag)) { ok = false; break; }
      tc_fence_after();
      drain<HN>(p, maps, stage, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * 2 * HN), member, row0, n0, half, lane, d,
                PAIR ? map_to_cta(smem_u32(&tempty[acc]), 0) : 0u, PAIR, &tempty[acc], boxes);
    }
    if (lane == 0) tma_store_wait_all();     // the bulk stores have read the staging boxes and reached memory
    if (!ok && lane == 0) give_up(33);
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) {
    if (threadIdx.x == 0) {
      st_cluster(map_to_cta(smem_u32(tmem_slot + 2), rank ^ 1), issued);
      st_cluster(map_to_cta(smem_u32(tmem_slot + 3), rank ^ 1), (uint32_t)*abort_flag);
    }
    cluster_sync_all();   // neither CTA leaves while its partner may still signal its barriers or read its operands
    if (*abort_flag || told[1]) {                // (both CTAs see the same)
      if (threadIdx.x == 0 && rank == 0) settle<STAGES, L::kStage>(full, issued, told[0]);
      cluster_sync_all();                        // nothing is in flight to either
    }
  }
  if (warp == 1) {
    if (PAIR) tmem_dealloc_pair(tmem_base, L::kCols);
    else tmem_dealloc(tmem_base, L::kCols);
  }
}

constexpr int kPairStages = 5;
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTcThreads, 1)
k_gated_tc_pair(const __grid_constant__ TileMaps maps, const __grid_constant__ TileParams p) {
  gated_tiles<true, 128, kPairStages>(maps, p);
}
// (as many stages as there is room for: few tiles and a long contraction wait for memory; one member's 128 rows, 4096 -> 4096, 64 tiles of 64 hidden units:
// four stages 25.8 us, five 23.8)
template <int HN, int STAGES>
__global__ void __launch_bounds__(kTcThreads, 1) k_gated_tc(const __grid_constant__ TileMaps maps, const __grid_constant__ TileParams p) {
  gated_tiles<false, HN, STAGES>(maps, p);
}

// ------------------------------------------------------------------------------------------------------------------
// Few rows
// ------------------------------------------------------------------------------------------------------------------
// Bound by reading the weight once, so the weight is the tall operand and up to 128 rows are the N columns of the accumulator; clusters of CTAs share a
// contraction.  Two products take this form:
//   forward   128 lanes: 64 hidden units' gate and up rows of the weight; N columns: rows of x
//   dx        128 lanes: columns of the weight, read as it lies (its rows are the contraction: MN-major); N columns: rows of [dg du]
// The partial sums of a cluster meet in shared memory, where every CTA adds up its own share of the rows over all CTAs' partial sums (in their
// order); there g and u of a hidden unit meet, too.
// Rows up to which the forward pass takes this form.  In it and in tiles, us: one member 1024 -> 2048, 32 rows 6.9 and 8.4; 2048 -> 4096, 32 rows 11.2 and 13.9, 40 rows
// 13.1 and 14.0, 64 rows 14.7 and 13.9; 4096 -> 4096, 32 rows 17.7 and 23.3, 64 rows 21.0 and 23.2, 128 rows 25.7 and 23.5.  More members, 32 rows: 4 x 1024 -> 1024 8.8
// and 8.6, 16 x 16.9 and 16.7, 40 x 512 -> 1024 22.8 and 20.9 (16 rows 7.5 and 8.7, 15.6 and 16.5, 22.0 and 20.8); 8 x 50 rows, 1024 -> 1024, 12.2 and 10.7.
constexpr int kRowsForward = 32;
constexpr int kRowsLanes = 128, kRowsPitch = kRowsLanes + 4;      // floats of a row's partial sums
constexpr int kRowsThreads = 192;
constexpr int kRowsSplits = 8;
constexpr int kSms = 148;              // a B200's, against which rules count tiles and splits (no result goes by it)

struct RowsParams {
  int rows, blocks;               // blocks of N rows of a member
  int hidden, width, k_blocks;
  int a_batched, b_batched;
  int activation, drop, vec;
  bf16* out;                      // h (or null), dx
  float* z; int pitch;            // or null
  dropout::Rule rule;
  Counters* counters;
};
// DEEP: for two CTAs an SM at most, with more of the weight under way; else more CTAs share it, one's set-up and end beside another's loads
template <int N, bool DEEP>
struct RowsTile {
  static constexpr int kStage = (128 + N) * kBK * 2;
  static constexpr int kStages = DEEP ? 5 : 3;
  static constexpr int kPerSm = DEEP ? 2 : N == 16 ? 4 : N <= 64 ? 3 : 2;
  static constexpr int kSums = N * kRowsPitch * 4;
  static constexpr int kBars = kStages * kStage > kSums ? kStages * kStage : (kSums + 255) / 256 * 256;
  static constexpr int kTotal = kBars + 256 + 1024;
  static constexpr uint32_t kCols = N < 32 ? 32 : N;
  static_assert(kTotal <= 232448, "shared memory of one CTA");
};

__device__ __forceinline__ float4 ld_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

template <int N, bool DX, bool DEEP, int THREADS>
__device__ __forceinline__ void rows_product(const CUtensorMap& tmA, const CUtensorMap& tmB, const RowsParams& p, uint8_t* smem_raw, int tile, int m, int t0) {
  typedef RowsTile<N, DEEP> L;
  constexpr int kUnits = DX ? kRowsLanes : kRowsLanes / 2;       // hidden units, or columns of dx
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* empty = full + L::kStages;
  uint64_t* done = empty + L::kStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int splits = (int)cluster_size(), rank = (int)cluster_ctarank(), n0 = tile * kUnits;
  const int kb0 = (int)((long long)p.k_blocks * rank / splits), kb1 = (int)((long long)p.k_blocks * (rank + 1) / splits);
  if (threadIdx.x == 32) { prefetch_map(&tmA); prefetch_map(&tmB); }
  if (threadIdx.x == 0) {
    for (int s = 0; s < L::kStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    mbar_init(done, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(tmem_slot, L::kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  float* sums = reinterpret_cast<float*>(smem);
  auto give_up = [&](int where) {
    *abort_flag = 1;
    atomicCAS(&p.counters->status, 0, PBT_ERR_TIMEOUT);
    p.counters->status_info = where;
  };

  if (warp == 0) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      const int ma = p.a_batched ? m : 0, mb = p.b_batched ? m : 0;
      auto load_a = [&](int kb, uint8_t* to, uint64_t* bar) {
        mbar_expect_tx(bar, L::kStage);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (DX) tma_load_3d(to + half * 8192, &tmA, bar, n0 + half * 64, kb * kBK, ma);
          else tma_load_3d(to + half * 8192, &tmA, bar, kb * kBK, half * p.hidden + n0, ma);
        }
      };
      // the weight of the first blocks is asked for before dg and du are there
      const int first = DX ? min(L::kStages, kb1 - kb0) : 0;
      for (int i = 0; i < first; ++i) load_a(kb0 + i, smem + i * L::kStage, &full[i]);
      if (DX) asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");      // dW may begin: it needs nothing of dx
      for (int kb = kb0; kb < kb1; ++kb) {
        uint8_t* to = smem + stage * L::kStage;
        if (kb - kb0 >= first) {
          if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) { ok = false; break; }
          load_a(kb, to, &full[stage]);
        }
        tma_load_3d(to + 16384, &tmB, &full[stage], kb * kBK, t0, mb);
        if (++stage == L::kStages) { stage = 0; phase ^= 1; }
      }
      if (!ok) give_up(41);
      // every stage that was armed has landed before its memory is used again
      for (int s = 0; s < L::kStages; ++s) mbar_wait_out(&full[s], s < (int)stage ? phase : phase ^ 1);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)DX << 15) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kRowsLanes >> 4) << 24);
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(&full[stage], phase, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t sa = smem_u32(smem + stage * L::kStage), sb = sa + 16384;
#pragma unroll
        for (int k = 0; k < kBK / 16; ++k)
          umma_bf16(tmem, DX ? smem_desc(sa + k * 2048, 8192, 1024) : smem_desc(sa + k * 32, 16, 1024), smem_desc(sb + k * 32, 16, 1024), idesc, (kb > kb0 || k > 0) ? 1u : 0u);
        umma_commit(&empty[stage]);
        if (++stage == L::kStages) { stage = 0; phase ^= 1; }
      }
      if (!ok) give_up(42);
      umma_commit(done);          // (also where a wait ran out: no instruction reads shared memory any more)
      mbar_wait_out(done, 0);
      tc_fence_before();
    }
  }
  __syncthreads();                // all loads have landed and all products are complete: the ring's memory becomes the sums
  const bool ok = *abort_flag == 0;
  if (warp >= 2 && warp < 6 && ok) {
    tc_fence_after();
    const int q = warp & 3;
    constexpr int kCols = N < 32 ? N : 32;
#pragma unroll 1
    for (int c0 = 0; c0 < N && t0 + c0 < p.rows; c0 += kCols) {
      uint32_t v[kCols];
      tmem_ld_cols<kCols>(tmem + ((uint32_t)(q * 32) << 16) + c0, v);
      tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < kCols; ++c) sums[(c0 + c) * kRowsPitch + q * 32 + lane] = __uint_as_float(v[c]);
    }
    tc_fence_before();
  }
  cluster_sync_all();
  // a thread has eight hidden units (columns) of a row
  for (int i = threadIdx.x; i < N / splits * (kUnits / 8); i += THREADS) {
    const int c = rank * (N / splits) + i / (kUnits / 8), t = t0 + c, j = i % (kUnits / 8) * 8, col = n0 + j, end = DX ? p.width : p.hidden;
    if (!ok || t >= p.rows || col >= end) continue;
    Eight g = {}, u = {};
    const uint32_t at = smem_u32(sums + c * kRowsPitch + j);
    for (int s = 0; s < splits; ++s) {
      const uint32_t from = map_to_cta(at, s);
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const float4 a = ld_cluster(from + e * 4);
        g.v[e] += a.x; g.v[e + 1] += a.y; g.v[e + 2] += a.z; g.v[e + 3] += a.w;
        if (!DX) {
          const float4 b = ld_cluster(from + (kUnits + e) * 4);
          u.v[e] += b.x; u.v[e + 1] += b.y; u.v[e + 2] += b.z; u.v[e + 3] += b.w;
        }
      }
    }
    const long long row = (long long)m * p.rows + t;
    if (!DX) {
      if (p.z) {                  // (whole groups: the pitch is a multiple of eight)
        float* z = p.z + row * 2 * p.pitch + col;
        store8(z, g);
        store8(z + p.pitch, u);
      }
      if (!p.out) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) g.v[e] = activation_bf16(p.activation, g.v[e]) * u.v[e];
      if (p.drop) {
        const dropout::Draw d = dropout::draw_of(p.rule, m);
        const uint32_t in = dropout::kept_bits(p.rule, d, (uint32_t)t * (uint32_t)((p.hidden + 7) / 8) + (uint32_t)(col / 8));
        const float f = d.on ? d.scale : 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) g.v[e] = (in >> e & 1u) ? g.v[e] * f : 0.f;
      }
    }
    bf16* out = p.out + row * end + col;
    if (p.vec) {
      store8(out, g);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < end) out[e] = __float2bfloat16_rn(g.v[e]);
    }
  }
  cluster_sync_all();             // no CTA leaves while another reads its sums
  if (warp == 1) tmem_dealloc(tmem, L::kCols);
}
// DX: launched while the kernel that makes dg and du runs
template <int N, bool DX, bool DEEP>
__global__ void __launch_bounds__(kRowsThreads, RowsTile<N, DEEP>::kPerSm) k_gated_rows(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const RowsParams p) {
  if (!DX) pdl_prologue();
  extern __shared__ uint8_t smem_raw[];
  rows_product<N, DX, DEEP, kRowsThreads>(tmA, tmB, p, smem_raw, (int)(blockIdx.x / cluster_size()), blockIdx.y / p.blocks, (int)(blockIdx.y % p.blocks) * N);
}

// the parts of a contraction: as many as there are places for CTAs, four blocks each at least
int rows_splits(long long tiles, int k_blocks, long long places) {
  int splits = 1;
  while (splits < kRowsSplits && tiles * splits * 2 <= places && k_blocks >= splits * 2 * 4) splits *= 2;
  return splits;
}
template <int N, bool DX, bool DEEP>
cudaError_t launch_rows(const pbt_gated_desc* d, const RowsParams& p, const CUtensorMap& tmA, const CUtensorMap& tmB, unsigned units, unsigned blocks, int splits,
                        bool after, cudaStream_t s) {
  typedef RowsTile<N, DEEP> L;
  static DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = device_setup(&setup, k_gated_rows<N, DX, DEEP>, L::kTotal, &sms);
  if (e != cudaSuccess) return e;
  return launch_clusters(dim3(units * splits, blocks), kRowsThreads, L::kTotal, splits, after, s, k_gated_rows<N, DX, DEEP>, tmA, tmB, p);
}
// (32 rows, 2048 -> 4096, 256 CTAs: 10.8 us deep, 12.0 else; 40 members x 20 rows, 512 -> 1024, 640: 26 and 22)
template <int N, bool DX>
cudaError_t launch_rows(const pbt_gated_desc* d, const RowsParams& p, const CUtensorMap& tmA, const CUtensorMap& tmB, bool after, cudaStream_t s) {
  const unsigned units = DX ? (d->width + 127) / 128 : (d->hidden + 63) / 64, blocks = (unsigned)p.blocks * d->members;
  const long long tiles = (long long)units * blocks;
  if constexpr (N <= 32) {
    const int splits = rows_splits(tiles, p.k_blocks, 2 * kSms);
    if (tiles * splits <= 2 * kSms) return launch_rows<N, DX, true>(d, p, tmA, tmB, units, blocks, splits, after, s);
  }
  return launch_rows<N, DX, false>(d, p, tmA, tmB, units, blocks, rows_splits(tiles, p.k_blocks, kSms * RowsTile<N, false>::kPerSm), after, s);
}
int rows_columns(const pbt_gated_desc* d) { return d->rows <= 16 ? 16 : d->rows <= 32 ? 32 : d->rows <= 64 ? 64 : 128; }
// what the two products of this form have in common; k: their contraction
bool rows_params(const pbt_gated_desc* d, bool dx, const Operand& b, int k, RowsParams* p, CUtensorMap* tmB) {
  const int n = rows_columns(d);
  p->rows = d->rows; p->hidden = d->hidden; p->width = d->width;
  p->blocks = (d->rows + n - 1) / n;
  p->k_blocks = (k + kBK - 1) / kBK;
  p->b_batched = d->members > 1 && b.member != 0;
  p->vec = (dx ? d->width : d->hidden) % 8 == 0 && ((uintptr_t)p->out & 15) == 0;
  p->counters = (Counters*)d->status_device;
  return make_map(tmB, b.p, k, d->rows, b.row, p->b_batched ? d->members : 1, b.member, n);
}
// dx: the weight as it lies, and everything that does not go by the number of rows
bool dx_params(const pbt_gated_desc* d, const Operand& dz, const Operand& w, RowsParams* p, CUtensorMap* tmA, CUtensorMap* tmB) {
  p->a_batched = d->members > 1 && w.member != 0;
  p->out = (bf16*)d->dx;
  return make_map(tmA, w.p, d->width, 2ll * d->hidden, w.row, p->a_batched ? d->members : 1, w.member, kBK) && rows_params(d, true, dz, 2 * d->hidden, p, tmB);
}

// ------------------------------------------------------------------------------------------------------------------
// dW of a few rows
// ------------------------------------------------------------------------------------------------------------------
// dW = [dg du]^T x with a contraction over at most 32 rows is bound by writing dW (72 members, one row, 344 -> 736: a whole backward pass 40 us, by the
// plain product 94).  A CTA writes 128 x 128 elements: a warp has 16 rows of them, one or two mma.sync steps each, and sends them through shared memory as
// whole 16-byte vectors.  It runs beside dx, which reads the weight meanwhile.
constexpr int kOuterMost = 32, kOuterTile = 128, kOuterHalf = 64, kOuterPitch = kOuterTile + 8;      // (a pitch of 17 x 16 bytes: ldmatrix without conflicts)
struct OuterParams {
  const bf16* dz; int dz_pitch;
  Operand x;
  bf16* dw;
  int rows, hidden2, width, vec;
};
__device__ __forceinline__ void ldmatrix4_trans(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int STEPS>
struct OuterShared {
  bf16 d[STEPS * 16][kOuterPitch], x[STEPS * 16][kOuterPitch];
  bf16 out[8][16][kOuterHalf + 8];
};
template <int STEPS>
__device__ __forceinline__ void outer_product(const OuterParams& p, OuterShared<STEPS>& sm, int c0, int n0, int m, bool wait) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bf16* dz = p.dz + (long long)m * p.rows * p.dz_pitch + n0;
  const bf16* x = p.x.p + m * p.x.member + c0;
  auto &sd = sm.d, &sx = sm.x;
  auto& out = sm.out;
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
  constexpr int kVectors = kOuterTile / 8;
  // (a row's last vector may end behind its last element, inside the same 16 bytes: those columns are not written)
#pragma unroll
  for (int i = threadIdx.x; i < STEPS * 16 * kVectors; i += 256) {
    const int t = i / kVectors, c = i % kVectors * 8;
    *reinterpret_cast<uint4*>(&sx[t][c]) = t < p.rows && c0 + c < p.width ? __ldg(reinterpret_cast<const uint4*>(x + t * p.x.row + c)) : none;
  }
  if (wait) asm volatile("griddepcontrol.wait;" ::: "memory");        // dg and du are there (and read past the read-only path)
#pragma unroll
  for (int i = threadIdx.x; i < STEPS * 16 * kVectors; i += 256) {
    const int t = i / kVectors, c = i % kVectors * 8;
    *reinterpret_cast<uint4*>(&sd[t][c]) = t < p.rows && n0 + c < p.hidden2 ? __ldcg(reinterpret_cast<const uint4*>(dz + (long long)t * p.dz_pitch + c)) : none;
  }
  __syncthreads();
  const int q = lane >> 3, r = lane & 7, gr = lane >> 2, tq = lane & 3;
  uint32_t a[STEPS][4];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) ldmatrix4_trans(a[k], smem_u32(&sd[k * 16 + (q >> 1) * 8 + r][warp * 16 + (q & 1) * 8]));
  const int rows = min(16, p.hidden2 - n0 - warp * 16);
  bf16* dw = p.dw + ((long long)m * p.hidden2 + n0 + warp * 16) * p.width + c0;
#pragma unroll
  for (int h = 0; h < kOuterTile; h += kOuterHalf) {
#pragma unroll
    for (int c = 0; c < kOuterHalf; c += 16) {
      float acc[2][4] = {};
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        uint32_t b[4];
        ldmatrix4_trans(b, smem_u32(&sx[k * 16 + (q & 1) * 8 + r][h + c + (q >> 1) * 8]));
        mma16816(acc[0], a[k], b[0], b[1]);
        mma16816(acc[1], a[k], b[2], b[3]);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        *reinterpret_cast<__nv_bfloat162*>(&out[warp][gr][c + j * 8 + tq * 2]) = __floats2bfloat162_rn(acc[j][0], acc[j][1]);
        *reinterpret_cast<__nv_bfloat162*>(&out[warp][gr + 8][c + j * 8 + tq * 2]) = __floats2bfloat162_rn(acc[j][2], acc[j][3]);
      }
    }
    __syncwarp();
    if (p.vec) {
#pragma unroll
      for (int i = lane; i < 16 * (kOuterHalf / 8); i += 32) {
        const int row = i / (kOuterHalf / 8), c = i % (kOuterHalf / 8) * 8;
        if (row < rows && c0 + h + c < p.width)
          *reinterpret_cast<uint4*>(dw + (long long)row * p.width + h + c) = *reinterpret_cast<const uint4*>(&out[warp][row][c]);
      }
    } else {
      for (int row = 0; row < rows; ++row) {       // pairs of columns from the row's first 4-byte boundary on
        bf16* to = dw + (long long)row * p.width + h;
        const int odd = (int)((uintptr_t)to >> 1) & 1, c = 2 * lane + odd, left = min(kOuterHalf, p.width - c0 - h);
        if (c + 1 < left) *reinterpret_cast<__nv_bfloat162*>(to + c) = __nv_bfloat162(out[warp][row][c], out[warp][row][c + 1]);
        else if (c < left) to[c] = out[warp][row][c];
        if (odd && lane == 0 && left > 0) to[0] = out[warp][row][0];
      }
    }
    __syncwarp();
  }
}

struct FewParams {
  RowsParams dx;
  OuterParams dw;
  int dx_tiles, dx_blocks, dw_columns, dw_rows;      // tiles of a member, CTAs of all members
  long long blocks;                                  // CTAs that have work
};
template <int N>
struct FewShared {
  static constexpr int kOuter = (int)sizeof(OuterShared<N / 16>) + 16;
  static constexpr int kTotal = RowsTile<N, false>::kTotal > kOuter ? RowsTile<N, false>::kTotal : kOuter;
};
// Clusters of CTAs for dx first, then a CTA for every tile of dW; launched while the kernel that makes dg and du runs.
template <int N>
__global__ void __launch_bounds__(256, N == 16 ? 4 : 3) k_gated_few_gradients(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const FewParams p) {
  extern __shared__ uint8_t smem_raw[];
  if ((int)blockIdx.x < p.dx_blocks) {
    const int cluster = (int)(blockIdx.x / cluster_size());
    rows_product<N, true, false, 256>(tmA, tmB, p.dx, smem_raw, cluster % p.dx_tiles, cluster / p.dx_tiles, 0);
    return;
  }
  if (blockIdx.x < p.blocks) {
    const int i = (int)blockIdx.x - p.dx_blocks, per_member = p.dw_columns * p.dw_rows, m = i / per_member, rest = i % per_member;
    outer_product<N / 16>(p.dw, *reinterpret_cast<OuterShared<N / 16>*>(((uintptr_t)smem_raw + 15) & ~(uintptr_t)15), rest % p.dw_columns * kOuterTile,
                          rest / p.dw_columns * kOuterTile, m, true);
  }
}
// A tile of dW alone, beside dx: launched when all CTAs of dx run, that is, when dg and du are complete; it ends after dx.
template <int STEPS>
__global__ void __launch_bounds__(256) k_gated_outer(const OuterParams p) {
  __shared__ __align__(16) OuterShared<STEPS> sm;
  outer_product<STEPS>(p, sm, blockIdx.x * kOuterTile, blockIdx.y * kOuterTile, blockIdx.z, false);
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
template <int N>
cudaError_t launch_few(const pbt_gated_desc* d, FewParams& p, const CUtensorMap& tmA, const CUtensorMap& tmB, cudaStream_t s) {
  static DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = device_setup(&setup, k_gated_few_gradients<N>, FewShared<N>::kTotal, &sms);
  if (e != cudaSuccess) return e;
  p.dx_tiles = (d->width + kRowsLanes - 1) / kRowsLanes;
  p.dw_columns = (d->width + kOuterTile - 1) / kOuterTile;
  p.dw_rows = (2 * d->hidden + kOuterTile - 1) / kOuterTile;
  const int splits = rows_splits((long long)p.dx_tiles * d->members, p.dx.k_blocks, (long long)sms * (N == 16 ? 4 : 3));
  const long long dx = (long long)p.dx_tiles * d->members * splits, dw = (long long)p.dw_columns * p.dw_rows * d->members;
  // Together while there is a place for every CTA (one token, 1024 -> 2048: a backward pass 8.7 us, one after the other 11.9); beyond that tiles of dW that
  // take the place of CTAs of dx hold them up (16 members x 5 rows, 1024 -> 1024: 55 and 35).
  if (dx + dw > (long long)sms * (N == 16 ? 4 : 3)) {
    const cudaError_t first = launch_rows<N, true>(d, p.dx, tmA, tmB, true, s);
    return first != cudaSuccess ? first : launch_after(dim3((unsigned)p.dw_columns, (unsigned)p.dw_rows, (unsigned)d->members), 256, 0, s, k_gated_outer<N / 16>, p.dw);
  }
  p.dx_blocks = (int)dx;
  p.blocks = dx + dw;
  return launch_clusters(dim3((unsigned)((p.blocks + splits - 1) / splits * splits)), 256, FewShared<N>::kTotal, splits, true, s, k_gated_few_gradients<N>, tmA, tmB, p);
}

// ------------------------------------------------------------------------------------------------------------------
// Operands whose rows are not multiples of 16 bytes are copied once into rows that are, both in one launch.
// ------------------------------------------------------------------------------------------------------------------
struct PackJob {
  const bf16* src; long long row, member;
  bf16* dst;
  int rows, cols, per_row;        // elements of a row, vectors of a packed one
  uint32_t vectors;
  Divisor by_row, by_member;      // vectors of a row; rows of a member
  unsigned block0;                // its first block
};
constexpr int kPackEach = 4;      // vectors of a thread
struct PackJobs {
  PackJob job[2];
  int n;
};
// Bound by issue as much as by the transfers.
__global__ void __launch_bounds__(256) k_gated_pack(const PackJobs a) {
  order_begin(kLeads);
  const bool second = a.n > 1 && blockIdx.x >= a.job[1].block0;
  const PackJob j = second ? a.job[1] : a.job[0];
  const uint32_t first = (blockIdx.x - j.block0) * (256 * kPackEach) + threadIdx.x;
  Pieces pieces[kPackEach];
#pragma unroll
  for (int u = 0; u < kPackEach; ++u) {
    const uint32_t i = first + u * 256;
    if (i >= j.vectors) continue;
    const uint32_t at = quotient(i, j.by_row), m = quotient(at, j.by_member);
    const int c = (int)(i - at * j.per_row) * 8;
    pieces[u] = pieces_of(j.src + m * j.member + (long long)(at - m * j.rows) * j.row + c, min(8, j.cols - c));
  }
#pragma unroll
  for (int u = 0; u < kPackEach; ++u) {
    const uint32_t i = first + u * 256;
    if (i < j.vectors) *reinterpret_cast<uint4*>(j.dst + (long long)i * 8) = joined(pieces[u]);
  }
}

}  // namespace

bool tc_aligned(const void* p, long long row, long long member, int members) {
  const long long limit = 1ll << 38;      // (a tensor map's strides end at 2^40 bytes)
  return ((uintptr_t)p & 15) == 0 && row % 8 == 0 && row < limit && (members == 1 || (member % 8 == 0 && member < limit));
}

cudaError_t tc_pack(const PackSource* src, int n, cudaStream_t s) {
  PackJobs a = {};
  unsigned blocks = 0;
  for (int i = 0; i < n; ++i) {
    const PackSource& q = src[i];
    const int per_row = (q.cols + 7) / 8;
    const unsigned long long vectors = (unsigned long long)q.members * q.rows * per_row;
    if (vectors > 0x7FFFF000ull) return cudaErrorInvalidConfiguration;      // (refused before)
    a.job[i] = {q.from.p, q.from.row, q.from.member, q.to, q.rows, q.cols, per_row, (uint32_t)vectors, divisor(per_row), divisor(q.rows), blocks};
    blocks += (unsigned)((vectors + 256 * kPackEach - 1) / (256 * kPackEach));
  }
  a.n = n;
  return launch_with(blocks, 256, 0, s)(k_gated_pack, a);
}

static cudaError_t rows_forward(const pbt_gated_desc* d, const Operand& x, const Operand& w, void* h, float* z, int pitch, bool packed, cudaStream_t s) {
  RowsParams p = {};
  p.a_batched = d->members > 1 && w.member != 0;
  p.activation = d->activation;
  p.drop = d->drop != nullptr;
  if (d->drop) p.rule = dropout::rule_of(*d->drop);
  p.out = (bf16*)h; p.z = z; p.pitch = pitch;
  CUtensorMap tmA, tmB;
  if (!make_map(&tmA, w.p, d->width, 2ll * d->hidden, w.row, p.a_batched ? d->members : 1, w.member, 64) || !rows_params(d, false, x, d->width, &p, &tmB))
    return cudaErrorInvalidValue;
  return rows_columns(d) == 16 ? launch_rows<16, false>(d, p, tmA, tmB, packed, s) : launch_rows<32, false>(d, p, tmA, tmB, packed, s);
}

// dx beyond the rows of tc_gradients: where larger tiles would leave a third of the SMs without one (one member's 500 rows, 2048 -> 2048: a whole backward pass
// 38 us, by the plain product 46; 20 x 250, 1024 -> 512, 320 tiles: 56 and 54).
bool tc_dx_few(const pbt_gated_desc* d) {
  return (long long)((d->rows + 127) / 128) * ((d->width + 127) / 128) * d->members <= 100;      // (blocks of rows times members stay below 65536)
}
cudaError_t tc_dx(const pbt_gated_desc* d, const Operand& dz, const Operand& w, cudaStream_t s) {
  RowsParams p = {};
  CUtensorMap tmA, tmB;
  if (!dx_params(d, dz, w, &p, &tmA, &tmB)) return cudaErrorInvalidValue;
  return rows_columns(d) == 64 ? launch_rows<64, true>(d, p, tmA, tmB, true, s) : launch_rows<128, true>(d, p, tmA, tmB, true, s);
}

bool tc_gradients_few(const pbt_gated_desc* d) { return d->rows <= kOuterMost; }
cudaError_t tc_gradients(const pbt_gated_desc* d, const Operand& dz, const Operand& w, const Operand& x, cudaStream_t s) {
  FewParams p = {};
  CUtensorMap tmA, tmB;
  if (!dx_params(d, dz, w, &p.dx, &tmA, &tmB)) return cudaErrorInvalidValue;
  p.dw = {dz.p, (int)dz.row, x, (bf16*)d->dweight, d->rows, 2 * d->hidden, d->width, d->width % 8 == 0 && ((uintptr_t)d->dweight & 15) == 0};
  return rows_columns(d) == 16 ? launch_few<16>(d, p, tmA, tmB, s) : launch_few<32>(d, p, tmA, tmB, s);
}

cudaError_t tc_forward(const pbt_gated_desc* d, const Operand& x, const Operand& w, void* h, float* z, int pitch, bool packed, cudaStream_t s) {
  if (d->rows <= kRowsForward) return rows_forward(d, x, w, h, z, pitch, packed, s);
  TileParams p;
  memset(&p, 0, sizeof(p));
  p.rows = d->rows; p.hidden = d->hidden;
  p.k_blocks = (d->width + kBK - 1) / kBK;
  p.x_batched = d->members > 1 && x.member != 0;
  p.w_batched = d->members > 1 && w.member != 0;
  p.activation = d->activation;
  p.h = (bf16*)h;
  p.want_z = z != nullptr;
  p.drop = d->drop != nullptr;
  if (d->drop) p.rule = dropout::rule_of(*d->drop);
  p.counters = (Counters*)d->status_device;

  static DeviceSetup setup_pair, setup_wide, setup_narrow;
  int sms = 0;
  cudaError_t e = device_setup(&setup_pair, k_gated_tc_pair, Tile<true, 128, kPairStages>::kTotal, &sms);
  if (e == cudaSuccess) e = device_setup(&setup_wide, k_gated_tc<128, 3>, Tile<false, 128, 3>::kTotal, &sms);
  if (e == cudaSuccess) e = device_setup(&setup_narrow, k_gated_tc<64, 5>, Tile<false, 64, 5>::kTotal, &sms);
  if (e != cudaSuccess) return e;
  // The kernel whose waves of tiles are the shortest together, in waves of a CTA's wide tiles.  A narrow tile has half the products and takes 0.6 of the
  // time; a pair's costs less the longer the contraction (8 members x 160 rows, 2048 -> 2048, two waves of pairs or wide tiles, four of narrow ones: 34,
  // 39 and 47 us; 40 x 512, 1024 -> 1024, 9, 9 and 18: 76, 81 and 102; 60 x 400, 300 -> 2000, 26, 26 and 52: 182, 160 and 187; 14 x 290, 1536 -> 336, 2, 1
  // and 2: 25, 17.5 and 21; 5 x 301, 1008 -> 515, one of each: 14, 14 and 10.6).
  auto waves = [&](int rows, int units, int at_once) {
    const long long tiles = (long long)((d->rows + rows - 1) / rows) * ((d->hidden + units - 1) / units) * d->members;
    return (double)((tiles + at_once - 1) / at_once);
  };
  const double pair = (0.85 + 1.3 / p.k_blocks) * waves(256, 128, sms / 2), wide = waves(128, 128, sms), narrow = 0.6 * waves(128, 64, sms);
  const int hn = narrow < wide && narrow < pair ? 64 : 128;
  const bool use_pair = hn == 128 && pair <= wide;
  const int rows = use_pair ? 256 : 128;
  p.tiles_m = (d->rows + rows - 1) / rows;
  p.tiles_n = (d->hidden + hn - 1) / hn;
  p.num_tiles = p.tiles_m * p.tiles_n * d->members;

  TileMaps maps;
  memset(&maps, 0, sizeof(maps));
  const long long all = (long long)d->rows;
  bool ok = make_map(&maps.x, x.p, d->width, all, x.row, p.x_batched ? d->members : 1, x.member, kBM) &&
            make_map(&maps.w, w.p, d->width, 2ll * d->hidden, w.row, p.w_batched ? d->members : 1, w.member, hn);
  if (h && d->hidden % 8 == 0 && ((uintptr_t)h & 15) == 0)
    p.h_tma = make_map(&maps.h, h, d->hidden, all, d->hidden, d->members, all * d->hidden, 32, 2, 32, 64);
  if (z)
    ok = ok && make_map(&maps.g, z, pitch, all, 2 * pitch, d->members, all * 2 * pitch, 32, 4, 32, 128) &&
         make_map(&maps.u, z + pitch, pitch, all, 2 * pitch, d->members, all * 2 * pitch, 32, 4, 32, 128);
  if (!ok) return cudaErrorInvalidValue;

  auto launch = [&](auto kernel, int bytes, int at_once, int ctas) {
    return launch_ordered(packed ? kAfter : 0, (unsigned)(ctas * std::min(p.num_tiles, at_once)), kTcThreads, bytes, s, kernel, maps, p);
  };
  if (use_pair) return launch(k_gated_tc_pair, Tile<true, 128, kPairStages>::kTotal, sms / 2, 2);
  if (hn == 128) return launch(k_gated_tc<128, 3>, Tile<false, 128, 3>::kTotal, sms, 1);
  return launch(k_gated_tc<64, 5>, Tile<false, 64, 5>::kTotal, sms, 1);
}

}  // namespace gated
}  // namespace pbt
