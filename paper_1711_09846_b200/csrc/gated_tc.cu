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
using dropout::Eight;
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
  pbt_drop_rule rule;
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

// a bounded wait of a whole warp: every lane gives up if one does
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag));
}

// h of 32 hidden units of a row, in the place of u
template <int KIND>
__device__ __forceinline__ void apply(const uint32_t* g, uint32_t* u) {
#pragma unroll
  for (int c = 0; c < 32; ++c) u[c] = __float_as_uint(activation(KIND, __uint_as_float(g[c])) * __uint_as_float(u[c]));
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
        const U4 w = dropout::draw_group(d, (uint32_t)row * groups + (uint32_t)(col / dropout::kGroup + j));
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

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0;
  const int first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;
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
        }
      }
      if (!ok) give_up(31);
      // Every stage that was armed has landed before the CTA ends, and been read unless a wait ran out.  What a pair's second CTA loads is
      // counted by the leader alone; when one of them gave up, it may not be counted at all, and has a millisecond to land.
      if (rank == 0)
        for (int s = 0; s < STAGES; ++s) mbar_wait_out(&full[s], s < (int)stage ? phase : phase ^ 1);
      for (int i = 0; PAIR && !ok && i < 16384; ++i) __nanosleep(64);
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
  if (PAIR) cluster_sync_all();   // neither CTA leaves while its partner may still signal its barriers or read its operands
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
template <int HN, int STAGES>
__global__ void __launch_bounds__(kTcThreads, 1) k_gated_tc(const __grid_constant__ TileMaps maps, const __grid_constant__ TileParams p) {
  gated_tiles<false, HN, STAGES>(maps, p);
}

// ------------------------------------------------------------------------------------------------------------------
// Few rows
// ------------------------------------------------------------------------------------------------------------------
// Up to 128 rows a member: bound by reading the weight once, so the weight is the tall operand.  A CTA has 64 hidden units, whose gate and up rows
// are the 128 lanes of the accumulator, and all rows of x as its N columns; a cluster of `splits` CTAs shares the contraction.  The partial sums meet
// in shared memory, where every CTA of the cluster adds up its own share of the rows over all CTAs' partial sums (in their order), and g and u
// of a hidden unit meet, too.
constexpr int kRowsUnits = 64, kRowsPitch = 2 * kRowsUnits + 4;      // floats of a row's partial sums: 64 g, 64 u
constexpr int kRowsMost = 128;
constexpr int kRowsThreads = 192;
constexpr int kRowsSplits = 8;

struct RowsParams {
  int rows, hidden, k_blocks;
  int x_batched, w_batched;
  int activation, drop, vec;
  bf16* h;                        // or null
  float* z; int pitch;            // or null
  pbt_drop_rule rule;
  Counters* counters;
};
template <int N>
struct RowsTile {
  static constexpr int kStage = (128 + N) * kBK * 2;
  static constexpr int kStages = N <= 32 ? 5 : N == 64 ? 4 : 6;          // two CTAs of an SM share its memory, one with 128 rows
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

template <int N>
__global__ void __launch_bounds__(kRowsThreads, N <= 64 ? 2 : 1) k_gated_rows(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const RowsParams p) {
  pdl_prologue();
  typedef RowsTile<N> L;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* empty = full + L::kStages;
  uint64_t* done = empty + L::kStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int splits = (int)cluster_size(), rank = (int)cluster_ctarank();
  const int n0 = (int)(blockIdx.x / splits) * kRowsUnits, m = blockIdx.y;
  const int kb0 = p.k_blocks * rank / splits, kb1 = p.k_blocks * (rank + 1) / splits;
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
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag)) { ok = false; break; }
        uint8_t* to = smem + stage * L::kStage;
        mbar_expect_tx(&full[stage], L::kStage);
        tma_load_3d(to, &tmW, &full[stage], kb * kBK, n0, p.w_batched ? m : 0);
        tma_load_3d(to + kRowsUnits * kBK * 2, &tmW, &full[stage], kb * kBK, p.hidden + n0, p.w_batched ? m : 0);
        tma_load_3d(to + 2 * kRowsUnits * kBK * 2, &tmX, &full[stage], kb * kBK, 0, p.x_batched ? m : 0);
        if (++stage == L::kStages) { stage = 0; phase ^= 1; }
      }
      if (!ok) give_up(41);
      // every stage that was armed has landed before its memory is used again
      for (int s = 0; s < L::kStages; ++s) mbar_wait_out(&full[s], s < (int)stage ? phase : phase ^ 1);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(&full[stage], phase, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t sa = smem_u32(smem + stage * L::kStage), sb = sa + 2 * kRowsUnits * kBK * 2;
#pragma unroll
        for (int k = 0; k < kBK / 16; ++k)
          umma_bf16(tmem, smem_desc(sa + k * 32, 16, 1024), smem_desc(sb + k * 32, 16, 1024), idesc, (kb > kb0 || k > 0) ? 1u : 0u);
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
  if (warp >= 2 && ok) {
    tc_fence_after();
    const int q = warp & 3;
    constexpr int kCols = N < 32 ? N : 32;
#pragma unroll 1
    for (int c0 = 0; c0 < N && c0 < p.rows; c0 += kCols) {
      uint32_t v[kCols];
      tmem_ld_cols<kCols>(tmem + ((uint32_t)(q * 32) << 16) + c0, v);
      tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < kCols; ++c) sums[(c0 + c) * kRowsPitch + q * 32 + lane] = __uint_as_float(v[c]);
    }
    tc_fence_before();
  }
  cluster_sync_all();
  // a thread has eight hidden units of a row
  for (int i = threadIdx.x; i < N / splits * (kRowsUnits / 8); i += kRowsThreads) {
    const int t = rank * (N / splits) + i / (kRowsUnits / 8), j = i % (kRowsUnits / 8) * 8, col = n0 + j;
    if (!ok || t >= p.rows || col >= p.hidden) continue;
    float g[8] = {}, u[8] = {};
    const uint32_t at = smem_u32(sums + t * kRowsPitch + j);
    for (int s = 0; s < splits; ++s) {
      const uint32_t from = map_to_cta(at, s);
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const float4 a = ld_cluster(from + e * 4), b = ld_cluster(from + (kRowsUnits + e) * 4);
        g[e] += a.x; g[e + 1] += a.y; g[e + 2] += a.z; g[e + 3] += a.w;
        u[e] += b.x; u[e + 1] += b.y; u[e + 2] += b.z; u[e + 3] += b.w;
      }
    }
    const long long row = (long long)m * p.rows + t;
    if (p.z) {                    // (whole groups: the pitch is a multiple of eight)
      float* z = p.z + row * 2 * p.pitch + col;
      store8(z, {g[0], g[1], g[2], g[3], g[4], g[5], g[6], g[7]});
      store8(z + p.pitch, {u[0], u[1], u[2], u[3], u[4], u[5], u[6], u[7]});
    }
    if (!p.h) continue;
    Eight v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v.v[e] = activation(p.activation, g[e]) * u[e];
    if (p.drop) {
      const dropout::Draw d = dropout::draw_of(p.rule, m);
      const uint32_t in = dropout::kept_bits(d, (uint32_t)t * (uint32_t)((p.hidden + 7) / 8) + (uint32_t)(col / 8));
      const float f = d.on ? d.scale : 1.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v.v[e] = (in >> e & 1u) ? v.v[e] * f : 0.f;
    }
    bf16* h = p.h + row * p.hidden + col;
    if (p.vec) {
      store8(h, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < p.hidden) h[e] = __float2bfloat16_rn(v.v[e]);
    }
  }
  cluster_sync_all();             // no CTA leaves while another reads its sums
  if (warp == 1) tmem_dealloc(tmem, L::kCols);
}

template <int N>
cudaError_t launch_rows(const pbt_gated_desc* d, const RowsParams& p, const CUtensorMap& tmX, const CUtensorMap& tmW, int splits, cudaStream_t s) {
  static DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = device_setup(&setup, k_gated_rows<N>, RowsTile<N>::kTotal, &sms);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((d->hidden + kRowsUnits - 1) / kRowsUnits * splits), (unsigned)d->members);
  cfg.blockDim = dim3(kRowsThreads);
  cfg.dynamicSmemBytes = RowsTile<N>::kTotal;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)splits;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_gated_rows<N>, tmX, tmW, p);
}

// ------------------------------------------------------------------------------------------------------------------
// Operands whose rows are not multiples of 16 bytes are copied once into rows that are, both in one launch.
// ------------------------------------------------------------------------------------------------------------------
struct PackJob {
  const bf16* src; long long row, member;
  bf16* dst;
  int members, rows, cols, to;    // elements of a row, and rounded up to 8
  unsigned block0;                // its first block
};
struct PackJobs {
  PackJob job[2];
  int n;
};
__global__ void __launch_bounds__(256) k_gated_pack(const PackJobs a) {
  pdl_prologue();
  const PackJob& j = a.job[a.n > 1 && blockIdx.x >= a.job[1].block0];
  const long long i = (long long)(blockIdx.x - j.block0) * 256 + threadIdx.x;
  const int per_row = j.to / 8;
  const long long at = i / per_row;
  if (at >= (long long)j.members * j.rows) return;
  const int c = (int)(i - at * per_row) * 8, m = (int)(at / j.rows);
  const bf16* from = j.src + m * j.member + (at - (long long)m * j.rows) * j.row + c;
  __align__(16) bf16 v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c + e < j.cols ? from[e] : __float2bfloat16_rn(0.f);
  *reinterpret_cast<uint4*>(j.dst + at * j.to + c) = *reinterpret_cast<const uint4*>(v);
}

}  // namespace

bool tc_aligned(const void* p, long long row, long long member, int members) {
  const long long limit = 1ll << 38;      // (a tensor map's strides end at 2^40 bytes)
  return ((uintptr_t)p & 15) == 0 && row % 8 == 0 && row < limit && (members == 1 || (member % 8 == 0 && member < limit));
}

cudaError_t tc_pack(const PackSource* src, int n, cudaStream_t s) {
  PackJobs a = {};
  unsigned long long blocks = 0;
  for (int i = 0; i < n; ++i) {
    const PackSource& q = src[i];
    const int to = (q.cols + 7) / 8 * 8;
    a.job[i] = {q.from.p, q.from.row, q.from.member, q.to, q.members, q.rows, q.cols, to, (unsigned)blocks};
    blocks += ((unsigned long long)q.members * q.rows * (to / 8) + 255) / 256;
  }
  if (blocks > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
  a.n = n;
  return launch_with((unsigned)blocks, 256, 0, s)(k_gated_pack, a);
}

static cudaError_t rows_forward(const pbt_gated_desc* d, const Operand& x, const Operand& w, void* h, float* z, int pitch, cudaStream_t s) {
  RowsParams p = {};
  p.rows = d->rows; p.hidden = d->hidden;
  p.k_blocks = (d->width + kBK - 1) / kBK;
  p.x_batched = d->members > 1 && x.member != 0;
  p.w_batched = d->members > 1 && w.member != 0;
  p.activation = d->activation;
  p.drop = d->drop != nullptr;
  if (d->drop) p.rule = *d->drop;
  p.vec = d->hidden % 8 == 0 && ((uintptr_t)h & 15) == 0;
  p.h = (bf16*)h; p.z = z; p.pitch = pitch;
  p.counters = (Counters*)d->status_device;
  const int n = d->rows <= 16 ? 16 : d->rows <= 32 ? 32 : d->rows <= 64 ? 64 : 128;
  CUtensorMap tmX, tmW;
  if (!make_map(&tmX, x.p, d->width, d->rows, x.row, p.x_batched ? d->members : 1, x.member, n) ||
      !make_map(&tmW, w.p, d->width, 2ll * d->hidden, w.row, p.w_batched ? d->members : 1, w.member, kRowsUnits))
    return cudaErrorInvalidValue;
  // as many parts of the contraction as there are SMs to spare for, four blocks of it each at least
  const long long tiles = (long long)((d->hidden + kRowsUnits - 1) / kRowsUnits) * d->members, room = n <= 64 ? 296 : 148;
  int splits = 1;
  while (splits < kRowsSplits && tiles * splits * 2 <= room && p.k_blocks >= splits * 2 * 4) splits *= 2;
  switch (n) {
    case 16: return launch_rows<16>(d, p, tmX, tmW, splits, s);
    case 32: return launch_rows<32>(d, p, tmX, tmW, splits, s);
    case 64: return launch_rows<64>(d, p, tmX, tmW, splits, s);
    default: return launch_rows<128>(d, p, tmX, tmW, splits, s);
  }
}

cudaError_t tc_forward(const pbt_gated_desc* d, const Operand& x, const Operand& w, void* h, float* z, int pitch, cudaStream_t s) {
  if (d->rows <= kRowsMost) return rows_forward(d, x, w, h, z, pitch, s);
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
  if (d->drop) p.rule = *d->drop;
  p.counters = (Counters*)d->status_device;

  int dev = 0, sms = 148;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  auto waves = [&](int rows, int units, int at_once) {
    const long long tiles = (long long)((d->rows + rows - 1) / rows) * ((d->hidden + units - 1) / units) * d->members;
    return (double)((tiles + at_once - 1) / at_once);
  };
  const double pair = 0.96 * waves(256, 128, sms / 2), wide = waves(128, 128, sms), narrow = 0.6 * waves(128, 64, sms);
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

  auto launch = [&](auto kernel, DeviceSetup* setup, int bytes, int at_once, int ctas) {
    int count = 0;
    const cudaError_t err = device_setup(setup, kernel, bytes, &count);
    if (err != cudaSuccess) return err;
    return launch_with((unsigned)(ctas * std::min(p.num_tiles, at_once)), kTcThreads, bytes, s)(kernel, maps, p);
  };
  static DeviceSetup setup_pair, setup_wide, setup_narrow;
  if (use_pair) return launch(k_gated_tc_pair, &setup_pair, Tile<true, 128, kPairStages>::kTotal, sms / 2, 2);
  if (hn == 128) return launch(k_gated_tc<128, 3>, &setup_wide, Tile<false, 128, 3>::kTotal, sms, 1);
  return launch(k_gated_tc<64, 4>, &setup_narrow, Tile<false, 64, 4>::kTotal, sms, 1);
}

}  // namespace gated
}  // namespace pbt
