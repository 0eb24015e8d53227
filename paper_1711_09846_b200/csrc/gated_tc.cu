// bf16 gated units on the tensor cores: both projections, the activation, the product and dropout in one kernel.
//
//   k_gated_tc_pair / k_gated_tc   tiles of 256 (128) rows and 128 (64) hidden units: the B operand of one tcgen05 product is the gate's weight
//                                  rows and the up-projection's for the same hidden units, so that g and u of a hidden unit meet in one TMEM lane
//   k_gated_rows                   a few rows (single tokens): bound by reading the weight once, mma.sync with eight gate rows and the eight
//                                  up rows of the same hidden units as the tall operand: g and u meet in one thread
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
constexpr int kRowsOut = 8;       // hidden units of a CTA

__device__ __forceinline__ void copy16(void* slot, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(slot)), "l"(from) : "memory");
}
__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct RowsParams {
  Operand x, w;
  int rows, hidden, width;        // width: elements of a row that exist, a multiple of 8
  int activation, drop;
  bf16* h;                        // or null
  float* z; int pitch;            // or null
  pbt_drop_rule rule;
};

// 8 hidden units of a member and all its rows: the eight warps take every eighth block of 64 inputs.  Eight gate rows and eight up rows of the
// weight are the tall operand of mma.sync (16 x 16), eight rows of x the narrow one; the contraction index runs in the order in which
// 16-byte loads deliver it, in both operands.  Blocks come through a ring of the warp's own (cp.async), every lane reading back what it copied.
// The warps' sums meet in shared memory.
template <int GROUPS> struct RowsRing {
  static constexpr int kStages = GROUPS == 8 ? 2 : GROUPS == 4 ? 3 : 4;
  static constexpr int kVectors = 4 + 2 * GROUPS;                   // 16-byte vectors of a lane in a block of 64 inputs
  static constexpr int kBytes = kVectors * 512;
  static constexpr int kPitch = GROUPS * 8 + 1;                     // of the sums [8 warps][8 gates, 8 ups][rows]
  static constexpr int kSums = 8 * 2 * kRowsOut * kPitch * 4;
  static constexpr int kTotal = 8 * kStages * kBytes > kSums ? 8 * kStages * kBytes : kSums;
};
template <int GROUPS>
__global__ void __launch_bounds__(256) k_gated_rows(const RowsParams a) {
  pdl_prologue();
  extern __shared__ __align__(16) uint8_t rows_smem[];
  typedef RowsRing<GROUPS> Ring;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, tq = lane & 3;
  const int n0 = blockIdx.x * kRowsOut, m = blockIdx.y, T = a.rows;
  uint8_t* ring = rows_smem + warp * (Ring::kStages * Ring::kBytes) + lane * 16;
  const bf16* w0 = a.w.p + m * a.w.member + (long long)(n0 + gr) * a.w.row;
  const bf16* w1 = w0 + a.hidden * a.w.row;
  const bf16* x = a.x.p + m * a.x.member + gr * a.x.row;
  const bool in_w = n0 + gr < a.hidden;
  auto put = [&](uint8_t* slot, const bf16* from, bool in) {
    if (in) copy16(slot, from);
    else *reinterpret_cast<uint4*>(slot) = make_uint4(0u, 0u, 0u, 0u);
  };
  auto ask = [&](int k0, int s) {
    if (k0 < a.width) {
      uint8_t* to = ring + s * Ring::kBytes;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + h * 32 + tq * 8;
        const bool in = k < a.width;
        put(to + h * 512, w0 + k, in && in_w);
        put(to + (2 + h) * 512, w1 + k, in && in_w);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) put(to + (4 + 2 * g + h) * 512, x + g * 8 * a.x.row + k, in && g * 8 + gr < T);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < Ring::kStages; ++s) ask(warp * 64 + s * 512, s);
  float acc[GROUPS][4] = {};      // [0, 1]: gate, [2, 3]: up, of two rows
  int stage = 0;
  for (int k0 = warp * 64; k0 < a.width; k0 += 512) {
    asm volatile("cp.async.wait_group %0;" ::"n"(Ring::kStages - 1) : "memory");
    const uint4* from = reinterpret_cast<const uint4*>(ring + stage * Ring::kBytes);
    uint4 wv[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) { wv[0][h] = from[h * 32]; wv[1][h] = from[(2 + h) * 32]; }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 xv = from[(4 + 2 * g + h) * 32];
        mma16816(acc[g], wv[0][h].x, wv[1][h].x, wv[0][h].y, wv[1][h].y, xv.x, xv.y);
        mma16816(acc[g], wv[0][h].z, wv[1][h].z, wv[0][h].w, wv[1][h].w, xv.z, xv.w);
      }
    ask(k0 + Ring::kStages * 512, stage);
    if (++stage == Ring::kStages) stage = 0;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();     // the rings' memory becomes the warps' sums
  float* red = reinterpret_cast<float*>(rows_smem);
#pragma unroll
  for (int g = 0; g < GROUPS; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[(warp * 2 * kRowsOut + gr + 8 * (e >> 1)) * Ring::kPitch + g * 8 + tq * 2 + (e & 1)] = acc[g][e];
  __syncthreads();
  const int n = threadIdx.x % kRowsOut, col = n0 + n;
  if (col >= a.hidden) return;
  dropout::Draw d = {};
  if (a.drop) d = dropout::draw_of(a.rule, m);
  for (int t = threadIdx.x / kRowsOut; t < T; t += 256 / kRowsOut) {
    float g = 0.f, u = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      g += red[(k * 2 * kRowsOut + n) * Ring::kPitch + t];
      u += red[(k * 2 * kRowsOut + kRowsOut + n) * Ring::kPitch + t];
    }
    const long long row = (long long)m * T + t;
    if (a.z) {
      a.z[row * 2 * a.pitch + col] = g;
      a.z[row * 2 * a.pitch + a.pitch + col] = u;
    }
    if (!a.h) continue;
    float v = activation(a.activation, g) * u;
    if (d.on) {
      static_assert(kRowsOut == dropout::kGroup, "a CTA's hidden units are one block of the generator");
      const U4 w = dropout::draw_group(d, (uint32_t)t * (uint32_t)gridDim.x + blockIdx.x);
      v = dropout::kept(w, n, d.limit) ? v * d.scale : 0.f;
    }
    a.h[row * a.hidden + col] = __float2bfloat16_rn(v);
  }
}

template <int GROUPS>
cudaError_t launch_rows(const RowsParams& a, int members, cudaStream_t s) {
  static DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = device_setup(&setup, k_gated_rows<GROUPS>, RowsRing<GROUPS>::kTotal, &sms);
  if (e != cudaSuccess) return e;
  return launch_with(dim3((a.hidden + kRowsOut - 1) / kRowsOut, members), 256, RowsRing<GROUPS>::kTotal, s)(k_gated_rows<GROUPS>, a);
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

cudaError_t tc_rows_forward(const pbt_gated_desc* d, const Operand& x, const Operand& w, void* h, float* z, int pitch, cudaStream_t s) {
  RowsParams a = {x, w, d->rows, d->hidden, (d->width + 7) / 8 * 8, d->activation, d->drop != nullptr, (bf16*)h, z, pitch, {}};
  if (d->drop) a.rule = *d->drop;
  if (d->rows <= 8) return launch_rows<1>(a, d->members, s);
  if (d->rows <= 16) return launch_rows<2>(a, d->members, s);
  if (d->rows <= 32) return launch_rows<4>(a, d->members, s);
  return launch_rows<8>(a, d->members, s);
}

cudaError_t tc_forward(const pbt_gated_desc* d, const Operand& x, const Operand& w, void* h, float* z, int pitch, cudaStream_t s) {
  if (tc_few_rows(d)) return tc_rows_forward(d, x, w, h, z, pitch, s);
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
