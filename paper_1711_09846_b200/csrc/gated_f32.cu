// fp32 gated units on the ALUs (their results are good to some 2^-24 of the sums' terms, which the tensor cores' formats do not give): the three
// products of a step over tiles of 16 to 128 rows by 64 columns,
//   forward   g, u = x W^T with the activation, the product and dropout in its epilogue
//   dx        [dg du] W
//   dW        [dg du]^T x
// Bound by shared memory's reads and the ALUs' issue together: 40 members, 128 rows, 512 -> 512 forward 139 us (38.6 TFLOP/s), both gradients 226 (47.5).
#include <algorithm>

#include "gated.cuh"
#include "tc_common.cuh"

namespace pbt {
namespace gated {
namespace {

using dropout::Eight;
using dropout::store8;

constexpr int kK = 16, kStages = 3, kSplits = 8, kCols = 64;
constexpr int kPitchN = kCols + 4;        // floats of a staged row of columns, and of the sums

// A tile of BM rows and 64 columns (forward: 32 hidden units' g and u); a thread has TM x 8 of its elements, a warp's lanes are 4 x 8 of the threads.
template <int BM_, int TM_, int WARPS>
struct Shape {
  static constexpr int BM = BM_, TM = TM_, kThreads = BM / TM * 8, kPerSm = WARPS * 32 / kThreads, kPitchM = BM + 4;
  static constexpr int kA = kK * kPitchM, kB = kK * kPitchN, kStage = kA + kB;      // floats
  static constexpr int kFloats = kStages * kStage > BM * kPitchN ? kStages * kStage : BM * kPitchN;
  static_assert(kThreads % 32 == 0 && (TM == 8 || TM == 4 || TM == 2), "whole warps; rows in vectors");
};
typedef Shape<128, 8, 12> Tall;
typedef Shape<64, 8, 12> Short;
typedef Shape<32, 4, 16> Half;
typedef Shape<16, 2, 16> Few;

// two fp32 multiply-adds in one instruction
__device__ __forceinline__ void fma2(unsigned long long& d, unsigned long long a, unsigned long long b) {
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(a), "l"(b));
}
__device__ __forceinline__ unsigned long long both(float v) {
  unsigned long long d;
  asm("mov.b64 %0, {%1, %1};" : "=l"(d) : "f"(v));
  return d;
}
__device__ __forceinline__ float2 halves(unsigned long long v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}

struct ProductParams {
  const float* a; long long lda, a_member;      // [M][K], or [K][M]
  const float* b; long long ldb, b_member;      // [N][K], or [K][N]; forward: row n of the first half of the columns and n + hidden
  float* c; long long ldc, c_member;            // [M][N]; forward: h, or null
  int M, N, K;                                  // forward: N hidden units
  int tiles_n;
  bool vec_a, vec_b, vec_c;
  // forward
  float* z; int pitch;
  int activation, drop;
  dropout::Rule rule;
};

// a box of kK rows and COLS floats into staged rows of PITCH, `rows` x `cols` of which exist (the others are zero)
template <int THREADS, int COLS, int PITCH>
__device__ __forceinline__ void copy_rows(uint32_t to, const float* from, long long ld, int rows, int cols, bool vectors) {
  if (vectors) {
    constexpr int kStep = THREADS / (COLS / 4);
    static_assert(kStep >= 1 && kK % kStep == 0, "whole steps");
    const int r0 = threadIdx.x / (COLS / 4), c = threadIdx.x % (COLS / 4) * 4, bytes = min(max(cols - c, 0), 4) * 4;
    const float* at = from + r0 * ld + c;
    const long long step = kStep * ld;
    to += (r0 * PITCH + c) * 4;
#pragma unroll
    for (int i = 0; i < kK / kStep; ++i) {
      const int have = r0 + i * kStep < rows ? bytes : 0;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + i * kStep * PITCH * 4), "l"(have ? at : from), "r"(have) : "memory");
      at += step;
    }
  } else {
    constexpr int kStep = THREADS > COLS ? THREADS / COLS : 1, kEach = COLS > THREADS ? COLS / THREADS : 1;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int r0 = threadIdx.x / COLS, c = threadIdx.x % COLS + e * THREADS, bytes = c < cols ? 4 : 0;
      const float* at = from + r0 * ld + c;
      const long long step = kStep * ld;
      const uint32_t out = to + (r0 * PITCH + c) * 4;
#pragma unroll 4
      for (int i = 0; i < kK / kStep; ++i) {
        const int have = r0 + i * kStep < rows ? bytes : 0;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(out + i * kStep * PITCH * 4), "l"(have ? at : from), "r"(have) : "memory");
        at += step;
      }
    }
  }
}
// The same of ROWS rows and kK floats, turned on the way: a staged row holds the box's column.  Single elements, of any alignment: a warp takes 64 bytes of
// two rows (staged as they lie, with vectors of k read for the products, 40 members, 128 rows, 512 -> 512 took 160 us, the loop over rows of m and n x).
template <int THREADS, int ROWS, int PITCH>
__device__ __forceinline__ void copy_turned(uint32_t to, const float* from, long long ld, int rows, int cols) {
  constexpr int kStep = THREADS / kK;
  static_assert(ROWS % kStep == 0, "whole steps");
  const int r0 = threadIdx.x / kK, k = threadIdx.x % kK, bytes = k < cols ? 4 : 0;
  const float* at = from + r0 * ld + k;
  const long long step = kStep * ld;
  to += (k * PITCH + r0) * 4;
#pragma unroll 8
  for (int i = 0; i < ROWS / kStep; ++i) {
    const int have = r0 + i * kStep < rows ? bytes : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + i * kStep * 4), "l"(have ? at : from), "r"(have) : "memory");
    at += step;
  }
}

// K goes in slices of 16 through a ring of cp.async stages, rows of m and of n for every k.  The CTAs of a cluster share the contraction; every one adds up its
// share of the tile's rows over all their sums, in their order.  Bound by shared memory: a thread's 8 x 8 multiply-adds take 16 values from it, a warp's
// loads as many cycles as its products (which go two to an instruction, or their issue would be the limit: 264 us instead of 226 for both gradients of
// 40 x 128, 512 -> 512).
template <typename S, bool A_MN, bool GATED>
__device__ __forceinline__ void product_tile(const ProductParams& p, float* f32_smem, int tile, int m, int splits, int rank) {
  constexpr int BM = S::BM, TM = S::TM, kThreads = S::kThreads, kPitchM = S::kPitchM, kUnits = GATED ? kCols / 2 : kCols;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tx = lane & 7, ty = warp * 4 + (lane >> 3);
  const int m0 = tile / p.tiles_n * BM, n0 = tile % p.tiles_n * kUnits, rows = min(BM, p.M - m0), cols = min(kUnits, p.N - n0);
  const int slices = (p.K + kK - 1) / kK, s0 = (int)((long long)slices * rank / splits), s1 = (int)((long long)slices * (rank + 1) / splits);
  const float* A = p.a + m * p.a_member + (A_MN ? m0 : m0 * p.lda);
  const float* B = p.b + m * p.b_member + (GATED ? n0 * p.ldb : n0);      // forward: [N][K], else [K][N]
  const float* B2 = B + p.N * p.ldb;                                      // forward: the up-projection's rows
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(f32_smem);

  int slot = 0;                                   // of the slice that is asked for next
  auto load = [&](int s) {
    if (s < s1) {
      const uint32_t sa = base + slot * S::kStage * 4, sb = sa + S::kA * 4;
      const int k0 = s * kK, ks = p.K - k0;
      if (A_MN) copy_rows<kThreads, BM, kPitchM>(sa, A + k0 * p.lda, p.lda, ks, rows, p.vec_a);
      else copy_turned<kThreads, BM, kPitchM>(sa, A + k0, p.lda, rows, ks);
      if (GATED) {
        copy_turned<kThreads, kUnits, kPitchN>(sb, B + k0, p.ldb, cols, ks);
        copy_turned<kThreads, kUnits, kPitchN>(sb + kUnits * 4, B2 + k0, p.ldb, cols, ks);
      } else {
        copy_rows<kThreads, kCols, kPitchN>(sb, B + k0 * p.ldb, p.ldb, ks, cols, p.vec_b);
      }
    }
    slot = slot + 1 == kStages ? 0 : slot + 1;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto row_of = [&](int i) { return TM >= 4 ? (i >> 2) * (BM / 2) + ty * 4 + (i & 3) : ty * TM + i; };

  unsigned long long acc[TM][4] = {};             // pairs of neighbouring columns: 4 tx .. and 32 + 4 tx ..
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) load(s0 + s);
  int at = 0;
#pragma unroll 1
  for (int s = s0; s < s1; ++s) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncthreads();
    load(s + kStages - 1);
    const float *sa = f32_smem + at * S::kStage, *sb = sa + S::kA;
    at = at + 1 == kStages ? 0 : at + 1;
#pragma unroll
    for (int k = 0; k < kK; ++k) {
      const ulonglong2 b0 = *reinterpret_cast<const ulonglong2*>(sb + k * kPitchN + tx * 4), b1 = *reinterpret_cast<const ulonglong2*>(sb + k * kPitchN + kCols / 2 + tx * 4);
      float a[TM];
      if constexpr (TM >= 4) {
#pragma unroll
        for (int h = 0; h < TM / 4; ++h) {
          const float4 q = *reinterpret_cast<const float4*>(sa + k * kPitchM + h * (BM / 2) + ty * 4);
          a[h * 4] = q.x; a[h * 4 + 1] = q.y; a[h * 4 + 2] = q.z; a[h * 4 + 3] = q.w;
        }
      } else {
        const float2 q = *reinterpret_cast<const float2*>(sa + k * kPitchM + ty * 2);
        a[0] = q.x; a[1] = q.y;
      }
#pragma unroll
      for (int r = 0; r < TM; ++r) {
        const unsigned long long a2 = both(a[r]);
        fma2(acc[r][0], a2, b0.x);
        fma2(acc[r][1], a2, b0.y);
        fma2(acc[r][2], a2, b1.x);
        fma2(acc[r][3], a2, b1.y);
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();              // the ring's memory becomes the sums
#pragma unroll
  for (int r = 0; r < TM; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<float2*>(f32_smem + row_of(r) * kPitchN + (j >> 1) * (kCols / 2) + tx * 4 + (j & 1) * 2) = halves(acc[r][j]);
  if (splits > 1) tc::cluster_sync_all();
  else __syncthreads();
  auto sum = [&](int r, int c, float* v) {      // four neighbouring columns
    const uint32_t at = base + (r * kPitchN + c) * 4;
    if (splits == 1) {
      const float4 q = *reinterpret_cast<const float4*>(f32_smem + r * kPitchN + c);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
      return;
    }
    v[0] = v[1] = v[2] = v[3] = 0.f;
    for (int s = 0; s < splits; ++s) {
      float4 q;
      asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "r"(tc::map_to_cta(at, s)) : "memory");
      v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
    }
  };
  const int share = BM / splits, first = rank * share;
  if (GATED) {
    // a thread has eight hidden units of a row
    for (int i = threadIdx.x; i < share * (kUnits / 8); i += kThreads) {
      const int r = first + i / (kUnits / 8), c = i % (kUnits / 8) * 8, col = n0 + c;
      if (r >= rows || c >= cols) continue;
      Eight g, u;
      sum(r, c, g.v);
      sum(r, c + 4, g.v + 4);
      sum(r, kUnits + c, u.v);
      sum(r, kUnits + c + 4, u.v + 4);
      const long long row = (long long)m * p.M + m0 + r;
      if (p.z) {                // (whole groups: the pitch is a multiple of eight)
        float* z = p.z + row * 2 * p.pitch + col;
        store8(z, g);
        store8(z + p.pitch, u);
      }
      if (!p.c) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) g.v[e] = activation<float>(p.activation, g.v[e]) * u.v[e];
      if (p.drop) {
        const dropout::Draw d = dropout::draw_of(p.rule, m);
        const uint32_t in = dropout::kept_bits(p.rule, d, (uint32_t)(m0 + r) * (uint32_t)((p.N + 7) / 8) + (uint32_t)(col / 8));
        const float f = d.on ? d.scale : 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) g.v[e] = (in >> e & 1u) ? f * g.v[e] : 0.f;
      }
      float* h = p.c + row * p.ldc + col;
      if (p.vec_c) {
        store8(h, g);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < cols) h[e] = g.v[e];
      }
    }
  } else {
    for (int i = threadIdx.x; i < share * (kCols / 4); i += kThreads) {
      const int r = first + i / (kCols / 4), c = i % (kCols / 4) * 4;
      if (r >= rows || c >= cols) continue;
      float v[4];
      sum(r, c, v);
      float* to = p.c + m * p.c_member + (m0 + r) * p.ldc + n0 + c;
      if (p.vec_c) {
        *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < cols) to[e] = v[e];
      }
    }
  }
  if (splits > 1) tc::cluster_sync_all();       // no CTA leaves while another reads its sums
}

template <typename S>
__global__ void __launch_bounds__(S::kThreads, S::kPerSm) k_gated_forward_f32(const ProductParams p) {
  pdl_prologue();
  extern __shared__ __align__(16) float f32_smem[];
  const int splits = (int)tc::cluster_size();
  product_tile<S, false, true>(p, f32_smem, blockIdx.x / splits, blockIdx.y, splits, (int)tc::cluster_ctarank());
}
// The CTAs of dx first, then those of dW, a cluster or one for a tile; launched while the kernel that makes dg and du runs.
struct GradientParams {
  ProductParams dx, dw;
  int dx_tiles, dw_tiles, dx_splits, dw_splits, dx_blocks, members;      // tiles of a member; CTAs of a tile (1, or the cluster's); CTAs of all members
  long long blocks;                                              // CTAs that have work (dx's are a whole number of clusters)
};
template <typename SX, typename SW>
struct GradientShape {
  static constexpr int kFloats = SX::kFloats > SW::kFloats ? SX::kFloats : SW::kFloats, kPerSm = SX::kPerSm < SW::kPerSm ? SX::kPerSm : SW::kPerSm;
  static_assert(SX::kThreads == SW::kThreads, "one launch");
};
template <typename SX, typename SW>
__global__ void __launch_bounds__(SX::kThreads, GradientShape<SX, SW>::kPerSm) k_gated_gradients_f32(const GradientParams p) {
  extern __shared__ __align__(16) float f32_smem[];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int rank = (int)tc::cluster_ctarank();
  if ((int)blockIdx.x < p.dx_blocks) {
    const int i = (int)blockIdx.x / p.dx_splits;
    if (i < p.dx_tiles * p.members) product_tile<SX, false, false>(p.dx, f32_smem, i % p.dx_tiles, i / p.dx_tiles, p.dx_splits, p.dx_splits > 1 ? rank : 0);
  } else if (blockIdx.x < p.blocks) {
    const int i = ((int)blockIdx.x - p.dx_blocks) / p.dw_splits;
    if (p.dw_splits == 1) product_tile<SW, true, false>(p.dw, f32_smem, i % p.dw_tiles, i / p.dw_tiles, 1, 0);
    else product_tile<SW, true, false>(p.dw, f32_smem, i % p.dw_tiles, i / p.dw_tiles, p.dw_splits, rank);
  }
}

void fill(const pbt_gated_desc* d, ProductParams* p, bool gated) {
  auto vectors = [&](const void* q, long long ld, long long member) {
    return ((uintptr_t)q & 15) == 0 && ld % 4 == 0 && (d->members == 1 || member % 4 == 0);
  };
  p->vec_a = vectors(p->a, p->lda, p->a_member);
  p->vec_b = vectors(p->b, p->ldb, p->b_member);
  p->vec_c = vectors(p->c, p->ldc, p->c_member) && p->N % (gated ? 8 : 4) == 0;
  const int units = gated ? kCols / 2 : kCols;
  p->tiles_n = (p->N + units - 1) / units;
}
template <typename S>
long long tiles_of(const ProductParams& p) { return (long long)((p.M + S::BM - 1) / S::BM) * p.tiles_n; }
// as many parts of a contraction as there are places for CTAs, two slices each at least
int splits_of(long long tiles, int K, long long places) {
  int splits = 1;
  while (splits < kSplits && tiles * splits * 2 <= places && (K + kK - 1) / kK >= splits * 2 * 2) splits *= 2;
  return splits;
}
// Tall tiles where every SM has one at least
bool tall(const pbt_gated_desc* d, const ProductParams& p) { return p.M > Short::BM && tiles_of<Tall>(p) * d->members >= 148; }

template <typename S>
cudaError_t launch_forward(const pbt_gated_desc* d, const ProductParams& p, cudaStream_t s) {
  static tc::DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = tc::device_setup(&setup, k_gated_forward_f32<S>, S::kFloats * 4, &sms);
  if (e != cudaSuccess) return e;
  const long long tiles = tiles_of<S>(p);
  const int splits = splits_of(tiles * d->members, p.K, (long long)S::kPerSm * sms);
  if (tiles * splits > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
  return launch_clusters(dim3((unsigned)(tiles * splits), (unsigned)d->members), S::kThreads, S::kFloats * 4, splits, false, s, k_gated_forward_f32<S>, p);
}
template <typename SX, typename SW>
cudaError_t launch_gradients(const pbt_gated_desc* d, const ProductParams& dx, const ProductParams& dw, cudaStream_t s) {
  typedef GradientShape<SX, SW> G;
  static tc::DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = tc::device_setup(&setup, k_gated_gradients_f32<SX, SW>, G::kFloats * 4, &sms);
  if (e != cudaSuccess) return e;
  const long long tx = tiles_of<SX>(dx) * d->members, tw = tiles_of<SW>(dw) * d->members, places = (long long)G::kPerSm * sms;
  const int sx = splits_of(tx, dx.K, places), sw = splits_of(tw, dw.K, places), cluster = std::max(sx, sw);
  GradientParams p = {dx, dw, (int)tiles_of<SX>(dx), (int)tiles_of<SW>(dw), sx > 1 ? cluster : 1, sw > 1 ? cluster : 1, 0, d->members, 0};
  const long long first = (tx * p.dx_splits + cluster - 1) / cluster * cluster;
  p.blocks = first + tw * p.dw_splits;
  if (p.blocks + cluster > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
  p.dx_blocks = (int)first;
  return launch_clusters(dim3((unsigned)((p.blocks + cluster - 1) / cluster * cluster)), SX::kThreads, G::kFloats * 4, cluster, true, s, k_gated_gradients_f32<SX, SW>, p);
}

}  // namespace

cudaError_t f32_forward(const pbt_gated_desc* d, float* h, float* z, int pitch, cudaStream_t s) {
  ProductParams p = {};
  p.a = (const float*)d->x; p.lda = d->x_row; p.a_member = d->x_member;
  p.b = (const float*)d->weight; p.ldb = d->weight_row; p.b_member = d->weight_member;
  p.c = h; p.ldc = d->hidden; p.c_member = (long long)d->rows * d->hidden;
  p.M = d->rows; p.N = d->hidden; p.K = d->width;
  p.z = z; p.pitch = pitch;
  p.activation = d->activation; p.drop = d->drop != nullptr;
  if (d->drop) p.rule = dropout::rule_of(*d->drop);
  fill(d, &p, true);
  if (p.M <= Few::BM) return launch_forward<Few>(d, p, s);
  if (p.M <= Half::BM) return launch_forward<Half>(d, p, s);
  return tall(d, p) ? launch_forward<Tall>(d, p, s) : launch_forward<Short>(d, p, s);
}

cudaError_t f32_backward(const pbt_gated_desc* d, const float* dz, int dz_pitch, cudaStream_t s) {
  ProductParams p = {};
  p.a = dz; p.lda = dz_pitch; p.a_member = (long long)d->rows * dz_pitch;
  p.b = (const float*)d->weight; p.ldb = d->weight_row; p.b_member = d->weight_member;
  p.c = (float*)d->dx; p.ldc = d->width; p.c_member = (long long)d->rows * d->width;
  p.M = d->rows; p.N = d->width; p.K = 2 * d->hidden;
  ProductParams dw = p;
  dw.b = (const float*)d->x; dw.ldb = d->x_row; dw.b_member = d->x_member;
  dw.c = (float*)d->dweight; dw.c_member = 2ll * d->hidden * d->width;
  dw.M = 2 * d->hidden; dw.K = d->rows;
  fill(d, &p, false);
  fill(d, &dw, false);
  if (p.M <= Few::BM) return launch_gradients<Few, Short>(d, p, dw, s);
  if (p.M <= Half::BM) return launch_gradients<Half, Short>(d, p, dw, s);
  return tall(d, p) ? launch_gradients<Tall, Tall>(d, p, dw, s) : launch_gradients<Short, Short>(d, p, dw, s);
}

}  // namespace gated
}  // namespace pbt
