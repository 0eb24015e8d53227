// Norms before and after a residual block, fused with the block's gate and residual scale (per member m, row i):
//   v = b rsqrt(mean b^2 + eps),  y = x + c_m sigmoid(z) (v w_post),  u = y rsqrt(mean y^2 + eps) w_next
// and the gradients of all of it.  b is the block's output, y the residual stream, u the next block's input.
//
// Memory-bound: the forward pass reads x, b, z and writes y, u once; the backward pass reads y, b, z, dy, du and writes
// dx, db, dz once.  A row is held in registers by W warps (16-byte vectors where the layout allows them, single
// elements otherwise), so nothing is read twice, and every sum is fp32 or wider.
//
// Backward, with yh = y r_y, dh = du w_next and p = c sigmoid(z) w_post v:
//   t1 = mean(dh yh),  dx = dy + r_y (dh - yh t1),  db = r_b (c g w_post dx - v t2),  t2 = mean(p dx)
// t2 is taken apart as mean(p (dy + r_y dh)) - t1 mean(p r_y yh), so that the row needs ONE reduction of three sums and
// not two that wait for one another.  Column sums (dw_post, dw_next, a per-member gate) stay in the registers of the
// threads that own the columns while a block walks rows of one member; each row group leaves one partial, and a second
// kernel adds the partials in a fixed order (no atomics: reproducible bit for bit).
#include <algorithm>
#include <type_traits>

#include "pbt_common.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace {

constexpr int kNormMaxWidth = 8192;
constexpr int kNormThreads = 256;   // threads of a block, unless one row takes more

struct NormTensor {
  const char* p;
  long long member, row;   // strides in elements
};

struct NormArgs {
  int members, rows, width;
  float eps, inv_width;
  NormTensor x, block, gate, dy, du;
  int gate_vector;
  const float *post_weight, *next_weight, *scale;
  char *y, *u;                       // forward results, contiguous
  float *rstd_block, *rstd_next;     // written by the forward pass, read by the backward pass
  char *dx, *dblock, *dgate;
  float *dpost, *dnext, *dscale;
  float *partial, *partial_scale;    // [members][slices][sums][width], [members][blocks per member]
  int warps_per_row, blocks_per_member, slices, sums;
};

template <typename T, int V> struct Vec;
template <> struct Vec<bf16, 8> {
  typedef uint4 Raw;
  static __device__ __forceinline__ Raw load(const bf16* p) {
    Raw r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
  }
  static __device__ __forceinline__ Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store(bf16* p, const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&t);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Vec<float, 4> {
  typedef float4 Raw;
  static __device__ __forceinline__ Raw load(const float* p) { return ld_stream(p); }
  static __device__ __forceinline__ Raw zero() { return make_float4(0.f, 0.f, 0.f, 0.f); }
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
  static __device__ __forceinline__ void store(float* p, const float* f) { st_stream(p, make_float4(f[0], f[1], f[2], f[3])); }
};
template <> struct Vec<float, 1> {
  typedef float Raw;
  static __device__ __forceinline__ Raw load(const float* p) { return *p; }
  static __device__ __forceinline__ Raw zero() { return 0.f; }
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) { f[0] = r; }
  static __device__ __forceinline__ void store(float* p, const float* f) { *p = f[0]; }
};
template <> struct Vec<bf16, 1> {
  typedef float Raw;
  static __device__ __forceinline__ Raw load(const bf16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ Raw zero() { return 0.f; }
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) { f[0] = r; }
  static __device__ __forceinline__ void store(bf16* p, const float* f) { *p = __float2bfloat16_rn(f[0]); }
};

// V weights (fp32; 16-byte loads where V allows, the launcher has checked the alignment)
template <int V>
__device__ __forceinline__ void load_weights(const float* p, float* f) {
  if constexpr (V == 1) {
    f[0] = __ldg(p);
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const float4 w = __ldg(reinterpret_cast<const float4*>(p + j));
      f[j] = w.x; f[j + 1] = w.y; f[j + 2] = w.z; f[j + 3] = w.w;
    }
  }
}

__device__ __forceinline__ float opened(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

// Sum of N values over the W warps of a row group.  scratch: [2][N][32] floats, used alternately (`turn`), so that one
// barrier per reduction is enough: a buffer is written again only after everybody has passed the next barrier.
template <int N, typename A>
__device__ __forceinline__ void row_sum(A* v, int W, int group, A* scratch, int& turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
  if (W == 1) return;
  const int warp = threadIdx.x >> 5;
  A* buf = scratch + turn * N * 32;
  turn ^= 1;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) buf[k * 32 + warp] = v[k];
  asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(W * 32) : "memory");
#pragma unroll
  for (int k = 0; k < N; ++k) {
    A s = 0;
    for (int w = 0; w < W; ++w) s += buf[k * 32 + group * W + w];
    v[k] = s;
  }
}

template <typename T, int V, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS) k_norm_forward(const NormArgs a) {
  pdl_prologue();
  __shared__ float scratch[2 * 32];
  typedef Vec<T, V> X;
  const int W = a.warps_per_row, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / W, slot = (warp % W) * 32 + lane, step = W * 32;
  const long long r = (long long)blockIdx.x * (blockDim.x / (W * 32)) + group;
  if (r >= (long long)a.members * a.rows) return;
  const int m = (int)(r / a.rows), i = (int)(r % a.rows);
  const int nv = a.width / V;
  int turn = 0;

  typename X::Raw xr[ITEMS], br[ITEMS], zr[ITEMS];
  const T* xp = reinterpret_cast<const T*>(a.x.p) + m * a.x.member + i * a.x.row;
  const T* bp = reinterpret_cast<const T*>(a.block.p) + m * a.block.member + i * a.block.row;
  const T* zp = reinterpret_cast<const T*>(a.gate.p) + m * a.gate.member + i * a.gate.row;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int c = slot + k * step;
    xr[k] = c < nv ? X::load(xp + c * V) : X::zero();
    if (a.block.p) br[k] = c < nv ? X::load(bp + c * V) : X::zero();
    if (a.gate.p) zr[k] = c < nv ? X::load(zp + c * V) : X::zero();
  }
  float y[ITEMS][V];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) X::unpack(xr[k], y[k]);
  const long long at = r * a.width;
  if (a.block.p) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      float b[V];
      X::unpack(br[k], b);
#pragma unroll
      for (int j = 0; j < V; ++j) s[0] = __fmaf_rn(b[j], b[j], s[0]);
    }
    row_sum<1>(s, W, group, scratch, turn);
    const float rb = rsqrtf(s[0] * a.inv_width + a.eps);
    const float crb = rb * (a.scale ? a.scale[m] : 1.f);
    if (a.rstd_block && slot == 0) a.rstd_block[r] = rb;
    const float* wp = a.post_weight + (long long)m * a.width;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int c = slot + k * step;
      if (c >= nv) continue;
      float b[V], z[V], w[V];
      X::unpack(br[k], b);
      load_weights<V>(wp + c * V, w);
      if (a.gate.p) X::unpack(zr[k], z);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float t = b[j] * crb * w[j];
        if (a.gate.p) t *= opened(z[j]);
        y[k][j] += t;
      }
      X::store(reinterpret_cast<T*>(a.y) + at + c * V, y[k]);
    }
  }
  if (a.u) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) s[0] = __fmaf_rn(y[k][j], y[k][j], s[0]);
    row_sum<1>(s, W, group, scratch, turn);
    const float ry = rsqrtf(s[0] * a.inv_width + a.eps);
    if (a.rstd_next && slot == 0) a.rstd_next[r] = ry;
    const float* wn = a.next_weight + (long long)m * a.width;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int c = slot + k * step;
      if (c >= nv) continue;
      float w[V], u[V];
      load_weights<V>(wn + c * V, w);
#pragma unroll
      for (int j = 0; j < V; ++j) u[j] = y[k][j] * ry * w[j];
      X::store(reinterpret_cast<T*>(a.u) + at + c * V, u);
    }
  }
}

// Sums of a row group, in the order in which a partial holds them: next, post, gate (the ones that exist).
// Rows of at most 256 single elements are worked out in fp64 (inputs, results and column sums keep their types): dx and
// db are what is left of dh and dn after the projection on the row is taken away, and in rows of one or two columns
// that is next to nothing, 1 - yh^2 of it, which fp32 loses altogether.
template <typename T, int V, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS) k_norm_backward(const NormArgs a) {
  pdl_prologue();
  typedef typename std::conditional<V == 1 && ITEMS == 1, double, float>::type A;
  __shared__ A scratch[2 * 3 * 32];
  __shared__ float scale_sum[32];
  typedef Vec<T, V> X;
  const int W = a.warps_per_row, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int groups = blockDim.x / (W * 32), group = warp / W, slot = (warp % W) * 32 + lane, step = W * 32;
  const int m = blockIdx.x / a.blocks_per_member, s = blockIdx.x % a.blocks_per_member;
  const int nv = a.width / V;
  const bool next = a.du.p != nullptr, block = a.block.p != nullptr, gate = a.gate.p != nullptr;
  const float c = a.scale ? a.scale[m] : 1.f;
  const float* wn = a.next_weight + (long long)m * a.width;
  const float* wp = a.post_weight + (long long)m * a.width;
  float acc_next[ITEMS][V], acc_post[ITEMS][V], acc_gate[ITEMS][V], acc_scale = 0.f;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) acc_next[k][j] = acc_post[k][j] = acc_gate[k][j] = 0.f;
  int turn = 0;
  for (int i = s * groups + group; i < a.rows; i += a.blocks_per_member * groups) {
    const long long r = (long long)m * a.rows + i, at = r * a.width;
    typename X::Raw yr[ITEMS], br[ITEMS], zr[ITEMS], dyr[ITEMS], dur[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = slot + k * step;
      const bool in = e < nv;
      dyr[k] = in && a.dy.p ? X::load(reinterpret_cast<const T*>(a.dy.p) + m * a.dy.member + i * a.dy.row + e * V) : X::zero();
      if (next) {
        yr[k] = in ? X::load(reinterpret_cast<const T*>(a.x.p) + m * a.x.member + i * a.x.row + e * V) : X::zero();
        dur[k] = in ? X::load(reinterpret_cast<const T*>(a.du.p) + m * a.du.member + i * a.du.row + e * V) : X::zero();
      }
      if (block) br[k] = in ? X::load(reinterpret_cast<const T*>(a.block.p) + m * a.block.member + i * a.block.row + e * V) : X::zero();
      if (gate) zr[k] = in ? X::load(reinterpret_cast<const T*>(a.gate.p) + m * a.gate.member + i * a.gate.row + e * V) : X::zero();
    }
    const A ry = next ? a.rstd_next[r] : 0.f, rb = block ? a.rstd_block[r] : 0.f;
    A sums[3] = {0, 0, 0};   // dh yh, p (dy + r_y dh), p r_y yh
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = slot + k * step;
      if (e >= nv) continue;
      float dy[V], du[V], y[V], b[V], z[V], w[V], q[V];
      X::unpack(dyr[k], dy);
      if (next) {
        X::unpack(dur[k], du);
        X::unpack(yr[k], y);
        load_weights<V>(wn + e * V, w);
      }
      if (block) {
        X::unpack(br[k], b);
        load_weights<V>(wp + e * V, q);
        if (gate) X::unpack(zr[k], z);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        A dh = 0, yh = 0;
        if (next) {
          dh = (A)du[j] * w[j];
          yh = y[j] * ry;
          sums[0] += dh * yh;
        }
        if (block) {
          A p = (A)c * q[j] * (b[j] * rb);
          if (gate) p *= opened(z[j]);
          sums[1] += p * (ry * dh + dy[j]);
          sums[2] += p * (ry * yh);
        }
      }
    }
    row_sum<3>(sums, W, group, scratch, turn);
    const A t1 = sums[0] / a.width, t2 = (sums[1] - t1 * sums[2]) / a.width;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = slot + k * step;
      if (e >= nv) continue;
      float dy[V];
      A dx[V];
      X::unpack(dyr[k], dy);
#pragma unroll
      for (int j = 0; j < V; ++j) dx[j] = dy[j];
      if (next) {
        float du[V], y[V], w[V];
        X::unpack(dur[k], du);
        X::unpack(yr[k], y);
        load_weights<V>(wn + e * V, w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const A yh = y[j] * ry;
          acc_next[k][j] += (float)(du[j] * yh);
          dx[j] += ry * ((A)du[j] * w[j] - yh * t1);
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) dy[j] = (float)dx[j];
      X::store(reinterpret_cast<T*>(a.dx) + at + e * V, dy);
      if (block) {
        float b[V], z[V], q[V], db[V], dz[V];
        X::unpack(br[k], b);
        load_weights<V>(wp + e * V, q);
        if (gate) X::unpack(zr[k], z);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const A g = gate ? opened(z[j]) : 1.f, v = b[j] * rb, gdx = g * dx[j];
          const A dn = c * gdx, o = gdx * v * q[j];
          acc_post[k][j] += (float)(dn * v);
          acc_scale += (float)o;
          db[j] = (float)(rb * (dn * q[j] - v * t2));
          dz[j] = (float)(c * o * (1 - g));
        }
        X::store(reinterpret_cast<T*>(a.dblock) + at + e * V, db);
        if (gate && a.gate_vector) {
#pragma unroll
          for (int j = 0; j < V; ++j) acc_gate[k][j] += dz[j];
        } else if (gate) {
          X::store(reinterpret_cast<T*>(a.dgate) + at + e * V, dz);
        }
      }
    }
  }
  float* out = a.partial + ((long long)m * a.slices + s * groups + group) * a.sums * a.width;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int e = slot + k * step;
    if (e >= nv) continue;
    float* o = out;
    if (next) { 
#pragma unroll
      for (int j = 0; j < V; ++j) o[e * V + j] = acc_next[k][j];
      o += a.width;
    }
    if (block) {
#pragma unroll
      for (int j = 0; j < V; ++j) o[e * V + j] = acc_post[k][j];
      o += a.width;
    }
    if (gate && a.gate_vector) {
#pragma unroll
      for (int j = 0; j < V; ++j) o[e * V + j] = acc_gate[k][j];
    }
  }
  if (block) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc_scale += __shfl_xor_sync(0xFFFFFFFFu, acc_scale, o);
    if (lane == 0) scale_sum[warp] = acc_scale;
    __syncthreads();
    if (threadIdx.x == 0) {
      float t = 0.f;
      for (int w = 0; w < (int)(blockDim.x >> 5); ++w) t += scale_sum[w];
      a.partial_scale[blockIdx.x] = t;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) k_norm_columns(const NormArgs a) {
  pdl_prologue();
  const int m = blockIdx.y, e = blockIdx.x * 256 + threadIdx.x;
  const bool next = a.du.p != nullptr, block = a.block.p != nullptr;
  if (e < a.width) {
    const float* p = a.partial + (long long)m * a.slices * a.sums * a.width + e;
    for (int q = 0; q < a.sums; ++q) {
      float t = 0.f;
      for (int s = 0; s < a.slices; ++s) t += p[((long long)s * a.sums + q) * a.width];
      const long long at = (long long)m * a.width + e;
      if (next && q == 0) a.dnext[at] = t;
      else if (q == (next ? 1 : 0)) a.dpost[at] = t;
      else Vec<T, 1>::store(reinterpret_cast<T*>(a.dgate) + at, &t);
    }
  }
  if (block && blockIdx.x == 0 && threadIdx.x == 0 && a.dscale) {
    float t = 0.f;
    for (int s = 0; s < a.blocks_per_member; ++s) t += a.partial_scale[m * a.blocks_per_member + s];
    a.dscale[m] = t;
  }
}

int norm_fail(int code, const char* msg) {
  set_last_error(msg);
  return code;
}

// Elements per vector: 16-byte vectors if the width and every pointer and stride allow them, single elements otherwise.
int norm_vector(const pbt_block_norm_desc* d, bool backward) {
  const int v = d->dtype ? 8 : 4;
  if (d->width % v) return 1;
  const int esz = d->dtype ? 2 : 4;
  bool ok = true;
  auto in = [&](const void* p, int64_t member, int64_t row) {
    if (p) ok = ok && ((uintptr_t)p & 15) == 0 && (member * esz) % 16 == 0 && (row * esz) % 16 == 0;
  };
  auto flat = [&](const void* p) { if (p) ok = ok && ((uintptr_t)p & 15) == 0; };
  in(d->x, d->x_member, d->x_row);
  in(d->block, d->block_member, d->block_row);
  in(d->gate, d->gate_member, d->gate_row);
  flat(d->post_weight);
  flat(d->next_weight);
  if (backward) {
    in(d->dy, d->dy_member, d->dy_row);
    in(d->du, d->du_member, d->du_row);
    flat(d->dx); flat(d->dblock); flat(d->dgate);
  } else {
    flat(d->y); flat(d->u);
  }
  return ok ? v : 1;
}

int norm_check(const pbt_block_norm_desc* d) {
  if (!d) return norm_fail(PBT_ERR_INVALID_ARG, "desc is NULL");
  if (d->members < 1 || d->rows < 0 || d->width < 1) return norm_fail(PBT_ERR_INVALID_ARG, "members and width must be positive, rows >= 0");
  if (d->dtype != 0 && d->dtype != 1) return norm_fail(PBT_ERR_UNSUPPORTED, "activations are float or bfloat16");
  if (d->width > kNormMaxWidth) return norm_fail(PBT_ERR_UNSUPPORTED, "width is larger than 8192");
  if (d->members > 65535) return norm_fail(PBT_ERR_UNSUPPORTED, "more than 65535 members");
  if (d->gate && !d->block) return norm_fail(PBT_ERR_INVALID_ARG, "a gate needs a block output");
  if (d->block && !d->post_weight) return norm_fail(PBT_ERR_INVALID_ARG, "a block output needs post_weight");
  if (!(d->eps >= 0.f)) return norm_fail(PBT_ERR_INVALID_ARG, "eps must be >= 0");
  return PBT_OK;
}

void norm_fill(NormArgs* a, const pbt_block_norm_desc* d) {
  memset(a, 0, sizeof(*a));
  a->members = d->members; a->rows = d->rows; a->width = d->width;
  a->eps = d->eps; a->inv_width = 1.f / (float)d->width;
  a->x = {(const char*)d->x, d->x_member, d->x_row};
  a->block = {(const char*)d->block, d->block_member, d->block_row};
  a->gate = {(const char*)d->gate, d->gate_member, d->gate_vector ? 0 : d->gate_row};
  a->dy = {(const char*)d->dy, d->dy_member, d->dy_row};
  a->du = {(const char*)d->du, d->du_member, d->du_row};
  a->gate_vector = d->gate_vector;
  a->post_weight = d->post_weight; a->next_weight = d->next_weight; a->scale = d->scale;
  a->y = (char*)d->y; a->u = (char*)d->u; a->rstd_block = d->rstd_block; a->rstd_next = d->rstd_next;
  a->dx = (char*)d->dx; a->dblock = (char*)d->dblock; a->dgate = (char*)d->dgate;
  a->dpost = d->dpost_weight; a->dnext = d->dnext_weight; a->dscale = d->dscale;
}

// Warps of a row and rows of a block for `items` vectors per thread.
void norm_shape(int width, int v, int items, int* warps, int* groups) {
  const int nv = width / v;
  *warps = std::max(1, (nv + items * 32 - 1) / (items * 32));
  *groups = std::max(1, kNormThreads / 32 / *warps);
}

// Most vectors per thread.  Forward: a row of 8192 fits eight warps (single elements: 32).  Backward: the three column
// sums of every element live in registers too, so a thread holds at most 16 elements and the widest rows take 16 warps.
constexpr int norm_most(int v, bool backward) { return v == 1 ? 8 : !backward ? (v == 4 ? 8 : 4) : v == 4 ? 4 : 2; }

// Vectors per thread: the smallest choice with at most eight warps per row, or the most there are.
int norm_items(int width, int v, bool backward) {
  const int nv = width / v, most = norm_most(v, backward);
  int items = 1;
  while (items < most && nv > items * 32 * 8) items *= 2;
  return items;
}

struct NormPlan { int v, items, warps, groups, blocks_per_member, slices, sums; size_t bytes; };

NormPlan norm_backward_plan(const pbt_block_norm_desc* d) {
  NormPlan p;
  p.v = norm_vector(d, true);
  p.items = norm_items(d->width, p.v, true);
  norm_shape(d->width, p.v, p.items, &p.warps, &p.groups);
  const int want = (2 * 148 + d->members - 1) / d->members;   // two blocks per SM over all members
  p.blocks_per_member = std::max(1, std::min(want, (d->rows + p.groups - 1) / p.groups));
  p.slices = p.blocks_per_member * p.groups;
  p.sums = (d->du ? 1 : 0) + (d->block ? 1 : 0) + (d->gate && d->gate_vector ? 1 : 0);
  p.bytes = ((size_t)d->members * p.slices * p.sums * d->width + (size_t)d->members * p.blocks_per_member) * sizeof(float);
  p.bytes = (p.bytes + 255) & ~(size_t)255;
  return p;
}

template <typename T, int V, int ITEMS>
cudaError_t launch_norm_items(bool backward, unsigned grid, int threads, const NormArgs& a, cudaStream_t s) {
  auto l = launch_with(grid, threads, 0, s);
  if (threads > kNormThreads) {
    // more than eight warps per row: the widest rows only
    if constexpr (V == 1 && ITEMS == norm_most(V, false))
      if (!backward) return l(k_norm_forward<T, V, ITEMS, 1024>, a);
    if constexpr (ITEMS == norm_most(V, true))
      if (backward) return l(k_norm_backward<T, V, ITEMS, (V == 1 ? 1024 : 512)>, a);
    return cudaErrorInvalidValue;
  }
  if constexpr (ITEMS <= norm_most(V, true))
    if (backward) return l(k_norm_backward<T, V, ITEMS, kNormThreads>, a);
  if constexpr (ITEMS <= norm_most(V, false))
    if (!backward) return l(k_norm_forward<T, V, ITEMS, kNormThreads>, a);
  return cudaErrorInvalidValue;
}
template <typename T, int V>
cudaError_t launch_norm(bool backward, int items, unsigned grid, int threads, const NormArgs& a, cudaStream_t s) {
  switch (items) {
    case 1: return launch_norm_items<T, V, 1>(backward, grid, threads, a, s);
    case 2: return launch_norm_items<T, V, 2>(backward, grid, threads, a, s);
    case 4: return launch_norm_items<T, V, 4>(backward, grid, threads, a, s);
    default: return launch_norm_items<T, V, 8>(backward, grid, threads, a, s);
  }
}
cudaError_t launch_norm(bool bf, int v, bool backward, int items, unsigned grid, int threads, const NormArgs& a, cudaStream_t s) {
  if (bf) return v == 1 ? launch_norm<bf16, 1>(backward, items, grid, threads, a, s) : launch_norm<bf16, 8>(backward, items, grid, threads, a, s);
  return v == 1 ? launch_norm<float, 1>(backward, items, grid, threads, a, s) : launch_norm<float, 4>(backward, items, grid, threads, a, s);
}

}  // namespace
}  // namespace pbt

extern "C" int pbt_block_norm_forward(const pbt_block_norm_desc* d, void* stream) {
  using namespace pbt;
  const int rc = norm_check(d);
  if (rc) return rc;
  if (!d->x && d->rows) return norm_fail(PBT_ERR_INVALID_ARG, "x is NULL");
  if (d->block && !d->y && d->rows) return norm_fail(PBT_ERR_INVALID_ARG, "y is NULL");
  if (d->u && !d->next_weight) return norm_fail(PBT_ERR_INVALID_ARG, "u needs next_weight");
  if (!d->block && !d->u && d->rows) return norm_fail(PBT_ERR_INVALID_ARG, "nothing to compute: neither a block output nor a next norm");
  if (!d->rows) return PBT_OK;
  NormArgs a;
  norm_fill(&a, d);
  const int v = norm_vector(d, false);
  const int items = norm_items(d->width, v, false);
  int groups = 1;
  norm_shape(d->width, v, items, &a.warps_per_row, &groups);
  const long long rows = (long long)d->members * d->rows, blocks = (rows + groups - 1) / groups;
  if (blocks > 0x7FFFFFFFll) return norm_fail(PBT_ERR_UNSUPPORTED, "too many rows");
  const int threads = groups * a.warps_per_row * 32;
  const cudaError_t e = launch_norm(d->dtype == 1, v, false, items, (unsigned)blocks, threads, a, (cudaStream_t)stream);
  if (e != cudaSuccess) return norm_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
  return PBT_OK;
}

extern "C" int pbt_block_norm_query_workspace(const pbt_block_norm_desc* d, size_t* bytes) {
  using namespace pbt;
  if (!bytes) return norm_fail(PBT_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = norm_check(d);
  if (rc) return rc;
  *bytes = norm_backward_plan(d).bytes;
  return PBT_OK;
}

extern "C" int pbt_block_norm_backward(const pbt_block_norm_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace pbt;
  const int rc = norm_check(d);
  if (rc) return rc;
  if (!d->du && !d->block) return norm_fail(PBT_ERR_INVALID_ARG, "nothing to differentiate: neither du nor a block output");
  if (d->du && (!d->next_weight || !d->dnext_weight)) return norm_fail(PBT_ERR_INVALID_ARG, "du needs next_weight and dnext_weight");
  if (d->block && !d->dpost_weight) return norm_fail(PBT_ERR_INVALID_ARG, "a block output needs dpost_weight");
  if (d->gate && !d->dgate && (d->rows || d->gate_vector)) return norm_fail(PBT_ERR_INVALID_ARG, "a gate needs dgate");
  if (d->rows && ((d->du && (!d->x || !d->rstd_next)) || (d->block && (!d->dblock || !d->rstd_block)) || !d->dx))
    return norm_fail(PBT_ERR_INVALID_ARG, "y, dx, dblock or a reciprocal root is NULL");
  const NormPlan p = norm_backward_plan(d);
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < p.bytes)
    return norm_fail(PBT_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than pbt_block_norm_query_workspace says");
  NormArgs a;
  norm_fill(&a, d);
  a.warps_per_row = p.warps; a.blocks_per_member = p.blocks_per_member; a.slices = p.slices; a.sums = p.sums;
  a.partial = (float*)workspace;
  a.partial_scale = a.partial + (long long)d->members * p.slices * p.sums * d->width;
  const unsigned grid = (unsigned)d->members * p.blocks_per_member;
  const int threads = p.groups * p.warps * 32;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e = launch_norm(d->dtype == 1, p.v, true, p.items, grid, threads, a, s);
  if (e == cudaSuccess) {
    auto l = launch_with(dim3((d->width + 255) / 256, d->members), 256, 0, s);
    e = d->dtype ? l(k_norm_columns<bf16>, a) : l(k_norm_columns<float>, a);
  }
  if (e != cudaSuccess) return norm_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
  return PBT_OK;
}
