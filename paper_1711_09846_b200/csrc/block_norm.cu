// Norms before and after a residual block, fused with the block's gate and residual scale (per member m, row i):
//   v = b rsqrt(mean b^2 + eps),  y = x + c_m sigmoid(z) (v w_post),  u = y rsqrt(mean y^2 + eps) w_next
// and the gradients of all of it.  b is the block's output, y the residual stream, u the next block's input.
//
// Memory-bound: the forward pass reads x, b, z and writes y, u once; the backward pass reads y, b, z, dy, du and writes
// dx, db, dz once.  With five streams in and three out the instructions are as long as the transfers, so they are kept
// few: several elements a thread, so that a row's reductions and addresses are shared by many, running pointers, and the
// rows on their way to shared memory (cp.async) while earlier ones are worked on.  (Packed fp32 pairs, fma.rn.f32x2, did
// not pay: 297 us against 275 for the backward pass of 80 x 512 x 2048, the moves into register pairs cost more than the
// halved arithmetic.)  Every sum is fp32 or wider.
//
// Backward, with yh = y r_y, dh = du w_next and p = sigmoid(z) w_post v:
//   t1 = mean(dh yh),  dx = dy + r_y (dh - yh t1),  db = r_b (c g w_post dx - c v t2),  t2 = mean(p dx)
// t2 is taken apart as mean(p (dy + r_y dh)) - r_y t1 mean(p yh), so that the row needs ONE reduction of three sums and
// not two that wait for one another.
//
// Work is dealt in consecutive rows, whatever the members: every row group (the warps of a row) gets the same number of
// rows, to within one.  Column sums (dw_post, dw_next, a per-member gate) stay in the registers of the threads that own
// the columns and are left as one partial result per (row group, member); a second kernel adds a member's partial results
// in a fixed order (no atomics: reproducible bit for bit).
#include <algorithm>
#include <type_traits>

#include "tc_common.cuh"

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
  float *partial, *partial_scale;    // [row groups + members][sums][width], [row groups + members][warps of a row]
  int warps_per_row, groups, sums;   // groups: row groups of the grid
};

// first row (of all members' rows, one after the other) of row group g
__device__ __forceinline__ long long norm_first_row(const NormArgs& a, int g) { return (long long)a.members * a.rows * g / a.groups; }
// the row group that has row r: the last one whose first row is not behind r
__device__ __forceinline__ int norm_group_of(const NormArgs& a, long long r) {
  return (int)(((r + 1) * a.groups - 1) / ((long long)a.members * a.rows));
}

// sigmoid(z) = 1 / (1 + 2^(-z log2 e)) by the special-function unit: relative error below (|z| + 3) 2^-22 for z >= -87; below that
// the result, less than 2^-125, may be 0
__device__ __forceinline__ float opened(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.44269504f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
// sigmoid(z) and 1 - sigmoid(z) for the backward pass, both with the error above for |z| <= 87, beyond which the smaller may be 0.  (1 minus a
// rounded sigmoid is off by 6 % at z = 16 and 0 from 17 on: a gate that is open would have no gradient.)
// BOTH: two numbers, e / (1 + e) being the second one; e is held to 2^127, whose reciprocal is 0, so that a closed gate is exactly closed.
// Else one, the smaller of the two with the sign of z: 1 minus it is the other one without cancellation.  Two registers an element pay where
// the weights of the next norm make room for them: 19 x 231 x 2048 bf16 45 us, with one 49; 19 x 231 x 2048 fp32, which keeps those weights,
// 61 us, with one 58.
template <bool BOTH> struct GateParts {
  float o, c;
  __device__ __forceinline__ void of(float z) {
    float t, e;
    asm("min.NaN.f32 %0, %1, 0f42FE0000;" : "=f"(t) : "f"(z * -1.44269504f));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(o) : "f"(1.f + e));
    c = e * o;
  }
  __device__ __forceinline__ void none() { o = 1.f; c = 0.f; }
  template <typename A> __device__ __forceinline__ A open() const { return o; }
  template <typename A> __device__ __forceinline__ A closed() const { return c; }
};
template <> struct GateParts<false> {
  float smaller;
  __device__ __forceinline__ void of(float z) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(z) * -1.44269504f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    smaller = copysignf(e * r, z);
  }
  __device__ __forceinline__ void none() { smaller = 0.f; }
  __device__ __forceinline__ bool negative() const { return __float_as_int(smaller) < 0; }      // (-0 is)
  template <typename A> __device__ __forceinline__ A open() const { return negative() ? -(A)smaller : 1 - (A)smaller; }
  template <typename A> __device__ __forceinline__ A closed() const { return negative() ? 1 + (A)smaller : (A)smaller; }
};

// V elements of type T as they lie in memory, and as values of type L (float; double for V == 1).
template <typename T, int V> struct Vec;
template <> struct Vec<bf16, 8> {
  typedef uint4 Raw;
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
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
  static __device__ __forceinline__ void store(float* p, const float* f) { st_stream(p, make_float4(f[0], f[1], f[2], f[3])); }
};
template <> struct Vec<float, 1> {
  typedef float Raw;
  static __device__ __forceinline__ Raw load(const float* p) { return *p; }
  template <typename L> static __device__ __forceinline__ void unpack(const Raw& r, L* f) { f[0] = r; }
  template <typename L> static __device__ __forceinline__ void store(float* p, const L* f) { *p = (float)f[0]; }
};
template <> struct Vec<bf16, 1> {
  typedef float Raw;
  static __device__ __forceinline__ Raw load(const bf16* p) { return __bfloat162float(*p); }
  template <typename L> static __device__ __forceinline__ void unpack(const Raw& r, L* f) { f[0] = r; }
  template <typename L> static __device__ __forceinline__ void store(bf16* p, const L* f) { *p = __float2bfloat16_rn((float)f[0]); }
};

template <> struct Vec<float, 2> {
  typedef float2 Raw;
  static __device__ __forceinline__ Raw load(const float* p) { return *reinterpret_cast<const float2*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) { f[0] = r.x; f[1] = r.y; }
  static __device__ __forceinline__ void store(float* p, const float* f) { *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]); }
};
template <> struct Vec<bf16, 2> {
  typedef uint32_t Raw;
  static __device__ __forceinline__ Raw load(const bf16* p) { return *reinterpret_cast<const uint32_t*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) { f[0] = __uint_as_float(r << 16); f[1] = __uint_as_float(r & 0xFFFF0000u); }
  static __device__ __forceinline__ void store(bf16* p, const float* f) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(f[0], f[1]); }
};

// V weights (fp32; 16-byte loads where V allows, the launcher has checked the alignment)
template <int V, typename L>
__device__ __forceinline__ void load_weights(const float* p, L* f) {
  if constexpr (V == 1) {
    f[0] = __ldg(p);
  } else if constexpr (V == 2) {
    const float2 w = __ldg(reinterpret_cast<const float2*>(p));
    f[0] = w.x; f[1] = w.y;
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const float4 w = __ldg(reinterpret_cast<const float4*>(p + j));
      f[j] = w.x; f[j + 1] = w.y; f[j + 2] = w.z; f[j + 3] = w.w;
    }
  }
}

// Sum of a value over the W warps of a row group.  scratch: [2][32], used alternately (`turn`), so that one barrier per
// reduction is enough: a buffer is written again only after everybody has passed the next barrier.
__device__ __forceinline__ float row_sum(float v, int W, int group, float* scratch, int& turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if (W == 1) return v;
  const int warp = threadIdx.x >> 5;
  float* buf = scratch + turn * 32;
  turn ^= 1;
  if ((threadIdx.x & 31) == 0) buf[warp] = v;
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(W * 32) : "memory");
  v = 0.f;
  for (int w = 0; w < W; ++w) v += buf[group * W + w];
  return v;
}

// The same for the backward pass's three sums (at most 16 warps).  The three are folded into one register on the way: after
// the first exchange the halves of a warp go on with different sums, after the second its quarters, so that a warp needs
// 6 shuffles and not 15; across warps the lanes read one partial sum each.  scratch: [2][64].
template <typename A>
__device__ __forceinline__ void row_sum3(A* v, int W, int group, A* scratch, int& turn) {
  const unsigned all_lanes = 0xFFFFFFFFu;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool hi = lane & 16, odd = lane & 8;
  A a = hi ? v[2] : v[0], b = hi ? (A)0 : v[1];
  a += __shfl_xor_sync(all_lanes, hi ? v[0] : v[2], 16);
  b += __shfl_xor_sync(all_lanes, hi ? v[1] : (A)0, 16);
  A s = odd ? b : a;
  s += __shfl_xor_sync(all_lanes, odd ? a : b, 8);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(all_lanes, s, o);
  // sum 0 is in lanes 0..7, sum 1 in 8..15, sum 2 in 16..23
  if (W > 1) {
    A* buf = scratch + turn * 64;
    turn ^= 1;
    if ((lane & 7) == 0) buf[warp * 4 + (lane >> 3)] = s;
    __syncwarp();
    asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(W * 32) : "memory");
    const A* mine = buf + group * W * 4;
    s = lane < 4 * W ? mine[lane] : (A)0;
    if (W > 8 && lane + 32 < 4 * W) s += mine[lane + 32];
#pragma unroll
    for (int o = 16; o > 2; o >>= 1) s += __shfl_xor_sync(all_lanes, s, o);
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] = __shfl_sync(all_lanes, s, k);
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) v[k] = __shfl_sync(all_lanes, s, 8 * k);
}

// Rows on their way from global memory to shared memory.
//
// Aligned rows (V > 2): a thread copies its own 16-byte vectors into its own slots, several rows ahead of the one it works
// on, and reads nobody else's, so that the ring needs no barrier.
// Other rows (V <= 2: pairs or single elements): the row group copies the 16-byte granules that the row touches, one row at
// a time, and reads them at the row's offset in them, so these need a barrier on either side of a row; the
// other row groups of the SM have theirs in flight meanwhile.  (A granule that holds a byte of the row lies in the same page
// as that byte.)
__device__ __forceinline__ void copy_ahead(void* slot, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(slot)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// bytes that the granules of an unaligned row of `width` elements can take
template <typename T>
__host__ __device__ __forceinline__ int norm_pitch(int width) { return (width * (int)sizeof(T) + 31) / 16 * 16; }

template <typename T, int V, int ITEMS, int ARRAYS, int STAGES, int THREADS>
struct RowRing {
  typedef typename Vec<T, V>::Raw Raw;
  uint4* slots;                  // this thread's (V > 2; its vectors are THREADS apart) or this row group's (V <= 2)
  const T* p[ARRAYS];            // the next row to ask for, at this thread's first vector (V <= 2: at its first element)
  long long row[ARRAYS], wrap[ARRAYS];   // to the next row, and from behind a member's last row to the next member's first
  int shift[ARRAYS];             // V <= 2: bytes between the first granule and the row that is staged
  bool have[ARRAYS];
  int slot, step, nv, rows, group;
  int pitch;                     // V <= 2: bytes of an array's row in shared memory
  int i, left;                   // the next row within its member, and how many there are to ask for

  __device__ __forceinline__ void set(int k, const NormTensor& t, bool used, int m) {
    p[k] = reinterpret_cast<const T*>(t.p) + m * t.member + i * t.row + (V > 2 ? slot * V : 0);
    row[k] = t.row;
    wrap[k] = t.member - rows * t.row;
    have[k] = used;
  }
  __device__ __forceinline__ uint4* at(int s, int k, int j) const { return slots + s * (ARRAYS * ITEMS * THREADS) + (k * ITEMS + j) * THREADS; }
  __device__ __forceinline__ char* staged(int k) const { return reinterpret_cast<char*>(slots) + k * pitch; }
  __device__ __forceinline__ void barrier() const {
    if (step == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(step) : "memory");
  }
  // ask for the next row (for nothing behind the last one) into stage s
  __device__ __forceinline__ void ask(int s) {
    if constexpr (V <= 2) barrier();     // everybody has read the row before
    if (left > 0) {
      const bool last = ++i == rows;
      if (last) i = 0;
      --left;
#pragma unroll
      for (int k = 0; k < ARRAYS; ++k)
        if (have[k]) {
          if constexpr (V > 2) {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j)
              if (slot + j * step < nv) copy_ahead(at(s, k, j), p[k] + j * (step * V));
          } else {
            shift[k] = (int)((uintptr_t)p[k] & 15);
            const int n = (shift[k] + nv * V * (int)sizeof(T) + 15) / 16;
            const char* from = reinterpret_cast<const char*>(p[k]) - shift[k];
            for (int e = slot; e < n; e += step) copy_ahead(staged(k) + e * 16, from + e * 16);
          }
          p[k] += row[k];
          if (last) p[k] += wrap[k];
        }
    }
    copy_commit();
  }
  // the oldest row asked for has arrived
  __device__ __forceinline__ void wait() const {
    copy_wait<STAGES - 1>();
    if constexpr (V <= 2) barrier();
  }
  // vector j of array k (which there is) of the oldest row, in stage s; the vector lies inside the row
  template <typename L>
  __device__ __forceinline__ void get(int s, int k, int j, L* f) const {
    if constexpr (V > 2) Vec<T, V>::unpack(*reinterpret_cast<const Raw*>(at(s, k, j)), f);
    else Vec<T, V>::unpack(Vec<T, V>::load(reinterpret_cast<const T*>(staged(k) + shift[k]) + (slot + j * step) * V), f);
  }
};

// Stages of a ring: what fits the block's share of an SM's shared memory (four forward blocks of 256 threads, two backward
// ones, or one of 512), at most three (a row that is worked on and two on their way).
template <int V, int ITEMS, int ARRAYS, int THREADS>
__host__ __device__ constexpr int norm_stages() {
  const int fit = (THREADS > kNormThreads ? 160 : ARRAYS == 3 ? 50 : 100) * 1024 / (ARRAYS * ITEMS * 16 * THREADS);
  return V <= 2 || fit < 1 ? 1 : fit > 3 ? 3 : fit;
}

template <typename T, int V, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS <= kNormThreads ? 4 : 1) k_norm_forward(const NormArgs a) {
  pdl_prologue();
  extern __shared__ uint4 norm_ring[];
  __shared__ float scratch[2 * 32];
  typedef Vec<T, V> X;
  constexpr int kStages = norm_stages<V, ITEMS, 3, THREADS>();
  const int W = a.warps_per_row, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / W, g = blockIdx.x * (blockDim.x / (W * 32)) + group;
  if (g >= a.groups) return;
  const bool block = a.block.p != nullptr, gate = a.gate.p != nullptr, next = a.u != nullptr;
  long long r = norm_first_row(a, g);
  const long long r_end = norm_first_row(a, g + 1);
  int m = (int)(r / a.rows), i = (int)(r % a.rows);
  RowRing<T, V, ITEMS, 3, kStages, THREADS> ring;
  ring.slot = (warp % W) * 32 + lane; ring.step = W * 32; ring.nv = a.width / V; ring.rows = a.rows; ring.group = group;
  ring.pitch = norm_pitch<T>(a.width);
  ring.slots = V > 2 ? norm_ring + threadIdx.x : norm_ring + group * (3 * ring.pitch / 16);
  ring.i = i; ring.left = (int)(r_end - r);
  ring.set(0, a.x, true, m); ring.set(1, a.block, block, m); ring.set(2, a.gate, gate, m);
#pragma unroll
  for (int s = 0; s < kStages; ++s) ring.ask(s);
  const int first = ring.slot * V, far = ring.step * V;      // this thread's first element and the distance to its next vector
  const float* wp = a.post_weight + (long long)m * a.width + first;
  const float* wn = a.next_weight + (long long)m * a.width + first;
  T* yp = reinterpret_cast<T*>(a.y) + r * a.width + first;
  T* up = reinterpret_cast<T*>(a.u) + r * a.width + first;
  float c = a.scale && block ? a.scale[m] : 1.f;
  int turn = 0, stage = 0;
  for (; r < r_end; ++r, yp += a.width, up += a.width) {
    ring.wait();
    float y[ITEMS][V];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      if (ring.slot + k * ring.step < ring.nv) {
        ring.get(stage, 0, k, y[k]);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) y[k][j] = 0.f;
      }
    }
    if (block) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        if (ring.slot + k * ring.step >= ring.nv) continue;
        float b[V];
        ring.get(stage, 1, k, b);
#pragma unroll
        for (int j = 0; j < V; ++j) s = __fmaf_rn(b[j], b[j], s);
      }
      const float rb = rsqrtf(row_sum(s, W, group, scratch, turn) * a.inv_width + a.eps);
      const float crb = c * rb;
      if (a.rstd_block && ring.slot == 0) a.rstd_block[r] = rb;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        if (ring.slot + k * ring.step >= ring.nv) continue;
        float b[V], w[V];
        ring.get(stage, 1, k, b);
        load_weights<V>(wp + k * far, w);
#pragma unroll
        for (int j = 0; j < V; ++j) b[j] = b[j] * crb * w[j];
        if (gate) {
          float z[V];
          ring.get(stage, 2, k, z);
#pragma unroll
          for (int j = 0; j < V; ++j) y[k][j] = __fmaf_rn(b[j], opened(z[j]), y[k][j]);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) y[k][j] += b[j];
        }
        X::store(yp + k * far, y[k]);
      }
    }
    ring.ask(stage);
    if (++stage == kStages) stage = 0;
    if (next) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) s = __fmaf_rn(y[k][j], y[k][j], s);
      const float ry = rsqrtf(row_sum(s, W, group, scratch, turn) * a.inv_width + a.eps);
      if (a.rstd_next && ring.slot == 0) a.rstd_next[r] = ry;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        if (ring.slot + k * ring.step >= ring.nv) continue;
        float w[V];
        load_weights<V>(wn + k * far, w);
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] *= y[k][j] * ry;
        X::store(up + k * far, w);
      }
    }
    if (++i == a.rows && r + 1 < r_end) {
      i = 0;
      ++m;
      wp += a.width;
      wn += a.width;
      if (a.scale && block) c = a.scale[m];
    }
  }
}

// Sums of a row group, in the order in which a partial result holds them: next, post, gate (the ones that exist).
// Up to 8 elements a thread, what the first pass over a row works out stays in registers for the second; the widest
// rows (16 elements a thread, whose column sums fill the registers) read the row from shared memory twice.
// Rows of at most 32 single elements are worked out in fp64 (inputs, results and column sums keep their types): dx and
// db are what is left of dh and dn after the projection on the row is taken away, and in rows of one or two columns
// that is next to nothing, 1 - yh^2 of it, which fp32 loses altogether.
template <typename T, int V, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS <= kNormThreads ? 2 : 1) k_norm_backward(const NormArgs a) {
  pdl_prologue();
  extern __shared__ uint4 norm_ring[];
  typedef typename std::conditional<V == 1 && ITEMS == 1, double, float>::type A;
  __shared__ A scratch[2 * 64];
  typedef Vec<T, V> X;
  constexpr int kStages = norm_stages<V, ITEMS, 5, THREADS>();
  constexpr bool kKeep = V * ITEMS <= 8;
  constexpr int kKept = kKeep ? ITEMS : 1;
  constexpr bool kBoth = kKeep && V == 8, kKeepNext = kKeep && !kBoth;
  const int W = a.warps_per_row, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / W, g = blockIdx.x * (blockDim.x / (W * 32)) + group;
  if (g >= a.groups) return;
  const bool has_dy = a.dy.p != nullptr, next = a.du.p != nullptr, block = a.block.p != nullptr;
  const bool gate = a.gate.p != nullptr, vector = gate && a.gate_vector;
  long long r = norm_first_row(a, g);
  const long long r_end = norm_first_row(a, g + 1);
  int m = (int)(r / a.rows), i = (int)(r % a.rows);
  enum { kDy, kDu, kY, kBlock, kGate };
  RowRing<T, V, ITEMS, 5, kStages, THREADS> ring;
  ring.slot = (warp % W) * 32 + lane; ring.step = W * 32; ring.nv = a.width / V; ring.rows = a.rows; ring.group = group;
  ring.pitch = norm_pitch<T>(a.width);
  ring.slots = V > 2 ? norm_ring + threadIdx.x : norm_ring + group * (5 * ring.pitch / 16);
  ring.i = i; ring.left = (int)(r_end - r);
  ring.set(kDy, a.dy, has_dy, m); ring.set(kDu, a.du, next, m); ring.set(kY, a.x, next, m);
  ring.set(kBlock, a.block, block, m); ring.set(kGate, a.gate, gate, m);
#pragma unroll
  for (int s = 0; s < kStages; ++s) ring.ask(s);
  float acc_next[ITEMS][V], acc_post[ITEMS][V], acc_gate[ITEMS][V];
  float acc_scale = 0.f;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) acc_next[k][j] = acc_post[k][j] = acc_gate[k][j] = 0.f;
  const int first = ring.slot * V, far = ring.step * V;      // this thread's first element and the distance to its next vector
  T* dx = reinterpret_cast<T*>(a.dx) + r * a.width + first;
  T* dblock = reinterpret_cast<T*>(a.dblock) + r * a.width + first;
  T* dgate = reinterpret_cast<T*>(a.dgate) + r * a.width + first;
  const float* rstd_next = a.rstd_next + r;
  const float* rstd_block = a.rstd_block + r;
  // the weights of the member at hand; the variants that keep their values keep these, too (but for the next norm's, see GateParts)
  A w_next[kKept][V], w_post[kKept][V];
  A c = 1;
  auto member = [&]() {
    if (a.scale && block) c = a.scale[m];
    if constexpr (kKeep) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        if (ring.slot + k * ring.step >= ring.nv) continue;
        if constexpr (kKeepNext)
          if (next) load_weights<V>(a.next_weight + (long long)m * a.width + first + k * far, w_next[k]);
        if (block) load_weights<V>(a.post_weight + (long long)m * a.width + first + k * far, w_post[k]);
      }
    }
  };
  member();
  int turn = 0, stage = 0;
  for (; r < r_end; ++r) {
    const A ry = next ? *rstd_next : 0.f, rb = block ? *rstd_block : 0.f;
    ring.wait();
    A sums[3] = {0, 0, 0};                                     // r_y dh yh, p (dy + r_y dh), p yh, with p = g w_post v
    A t[kKept][V], yh[kKept][V], v[kKept][V];   // dy + r_y dh, yh, v
    GateParts<kBoth> parts[kKept][V];
    // the vectors k of the row; `once`: with the sums that do not wait for the reduction
    auto values = [&](int k, int to, bool once) {
#pragma unroll
      for (int j = 0; j < V; ++j) t[to][j] = yh[to][j] = 0;
      if (has_dy) ring.get(stage, kDy, k, t[to]);
      if (next) {
        A du[V];
        ring.get(stage, kDu, k, du);
        ring.get(stage, kY, k, yh[to]);
        if constexpr (!kKeepNext) load_weights<V>(a.next_weight + (long long)m * a.width + first + k * far, w_next[to]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          yh[to][j] *= ry;
          if (once) acc_next[k][j] += (float)(du[j] * yh[to][j]);
          du[j] *= ry * w_next[to][j];
          if (once) sums[0] += du[j] * yh[to][j];
          t[to][j] += du[j];
        }
      }
      if (block) {
        A open[V];      // where the row is read twice, its first pass takes no more of the gate (19 x 231 x 8192 bf16: 222 us, with both parts 234)
        ring.get(stage, kBlock, k, v[to]);
        if constexpr (!kKeep) load_weights<V>(a.post_weight + (long long)m * a.width + first + k * far, w_post[to]);
        if (gate) {
          A z[V];
          ring.get(stage, kGate, k, z);
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (kKeep || !once) parts[to][j].of((float)z[j]);
            else open[j] = opened((float)z[j]);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            parts[to][j].none();
            open[j] = 1;
          }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          v[to][j] *= rb;
          if (once) {
            const A p = v[to][j] * w_post[to][j] * (kKeep ? parts[to][j].template open<A>() : open[j]);
            sums[1] += p * t[to][j];
            sums[2] += p * yh[to][j];
          }
        }
      }
    };
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
      if (ring.slot + k * ring.step < ring.nv) values(k, kKeep ? k : 0, true);
    if constexpr (kKeep) {          // the row has left the stage
      ring.ask(stage);
      if (++stage == kStages) stage = 0;
    }
    row_sum3(sums, W, group, scratch, turn);
    const A share = (A)1 / a.width;
    const A t1 = sums[0] * share;                                             // r_y t1
    const A crb = c * rb, t2 = crb * (sums[1] - t1 * sums[2]) * share;          // c r_b t2
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int from = kKeep ? k : 0;
      if (ring.slot + k * ring.step >= ring.nv) continue;
      if constexpr (!kKeep) values(k, 0, false);
#pragma unroll
      for (int j = 0; j < V; ++j) t[from][j] -= yh[from][j] * t1;
      X::store(dx + k * far, t[from]);
      if (block) {
        A db[V], dz[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const A gdx = parts[from][j].template open<A>() * t[from][j], gwdx = gdx * w_post[from][j], o = gwdx * v[from][j];
          acc_post[k][j] += (float)(gdx * v[from][j]);
          acc_scale += (float)o;
          db[j] = crb * gwdx - v[from][j] * t2;
          dz[j] = c * o * parts[from][j].template closed<A>();
        }
        X::store(dblock + k * far, db);
        if (vector) {
#pragma unroll
          for (int j = 0; j < V; ++j) acc_gate[k][j] += (float)dz[j];
        } else if (gate) {
          X::store(dgate + k * far, dz);
        }
      }
    }
    if constexpr (!kKeep) {
      ring.ask(stage);
      if (++stage == kStages) stage = 0;
    }
    dx += a.width;
    dblock += a.width;
    dgate += a.width;
    ++rstd_next;
    ++rstd_block;
    if (++i < a.rows && r + 1 < r_end) continue;
    // the last row here of this member: leave its sums.  The pairs (row group, member) ascend in g + m.
    float* out = a.partial + (long long)(g + m) * a.sums * a.width + first;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      if (ring.slot + k * ring.step >= ring.nv) continue;
      float* o = out + k * far;
      auto leave = [&](float* acc) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          o[j] = acc[j];
          acc[j] = 0.f;
        }
        o += a.width;
      };
      if (next) leave(acc_next[k]);
      if (block) {
#pragma unroll
        for (int j = 0; j < V; ++j) acc_post[k][j] *= (float)c;      // the member's scale, once for all its rows
        leave(acc_post[k]);
      }
      if (vector) leave(acc_gate[k]);
    }
    if (block) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc_scale += __shfl_xor_sync(0xFFFFFFFFu, acc_scale, o);
      if (lane == 0) a.partial_scale[(long long)(g + m) * W + warp % W] = acc_scale;
      acc_scale = 0.f;
    }
    i = 0;
    ++m;
    if (r + 1 < r_end) member();
  }
}

// A member's column sums (blockIdx.z: which of them) from the partial results of its row groups.  WAYS == 1: a thread adds up a
// column.  WAYS == 8, for members with many row groups: a block takes 32 columns, its eight warps every eighth row group,
// and adds the warps' sums in order.
template <typename T, int WAYS>
__global__ void __launch_bounds__(256) k_norm_columns(const NormArgs a) {
  pdl_prologue();
  __shared__ float part[8][33];
  const int m = blockIdx.y, q = blockIdx.z, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int e = WAYS == 1 ? blockIdx.x * 256 + threadIdx.x : blockIdx.x * 32 + lane, way = WAYS == 1 ? 0 : warp;
  const bool next = a.du.p != nullptr, block = a.block.p != nullptr;
  const int g0 = norm_group_of(a, (long long)m * a.rows), g1 = norm_group_of(a, (long long)(m + 1) * a.rows - 1);
  float t = 0.f;
  if (e < a.width) {
    const float* p = a.partial + ((long long)(g0 + way + m) * a.sums + q) * a.width + e;
    const long long step = (long long)WAYS * a.sums * a.width;
#pragma unroll 8
    for (int g = g0 + way; g <= g1; g += WAYS, p += step) t += __ldcg(p);
  }
  if (WAYS > 1) {
    part[warp][lane] = t;
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int w = 1; w < 8; ++w) t += part[w][lane];
    }
    __syncthreads();
  }
  if (e < a.width && (WAYS == 1 || warp == 0)) {
    const long long at = (long long)m * a.width + e;
    if (next && q == 0) a.dnext[at] = t;
    else if (q == (next ? 1 : 0)) a.dpost[at] = t;
    else Vec<T, 1>::store(reinterpret_cast<T*>(a.dgate) + at, &t);
  }
  if (block && blockIdx.x == 0 && q == 0 && a.dscale) {
    const int n = (g1 - g0 + 1) * a.warps_per_row;
    const float* p = a.partial_scale + (long long)(g0 + m) * a.warps_per_row;
    t = 0.f;
    for (int k = threadIdx.x; k < n; k += 256) t += p[k];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
    if (lane == 0) part[warp][0] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < 8; ++w) t += part[w][0];
      a.dscale[m] = t;
    }
  }
}
template <typename T>
cudaError_t launch_norm_columns(const NormArgs& a, cudaStream_t s) {
  // one thread a column is enough work for the SMs' latency while a member has few row groups (80 x 512 x 2048, 8 each: the backward pass 278 us,
  // with eight warps a column 295; 1 x 4096 x 1024, 592: 55 and 33)
  if (a.groups / a.members <= 16) return launch_with(dim3((a.width + 255) / 256, a.members, a.sums), 256, 0, s)(k_norm_columns<T, 1>, a);
  return launch_with(dim3((a.width + 31) / 32, a.members, a.sums), 256, 0, s)(k_norm_columns<T, 8>, a);
}

int norm_fail(int code, const char* msg) {
  set_last_error(msg);
  return code;
}

// Elements per vector: 16-byte vectors if the width and every pointer and stride allow them, else pairs (but for the narrow rows that are
// worked out in fp64), else single elements.  19 x 231 x 2050 bf16: pairs 35 us forward and 89 backward, single elements 53 and 132 (2048 columns in
// 16-byte vectors: 23 and 48).
int norm_vector(const pbt_block_norm_desc* d, bool backward) {
  const int esz = d->dtype ? 2 : 4;
  auto fits = [&](int v) {
    const int bytes = v * esz;      // of a vector; weights are read with at most 16 bytes at a time
    bool ok = d->width % v == 0;
    auto in = [&](const void* p, int64_t member, int64_t row) {
      if (p) ok = ok && (uintptr_t)p % bytes == 0 && (member * esz) % bytes == 0 && (row * esz) % bytes == 0;
    };
    auto flat = [&](const void* p) { if (p) ok = ok && (uintptr_t)p % bytes == 0; };
    auto weights = [&](const void* p) { if (p) ok = ok && (uintptr_t)p % std::min(16, v * 4) == 0; };
    in(d->x, d->x_member, d->x_row);
    in(d->block, d->block_member, d->block_row);
    in(d->gate, d->gate_member, d->gate_row);
    weights(d->post_weight);
    weights(d->next_weight);
    if (backward) {
      in(d->dy, d->dy_member, d->dy_row);
      in(d->du, d->du_member, d->du_row);
      flat(d->dx); flat(d->dblock); flat(d->dgate);
    } else {
      flat(d->y); flat(d->u);
    }
    return ok;
  };
  return fits(16 / esz) ? 16 / esz : d->width > 32 && fits(2) ? 2 : 1;
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

// Elements of a thread (`items` vectors) and warps of a row.  Forward: 16 elements a thread before a row takes another warp
// (fewer warps: cheaper reductions; 2048 bf16 columns 169 us with 16, 228 us with 8).  Backward: 8, which leaves registers
// for what the first pass works out (344 us with 16), and 16 beyond 4096 columns.  Blocks have 256 threads as long as eight
// warps hold a row, 512 beyond.  When rows are so few that a row group would get fewer than four, a row takes up to eight
// warps instead: its latency is what counts then.
struct NormShape { int items, warps, groups, threads; };
NormShape norm_shape(const pbt_block_norm_desc* d, int v, bool backward) {
  const int nv = d->width / v, most = backward && d->width <= 4096 ? 8 : 16;
  const long long rows = (long long)d->members * d->rows;
  NormShape s;
  s.items = 1;
  while (s.items * v < most && nv > s.items * 32) s.items *= 2;
  auto fill = [&]() {
    s.warps = (nv + s.items * 32 - 1) / (s.items * 32);
    s.groups = std::max(1, kNormThreads / 32 / s.warps);
  };
  fill();
  while (s.items > (v == 1 ? 2 : 1) && s.warps <= 4 && rows < 4ll * 2 * 148 * s.groups) {
    s.items /= 2;
    fill();
  }
  s.threads = s.groups * s.warps * 32;
  return s;
}

// Blocks of the grid: `per_sm` per SM, or fewer so that every row group has a row.
int norm_blocks(const pbt_block_norm_desc* d, int groups, int per_sm) {
  const long long most = ((long long)d->members * d->rows + groups - 1) / groups;
  return (int)std::max<long long>(1, std::min<long long>(per_sm * 148, most));
}
int norm_groups(const pbt_block_norm_desc* d, int groups, int blocks) {
  return (int)std::max<long long>(1, std::min<long long>((long long)blocks * groups, (long long)d->members * d->rows));
}

struct NormPlan { int v, blocks, groups, sums; NormShape shape; size_t slots, bytes; };

NormPlan norm_backward_plan(const pbt_block_norm_desc* d) {
  NormPlan p;
  p.v = norm_vector(d, true);
  p.shape = norm_shape(d, p.v, true);
  p.blocks = norm_blocks(d, p.shape.groups, p.shape.threads > kNormThreads ? 1 : 2);
  p.groups = norm_groups(d, p.shape.groups, p.blocks);
  p.sums = (d->du ? 1 : 0) + (d->block ? 1 : 0) + (d->gate && d->gate_vector ? 1 : 0);
  p.slots = (size_t)p.groups + d->members;
  p.bytes = p.slots * ((size_t)p.sums * d->width + p.shape.warps) * sizeof(float);
  p.bytes = (p.bytes + 255) & ~(size_t)255;
  return p;
}

template <typename T, int V, int ITEMS, int THREADS>
cudaError_t launch_norm_backward(unsigned grid, int threads, const NormArgs& a, cudaStream_t s) {
  // unaligned rows: at most 16 elements and two granules' edges a thread
  constexpr int most = V <= 2 ? 5 * (THREADS * ITEMS * V * (int)sizeof(T) + THREADS / 32 * 32) : norm_stages<V, ITEMS, 5, THREADS>() * 5 * ITEMS * 16 * THREADS;
  const int smem = V <= 2 ? 5 * norm_pitch<T>(a.width) * (threads / (a.warps_per_row * 32)) : most;
  static tc::DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = tc::device_setup(&setup, k_norm_backward<T, V, ITEMS, THREADS>, most, &sms);
  if (e != cudaSuccess) return e;
  return launch_with(grid, threads, smem, s)(k_norm_backward<T, V, ITEMS, THREADS>, a);
}
template <typename T, int V, int ITEMS, int THREADS>
cudaError_t launch_norm_forward(unsigned grid, int threads, const NormArgs& a, cudaStream_t s) {
  // unaligned rows: at most 16 elements and two granules' edges a thread
  constexpr int most = V <= 2 ? 3 * (THREADS * ITEMS * V * (int)sizeof(T) + THREADS / 32 * 32) : norm_stages<V, ITEMS, 3, THREADS>() * 3 * ITEMS * 16 * THREADS;
  const int smem = V <= 2 ? 3 * norm_pitch<T>(a.width) * (threads / (a.warps_per_row * 32)) : most;
  static tc::DeviceSetup setup;
  int sms = 0;
  const cudaError_t e = tc::device_setup(&setup, k_norm_forward<T, V, ITEMS, THREADS>, most, &sms);
  if (e != cudaSuccess) return e;
  return launch_with(grid, threads, smem, s)(k_norm_forward<T, V, ITEMS, THREADS>, a);
}
// The instantiations that norm_shape can ask for: blocks of 512 threads belong to the most elements a thread.
template <typename T, int V, int ITEMS>
cudaError_t launch_norm(bool backward, const NormShape& p, unsigned grid, const NormArgs& a, cudaStream_t s) {
  if (!backward) {
    if constexpr (ITEMS * V == 16)
      if (p.threads > kNormThreads) return launch_norm_forward<T, V, ITEMS, 512>(grid, p.threads, a, s);
    return launch_norm_forward<T, V, ITEMS, kNormThreads>(grid, p.threads, a, s);
  }
  if constexpr (ITEMS * V >= 8)
    if (p.threads > kNormThreads) return launch_norm_backward<T, V, ITEMS, 512>(grid, p.threads, a, s);
  if constexpr (ITEMS * V <= 8) return launch_norm_backward<T, V, ITEMS, kNormThreads>(grid, p.threads, a, s);
  return cudaErrorInvalidValue;
}
template <typename T, int V>
cudaError_t launch_norm(bool backward, const NormShape& p, unsigned grid, const NormArgs& a, cudaStream_t s) {
  if (p.items == 1) return launch_norm<T, V, 1>(backward, p, grid, a, s);
  if (p.items == 2) return launch_norm<T, V, 2>(backward, p, grid, a, s);
  if constexpr (V <= 4)
    if (p.items == 4) return launch_norm<T, V, 4>(backward, p, grid, a, s);
  if constexpr (V <= 2)
    if (p.items == 8) return launch_norm<T, V, 8>(backward, p, grid, a, s);
  if constexpr (V == 1) {
    if (p.items == 16) return launch_norm<T, V, 16>(backward, p, grid, a, s);
  }
  return cudaErrorInvalidValue;
}
cudaError_t launch_norm(bool bf, int v, bool backward, const NormShape& p, unsigned grid, const NormArgs& a, cudaStream_t s) {
  if (bf) return v == 1 ? launch_norm<bf16, 1>(backward, p, grid, a, s) : v == 2 ? launch_norm<bf16, 2>(backward, p, grid, a, s) : launch_norm<bf16, 8>(backward, p, grid, a, s);
  return v == 1 ? launch_norm<float, 1>(backward, p, grid, a, s) : v == 2 ? launch_norm<float, 2>(backward, p, grid, a, s) : launch_norm<float, 4>(backward, p, grid, a, s);
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
  const NormShape shape = norm_shape(d, v, false);
  const int blocks = norm_blocks(d, shape.groups, shape.threads > kNormThreads ? 1 : 4);
  a.warps_per_row = shape.warps;
  a.groups = norm_groups(d, shape.groups, blocks);
  const cudaError_t e = launch_norm(d->dtype == 1, v, false, shape, (unsigned)blocks, a, (cudaStream_t)stream);
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
  if (!d->rows) {   // no row contributes: the sums over rows are zero
    const size_t n = (size_t)d->members * d->width;
    cudaError_t e = cudaSuccess;
    auto zero = [&](void* q, size_t bytes) { if (q && e == cudaSuccess) e = cudaMemsetAsync(q, 0, bytes, (cudaStream_t)stream); };
    if (d->du) zero(d->dnext_weight, n * sizeof(float));
    if (d->block) zero(d->dpost_weight, n * sizeof(float));
    if (d->block) zero(d->dscale, d->members * sizeof(float));
    if (d->gate && d->gate_vector) zero(d->dgate, n * (d->dtype ? 2 : 4));
    return e == cudaSuccess ? PBT_OK : norm_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
  }
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < p.bytes)
    return norm_fail(PBT_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than pbt_block_norm_query_workspace says");
  NormArgs a;
  norm_fill(&a, d);
  a.warps_per_row = p.shape.warps; a.groups = p.groups; a.sums = p.sums;
  a.partial = (float*)workspace;
  a.partial_scale = a.partial + p.slots * p.sums * d->width;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e = launch_norm(d->dtype == 1, p.v, true, p.shape, (unsigned)p.blocks, a, s);
  if (e == cudaSuccess) e = d->dtype ? launch_norm_columns<bf16>(a, s) : launch_norm_columns<float>(a, s);
  if (e != cudaSuccess) return norm_fail(PBT_ERR_CUDA, cudaGetErrorString(e));
  return PBT_OK;
}
