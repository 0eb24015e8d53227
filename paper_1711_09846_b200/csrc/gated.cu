// Gated units of a population, h = keep / (1 - rate) act(x Wg^T) (x Wu^T) per member, and their gradients: entry points and the element-wise part of
// the backward pass.  The products are in gated_tc.cu (bf16) and gated_f32.cu, and in the framework's member-batched GEMMs.
//
// g and u stay in fp32 for the backward pass: as bf16 numbers they would add their own rounding to that of every gradient (dg and du have it once, as operands),
// and a kept fp32 pair costs 0.2 ms of 2 for 80 members x 512 rows x 2048 hidden units, working it out anew 0.5.
//
// dg and du of a bf16 pass are rounded to bf16 before dx and dW, which then are off by 0.0023 of their 2-norm, 1.4 times what the rounding of the results alone leaves (0.0017).
// A tensor-core product takes both operands in one 16-bit type; dg and du of 32 bits would go through it as two bf16 numbers each and double both products (another
// 1.1 ms of 2 at that size).  Whoever needs gradients without that rounding has the fp32 unit.
#include <algorithm>

#include "gated.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace gated {
namespace {

using dropout::as_float;
using dropout::Eight;
using dropout::kGroup;
using dropout::load16;
using dropout::store;
using dropout::store8;
using dropout::unpack;

int fail(int code, const char* msg) {
  set_last_error(msg);
  return code;
}

int round_up(int n, int m) { return (n + m - 1) / m * m; }

// dg and du of a row's hidden units from g, u and dh; a thread has eight neighbouring ones, a block of the generator.
template <typename T>
struct CellArgs {
  const float* z; int pitch;                      // [members][rows][2][pitch]: g, then u
  const T* dh; long long dh_member, dh_row;
  T* out; long long out_pitch;                    // [dg du] [members][rows][out_pitch]
  uint32_t rows, hidden, groups;
  int activation, drop, beside;
  dropout::Rule rule;
};

__device__ __forceinline__ void store_pairs(float* p, const Eight& e) {
#pragma unroll
  for (int c = 0; c < kGroup; ++c) p[c] = e.v[c];
}
// pairs from the first 4-byte boundary on
__device__ __forceinline__ void store_pairs(bf16* p, const Eight& e) {
  auto pair = [&](int c) { *reinterpret_cast<__nv_bfloat162*>(p + c) = __floats2bfloat162_rn(e.v[c], e.v[c + 1]); };
  if (((uintptr_t)p & 3) == 0) {
#pragma unroll
    for (int c = 0; c < kGroup; c += 2) pair(c);
  } else {
    store(p, e.v[0]);
#pragma unroll
    for (int c = 1; c < kGroup - 1; c += 2) pair(c);
    store(p + kGroup - 1, e.v[kGroup - 1]);
  }
}
// Beside the kernel that packs operands, which it needs nothing of: the products, which do, may begin when both are done.
struct Turn {
  bool beside;
  __device__ __forceinline__ Turn(bool b) : beside(b) {
    if (beside) return;
    pdl_prologue();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the products may begin with their other operands
  }
  __device__ __forceinline__ ~Turn() {
    if (!beside) return;
    pdl_prologue();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
};
// VEC: 16-byte loads and stores everywhere.  Bound by its bytes, 14 a hidden unit in bf16 (80 x 512 x 2048: 189 us, 6.2 TB/s).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_gated_cells(const CellArgs<T> a) {
  const Turn turn(a.beside);
  const int m = blockIdx.y;
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (uint64_t)a.rows * a.groups) return;
  const uint32_t row = (uint32_t)i / a.groups, c0 = ((uint32_t)i - row * a.groups) * kGroup, n = VEC ? kGroup : min(a.hidden - c0, (uint32_t)kGroup);
  const long long at = (long long)m * a.rows + row;
  const float* z = a.z + at * 2 * a.pitch + c0;           // (the pitch is a multiple of eight: whole groups)
  T* out = a.out + at * a.out_pitch + c0;
  const T* from = a.dh + m * a.dh_member + row * a.dh_row + c0;
  const uint4 z0 = load16(z), z1 = load16(z + 4), z2 = load16(z + a.pitch), z3 = load16(z + a.pitch + 4);
  Eight dh;
  if constexpr (sizeof(T) == 2) {
    dh = unpack(VEC ? load16(from) : joined(pieces_of(from, (int)n)));
  } else if constexpr (VEC) {
    dh = unpack(load16(from), load16(from + 4));
  } else {
#pragma unroll
    for (int c = 0; c < kGroup; ++c) dh.v[c] = c < n ? as_float(from[c]) : 0.f;
  }
  const Eight g = unpack(z0, z1), u = unpack(z2, z3);
  uint32_t in = 0xFFu;
  float f = 1.f;
  if (a.drop) {
    const dropout::Draw d = dropout::draw_of(a.rule, m);
    in = dropout::kept_bits(a.rule, d, (uint32_t)i);
    if (d.on) f = d.scale;
  }
  Eight dg, du;
#pragma unroll
  for (int c = 0; c < kGroup; ++c) {
    const bool keep = in >> c & 1u;
    float slope;
    const float act = activation<T>(a.activation, g.v[c], &slope), v = f * dh.v[c];
    dg.v[c] = keep ? v * u.v[c] * slope : 0.f;
    du.v[c] = keep ? v * act : 0.f;
  }
  if constexpr (VEC) {
    store8(out, dg);
    store8(out + a.hidden, du);
  } else if (n == kGroup) {
    store8(out, dg);              // (a row of dg and du begins on 16 bytes, du within it anywhere)
    store_pairs(out + a.hidden, du);
  } else {
#pragma unroll
    for (int c = 0; c < kGroup; ++c) {
      if (c >= n) break;
      store(out + c, dg.v[c]);
      store(out + a.hidden + c, du.v[c]);
    }
  }
}

// What a call does and where things lie in its workspace.
struct Plan {
  int pitch;                      // of g and u
  int dz_pitch;
  size_t z, dz, x, w, bytes;      // offsets; z: a backward pass for which nothing was kept
  bool pack_x, pack_w;     // pack: bf16 rows that are not multiples of 16 bytes are laid out anew
};
Plan plan_of(const pbt_gated_desc* d, bool backward) {
  Plan p = {};
  p.pitch = round_up(d->hidden, kGroup);
  p.dz_pitch = round_up(2 * d->hidden, kGroup);
  const size_t rows = (size_t)d->members * d->rows, size = d->dtype ? 2 : 4;
  auto take = [&](size_t bytes) { const size_t at = p.bytes; p.bytes += (bytes + 255) & ~(size_t)255; return at; };
  if (!d->kept && backward) p.z = take(rows * 2 * p.pitch * sizeof(float));
  if (backward) p.dz = take(rows * p.dz_pitch * size);
  if (d->dtype) {
    p.pack_x = !tc_aligned(d->x, d->x_row, d->x_member, d->members);
    p.pack_w = !tc_aligned(d->weight, d->weight_row, d->weight_member, d->members);
    const size_t width = round_up(d->width, 8);
    if (p.pack_x) p.x = take(rows * width * size);
    if (p.pack_w) p.w = take((d->weight_member ? d->members : 1) * 2 * (size_t)d->hidden * width * size);
  }
  return p;
}

// x and the weight as the kernels take them, packed where that is needed
struct Operands {
  Operand x, w;
};
cudaError_t operands_of(const pbt_gated_desc* d, const Plan& p, char* ws, Operands* o, cudaStream_t s) {
  o->x = {(const bf16*)d->x, d->x_row, d->x_member};
  o->w = {(const bf16*)d->weight, d->weight_row, d->members > 1 ? d->weight_member : 0};
  const int width = round_up(d->width, 8);
  PackSource jobs[2];
  int n = 0;
  if (p.pack_x) {
    jobs[n++] = {o->x, (bf16*)(ws + p.x), d->members, d->rows, d->width};
    o->x = {(const bf16*)(ws + p.x), width, (long long)d->rows * width};
  }
  if (p.pack_w) {
    const int members = o->w.member ? d->members : 1;
    jobs[n++] = {o->w, (bf16*)(ws + p.w), members, 2 * d->hidden, d->width};
    o->w = {(const bf16*)(ws + p.w), width, members > 1 ? 2ll * d->hidden * width : 0};
  }
  return n ? tc_pack(jobs, n, s) : cudaSuccess;
}

template <typename T>
CellArgs<T> cells_of(const pbt_gated_desc* d, const Plan& p, const float* z) {
  CellArgs<T> a = {};
  a.z = z; a.pitch = p.pitch;
  a.rows = (uint32_t)d->rows; a.hidden = (uint32_t)d->hidden; a.groups = (uint32_t)(p.pitch / kGroup);
  a.activation = d->activation; a.drop = d->drop != nullptr;
  if (d->drop) a.rule = dropout::rule_of(*d->drop);
  return a;
}
template <typename T>
cudaError_t launch_cells(const pbt_gated_desc* d, const CellArgs<T>& a, cudaStream_t s) {
  const dim3 grid((unsigned)(((uint64_t)a.rows * a.groups + 255) / 256), (unsigned)d->members);
  // (dh: any base, row and member stride that keeps 16 bytes; what this library lays out has them where hidden is a multiple of eight)
  constexpr int kStep = 16 / sizeof(T);
  const bool vec = d->hidden % kGroup == 0 && ((uintptr_t)a.out & 15) == 0 && a.out_pitch % kStep == 0 &&
                   ((uintptr_t)a.dh & 15) == 0 && (d->rows == 1 || a.dh_row % kStep == 0) && (d->members == 1 || a.dh_member % kStep == 0);
  const int order = a.beside ? kBeside : 0;
  return vec ? launch_ordered(order, grid, 256, 0, s, k_gated_cells<T, true>, a) : launch_ordered(order, grid, 256, 0, s, k_gated_cells<T, false>, a);
}

GemmArgs product(const pbt_gated_desc* d) {
  GemmArgs g;
  memset(&g, 0, sizeof(g));
  g.batch = d->members;
  g.in_dtype = g.out_dtype = kBF16;
  return g;
}

cudaError_t forward(const pbt_gated_desc* d, char* ws, cudaStream_t s) {
  const Plan p = plan_of(d, false);
  if (d->dtype) {
    Operands o;
    const cudaError_t e = operands_of(d, p, ws, &o, s);
    return e == cudaSuccess ? tc_forward(d, o.x, o.w, d->h, d->kept, p.pitch, p.pack_x || p.pack_w, s) : e;
  }
  return f32_forward(d, (float*)d->h, d->kept, p.pitch, s);
}

// The faster of the tensor-core products, which take any number of rows here: tensor maps fill what is missing with zeros.  In waves of 128 x 256 (a pair:
// 256 x 256) tiles; launch_gemm_tc halves its tiles where that shortens the last wave.  A pair's cost less from contractions of 384 on (40 members,
// 512 rows, 1024 -> 1024: dW 10 us less, 8 x 160, 2048 -> 2048: 4 us more).
cudaError_t run_product(const pbt_gated_desc* d, const GemmArgs& g, cudaStream_t s) {
  auto waves = [&](int rows, int cols, int at_once) {
    const long long tiles = (long long)((g.M + rows - 1) / rows) * ((g.N + cols - 1) / cols) * g.batch;
    return (double)((tiles + at_once - 1) / at_once);
  };
  const double pair = (g.K >= 384 ? 0.95 : 1.03) * waves(256, 256, 74), single = std::min(waves(128, 256, 148), 0.575 * waves(128, 128, 148));
  Counters* counters = (Counters*)d->status_device;
  return g.M >= 256 && g.N >= 256 && pair < single ? launch_gemm_tc_pair(g, counters, s) : launch_gemm_tc(g, counters, s);
}

template <typename T>
cudaError_t backward(const pbt_gated_desc* d, char* ws, cudaStream_t s) {
  const Plan p = plan_of(d, true);
  const float* z = d->kept;
  cudaError_t e = cudaSuccess;
  Operands o = {};
  if (d->dtype) e = operands_of(d, p, ws, &o, s);
  if (e == cudaSuccess && !z) {
    float* made = (float*)(ws + p.z);
    e = d->dtype ? tc_forward(d, o.x, o.w, nullptr, made, p.pitch, p.pack_x || p.pack_w, s) : f32_forward(d, nullptr, made, p.pitch, s);
    z = made;
  }
  if (e != cudaSuccess) return e;
  T* dz = (T*)(ws + p.dz);
  CellArgs<T> a = cells_of<T>(d, p, z);
  a.dh = (const T*)d->dh; a.dh_member = d->dh_member; a.dh_row = d->dh_row;
  a.out = dz; a.out_pitch = p.dz_pitch;
  a.beside = d->kept && (p.pack_x || p.pack_w);
  e = launch_cells<T>(d, a, s);
  if (e != cudaSuccess) return e;
  if (!d->dtype) return f32_backward(d, (const float*)dz, p.dz_pitch, s);
  const Operand left = {(const bf16*)dz, p.dz_pitch, (long long)d->rows * p.dz_pitch};
  if (tc_gradients_few(d)) return tc_gradients(d, left, o.w, o.x, s);
  GemmArgs g = product(d);
  g.A = dz; g.lda = p.dz_pitch; g.strideA = (long long)d->rows * p.dz_pitch;
  g.M = d->rows; g.N = d->width; g.K = 2 * d->hidden;
  g.b_mn = 1;
  g.B = o.w.p; g.ldb = o.w.row; g.strideB = o.w.member;
  g.C = d->dx; g.ldc = d->width; g.strideC = (long long)d->rows * d->width;
  g.order = kAfter | kLeads;
  if (tc_dx_few(d)) e = tc_dx(d, left, o.w, s);
  else e = run_product(d, g, s);
  if (e != cudaSuccess) return e;
  g.order = kBeside;      // dW takes the SMs that dx leaves in its last wave
  g.a_mn = 1;
  g.M = 2 * d->hidden; g.K = d->rows;
  g.B = o.x.p; g.ldb = o.x.row; g.strideB = o.x.member;
  g.C = d->dweight; g.strideC = 2ll * d->hidden * d->width;
  return run_product(d, g, s);
}

int check(const pbt_gated_desc* d) {
  if (!d) return fail(PBT_ERR_INVALID_ARG, "desc is NULL");
  if (d->members < 1 || d->rows < 0 || d->width < 1 || d->hidden < 1) return fail(PBT_ERR_INVALID_ARG, "members, width and hidden must be positive, rows >= 0");
  if (d->members > 65535) return fail(PBT_ERR_UNSUPPORTED, "more than 65535 members");
  if (d->rows >= 1 << 22 || d->width >= 1 << 22 || d->hidden >= 1 << 21) return fail(PBT_ERR_UNSUPPORTED, "rows, width and 2 hidden must stay below 2^22");
  // tiles are counted in 32 bits (the smallest have 64 rows and 64 columns)
  auto tiles = [&](long long m, long long n) { return (m + 63) / 64 * ((n + 63) / 64) * d->members > 0x7FFFFFFFll; };
  if (tiles(d->rows, 2ll * d->hidden) || tiles(d->rows, d->width) || tiles(2ll * d->hidden, d->width))
    return fail(PBT_ERR_UNSUPPORTED, "more than 2^31 - 1 tiles of 64 x 64 elements in a call: split the members or the rows");
  if (d->dtype != 0 && d->dtype != 1) return fail(PBT_ERR_UNSUPPORTED, "operands are float or bfloat16");
  if (d->activation < 0 || d->activation > 3) return fail(PBT_ERR_UNSUPPORTED, "activation is 0 (silu), 1 (gelu), 2 (relu) or 3 (sigmoid)");
  if (!d->weight) return fail(PBT_ERR_INVALID_ARG, "weight is NULL");
  if (d->dtype == 1 && !d->status_device) return fail(PBT_ERR_INVALID_ARG, "status_device is required by the tensor-core kernels");
  if (d->weight_row < d->width || d->weight_member < 0) return fail(PBT_ERR_INVALID_ARG, "weight_row is smaller than a row, or weight_member negative");
  if (d->rows && (!d->x || d->x_row < d->width || d->x_member < 0)) return fail(PBT_ERR_INVALID_ARG, "x is NULL, its row stride smaller than a row or its member stride negative");
  if ((uintptr_t)d->kept & 15) return fail(PBT_ERR_INVALID_ARG, "kept has to begin on 16 bytes");
  if (d->dtype) {
    const Plan p = plan_of(d, false);
    const unsigned long long per_row = (d->width + 7) / 8, most = 0x7FFFF000ull;      // (32 GB)
    if ((p.pack_x && (unsigned long long)d->members * d->rows * per_row > most) || (p.pack_w && (unsigned long long)d->members * 2 * d->hidden * per_row > most))
      return fail(PBT_ERR_UNSUPPORTED, "rows of x or weight that are not multiples of 16 bytes are laid out anew, 2^34 elements at most");
  }
  return d->drop ? dropout::check_rule(d->drop, d->members, d->rows, d->hidden) : PBT_OK;
}

int check_workspace(const pbt_gated_desc* d, bool backward, const void* workspace, size_t bytes) {
  const size_t need = plan_of(d, backward).bytes;
  if (!need || (workspace && ((uintptr_t)workspace & 255) == 0 && bytes >= need)) return PBT_OK;
  return fail(PBT_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than pbt_gated_query_workspace says");
}

}  // namespace
}  // namespace gated
}  // namespace pbt

extern "C" int pbt_gated_query_workspace(const pbt_gated_desc* d, int backward, size_t* bytes) {
  using namespace pbt::gated;
  if (!bytes) return fail(PBT_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = check(d);
  if (rc) return rc;
  *bytes = plan_of(d, backward != 0).bytes;
  return PBT_OK;
}

extern "C" int pbt_gated_forward(const pbt_gated_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace pbt;
  using namespace pbt::gated;
  int rc = check(d);
  if (rc) return rc;
  if (!d->rows) return PBT_OK;
  if (!d->h) return fail(PBT_ERR_INVALID_ARG, "h is NULL");
  rc = check_workspace(d, false, workspace, workspace_bytes);
  if (rc) return rc;
  const cudaError_t e = forward(d, (char*)workspace, (cudaStream_t)stream);
  return e == cudaSuccess ? PBT_OK : fail(PBT_ERR_CUDA, cudaGetErrorString(e));
}

extern "C" int pbt_gated_backward(const pbt_gated_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace pbt;
  using namespace pbt::gated;
  int rc = check(d);
  if (rc) return rc;
  if (!d->dweight) return fail(PBT_ERR_INVALID_ARG, "dweight is NULL");
  cudaError_t e;
  if (!d->rows) {
    e = cudaMemsetAsync(d->dweight, 0, (size_t)d->members * 2 * d->hidden * d->width * (d->dtype ? 2 : 4), (cudaStream_t)stream);
  } else {
    if (!d->dx || !d->dh || d->dh_row < d->hidden || d->dh_member < 0)
      return fail(PBT_ERR_INVALID_ARG, "dx or dh is NULL, the row stride of dh smaller than a row or its member stride negative");
    rc = check_workspace(d, true, workspace, workspace_bytes);
    if (rc) return rc;
    e = d->dtype ? backward<bf16>(d, (char*)workspace, (cudaStream_t)stream) : backward<float>(d, (char*)workspace, (cudaStream_t)stream);
  }
  return e == cudaSuccess ? PBT_OK : fail(PBT_ERR_CUDA, cudaGetErrorString(e));
}
