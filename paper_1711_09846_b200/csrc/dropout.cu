// Dropout of activations, with masks that are drawn where they are needed: y = residual + keep x / (1 - rate).
//
// One pass over x (and residual): 4 or 6 bytes an element in bf16, 8 or 12 in fp32.  A group of eight neighbouring columns shares one
// block of the generator (20 32-bit multiplications with a 64-bit product), so that the draws cost less than the transfers.
#include "dropout.cuh"

namespace pbt {
void set_last_error(const char* msg);

namespace dropout {
namespace {

int fail(int code, const char* msg) {
  set_last_error(msg);
  return code;
}

template <typename T>
struct Args {
  const T* x; long long x_member, x_row;
  const T* residual; long long residual_member, residual_row;
  T* y;
  uint32_t rows, width, groups;     // groups of a row
  pbt_drop_rule rule;
};

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(256) k_dropout(const Args<T> a) {
  pdl_prologue();
  const int m = blockIdx.y;
  const Draw d = draw_of(a.rule, m);
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (uint64_t)a.rows * a.groups) return;
  const uint32_t row = (uint32_t)i / a.groups, c0 = ((uint32_t)i - row * a.groups) * kGroup, n = min(a.width - c0, (uint32_t)kGroup);
  const T* x = a.x + m * a.x_member + row * a.x_row + c0;
  const T* r = RESIDUAL ? a.residual + m * a.residual_member + row * a.residual_row + c0 : nullptr;
  T* y = a.y + ((long long)m * a.rows + row) * a.width + c0;
  U4 w = {};
  if (d.on) w = draw_group(d, (uint32_t)i);
#pragma unroll
  for (int c = 0; c < kGroup; ++c) {
    if (c >= n) break;
    float v = !d.on ? as_float(x[c]) : kept(w, c, d.limit) ? as_float(x[c]) * d.scale : 0.f;
    if (RESIDUAL) v += as_float(r[c]);
    store(y + c, v);
  }
}

template <typename T>
cudaError_t launch(const pbt_dropout_desc* d, cudaStream_t s) {
  const uint32_t groups = (uint32_t)((d->width + kGroup - 1) / kGroup);
  const Args<T> a = {(const T*)d->x, d->x_member, d->x_row, (const T*)d->residual, d->residual_member, d->residual_row, (T*)d->y,
                     (uint32_t)d->rows, (uint32_t)d->width, groups, d->rule};
  const dim3 grid((unsigned)(((uint64_t)d->rows * groups + 255) / 256), (unsigned)d->members);
  return d->residual ? launch_with(grid, 256, 0, s)(k_dropout<T, true>, a) : launch_with(grid, 256, 0, s)(k_dropout<T, false>, a);
}

}  // namespace

int check_rule(const pbt_drop_rule* r, long long members, long long rows, long long width) {
  if (r->site < 0 || r->site > (1 << 30)) return fail(PBT_ERR_INVALID_ARG, "a dropout's site must lie in [0, 2^30]");
  if (r->first_member < 0 || (long long)r->first_member + members > 0x7FFFFFFFll)
    return fail(PBT_ERR_INVALID_ARG, "first_member must be >= 0, and every member's index below 2^31");
  if (!r->rate && !(r->rate_all >= 0.f && r->rate_all <= 1.f)) return fail(PBT_ERR_INVALID_ARG, "a dropout rate must lie in [0, 1]");
  if (rows * ((width + kGroup - 1) / kGroup) > 0xFFFFFFFFll) return fail(PBT_ERR_UNSUPPORTED, "rows times ceil(width / 8) must stay below 2^32 (the generator's block number)");
  return PBT_OK;
}

}  // namespace dropout
}  // namespace pbt

extern "C" int pbt_dropout(const pbt_dropout_desc* d, void* stream) {
  using namespace pbt;
  using namespace pbt::dropout;
  if (!d) return fail(PBT_ERR_INVALID_ARG, "desc is NULL");
  if (d->members < 1 || d->rows < 0 || d->width < 1) return fail(PBT_ERR_INVALID_ARG, "members and width must be positive, rows >= 0");
  if (d->members > 65535) return fail(PBT_ERR_UNSUPPORTED, "more than 65535 members");
  if (d->dtype != 0 && d->dtype != 1) return fail(PBT_ERR_UNSUPPORTED, "activations are float or bfloat16");
  const int rc = check_rule(&d->rule, d->members, d->rows, d->width);
  if (rc) return rc;
  if (!d->rows) return PBT_OK;
  if (!d->x || !d->y) return fail(PBT_ERR_INVALID_ARG, "x or y is NULL");
  const cudaError_t e = d->dtype ? launch<bf16>(d, (cudaStream_t)stream) : launch<float>(d, (cudaStream_t)stream);
  return e == cudaSuccess ? PBT_OK : fail(PBT_ERR_CUDA, cudaGetErrorString(e));
}
