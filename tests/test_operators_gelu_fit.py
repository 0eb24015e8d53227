"""The bf16 gated unit's fit of the complementary error function, before its result is rounded.

The form is t exp(-x^2 + P(t)), t = 1 / (1 + x / 2) (Press, Teukolsky, Vetterling, Flannery, Numerical Recipes, section 6.2), with P of degree five; its
error is at most 8e-6 of the value.  In fp32 (eps = 2^-24), with x = |g| / sqrt 2: the exponent in powers of two, of size 1.45 x^2 + 3, comes from x (1.3 eps of it),
x^2 and a constant, 5 eps x^2 1.45 with its own rounding, and from P, 18 eps; as a factor of the result that is ln 2 of it, (5.1 x^2 + 12.5) eps.  The quotient t is off by
2 ulp and a rounding, 5 eps, which the result takes at most three times; the power of two by 4 eps; two products by 2.  Together 8e-6 + (5.1 x^2 + 34) eps of erfc / 2,
and two eps of the result; a result below 2^-126 is a multiple of 2^-149, half a step off its product.  A power of two below 2^-126 is taken for zero."""
import os
import re
import subprocess
import sys
import textwrap

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1711_09846_b200", "csrc")
FIT, EPS = 8e-6, 2.0 ** -24


def test_the_fit_is_as_good_as_it_says():
    """The coefficients as they stand in the source, in 64 bits, up to x = 10: erfc(10) / 2 = 1.04e-45 is below the smallest fp32 number, 2^-149 = 1.4e-45."""
    from scipy.special import erfcx
    with open(os.path.join(CSRC, "gated.cuh")) as f:
        body = f.read().split("float activation_bf16(int kind, float g) {")[1].split("\n}\n")[0]
    first = re.search(r"q = fmaf\((-?[\d.]+)f, t, (-?[\d.]+)f\);", body).groups()
    rest = re.findall(r"q = fmaf\(q, t, (-?[\d.]+)f\);", body)
    assert len(rest) == 4
    x = np.concatenate([np.linspace(0, 10, 400_001), np.geomspace(1e-30, 1e-3, 1001)])
    t = 1 / (1 + x / 2)
    q = np.polyval([float(np.float32(c)) for c in (*first, *rest)], t)
    off = np.abs(2 * t * np.exp2(q) / erfcx(x) - 1)
    assert off.max() <= FIT, off.max()


PROBE = '''
#include "gated.cuh"
namespace {
__global__ void k(const float* g, float* out, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) out[i] = pbt::gated::activation_bf16(pbt::gated::kGelu, g[i]);
}
}
extern "C" int probe(const float* g, float* out, int n) {
  k<<<(n + 255) / 256, 256>>>(g, out, n);
  return (int)cudaGetLastError();
}
'''

RUN = '''
    import ctypes as C, sys
    import torch
    lib = C.CDLL({library!r})
    halves = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()          # every bf16 number
    g = torch.cat([halves[halves.isfinite()], torch.linspace(-14, 14, 1_000_003)]).cuda()
    out = torch.full_like(g, float("nan"))
    assert lib.probe(C.c_void_p(g.data_ptr()), C.c_void_p(out.data_ptr()), g.numel()) == 0
    torch.cuda.synchronize()
    v = g.double()
    x = v.abs() * 0.5 ** 0.5
    tail = 0.5 * torch.special.erfcx(x) * torch.exp(-x * x)
    want = v * torch.where(v < 0, tail, 1 - tail)
    tol = v.abs() * (({fit} + (5.1 * x * x).clamp_max(1e4) * {eps} + 34 * {eps}) * tail + 2.0 ** -126) + 2 * {eps} * want.abs() + 2.0 ** -150
    off = (out.double() - want).abs()
    assert (off <= tol).all(), (g[off > tol][:9].tolist(), (off / tol)[off > tol].max().item())
'''


@pytest.mark.gpu
def test_the_kernels_function_is_off_by_the_fit_and_the_roundings(tmp_path):
    from paper_1711_09846_b200 import build
    (tmp_path / "probe.cu").write_text(PROBE)
    library = str(tmp_path / "probe.so")
    subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-shared", "-o", library, str(tmp_path / "probe.cu"), "-lcudart"], check=True, capture_output=True)
    code = textwrap.dedent(RUN).format(library=library, fit=FIT, eps=EPS)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
