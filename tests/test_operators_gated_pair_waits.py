"""The way out of a gated unit's CTA pair whose bounded waits ran out: what either CTA has in flight is waited for, load by load, however far apart
the two gave up; no kernel takes time that has passed for a copy that has landed."""
import glob
import os
import re
import shutil
import subprocess
import sys
import textwrap
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_operators_gated_waits import ROOT, SOURCES, STUBS

CSRC = os.path.join(ROOT, "paper_1711_09846_b200", "csrc")


def test_no_kernel_waits_by_the_clock():
    """A loop that sleeps looks at something in every turn."""
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        with open(path) as f:
            assert not re.search(r"\bfor\s*\([^;]*;[^;]*;[^;{}()]*\)\s*__nanosleep", f.read()), path


# a model of the barrier of one stage: (announcements, bytes of a CTA announced, bytes landed) of its loads, in halves of a stage
@pytest.mark.parametrize("stages", [2, 5])
def test_the_loads_that_one_of_the_two_lacks_are_settled(stages):
    """Leader and partner have issued a and b loads, at most a ring apart: with what settling adds, every load's phase is complete once what is in flight has landed."""
    for a in range(4 * stages):
        for b in range(max(0, a - stages), a + stages + 1):
            arrived = {i: 1 for i in range(a)}
            announced, landed = {i: 2 for i in range(a)}, {}
            for i in range(max(a, b)):
                landed[i] = (i < a) + (i < b)
            touched = set()
            for i in range(min(a, b), max(a, b)):      # (what the kernel does)
                assert i % stages not in touched        # no two loads of a stage are unsettled
                touched.add(i % stages)
                if i >= b:
                    landed[i] += 1
                else:
                    arrived[i], announced[i] = 1, 1
            assert all(arrived[i] == 1 and announced[i] == landed[i] for i in range(max(a, b))), (a, b)


RUN = '''
    import ctypes as C, sys
    sys.path.insert(0, {root!r})
    import torch
    from paper_1711_09846_b200.binding import PbtGatedDesc
    lib = C.CDLL({library!r})
    seen = 0
    for m, rows, width, hidden in ((3, 600, 1024, 1024), (20, 512, 512, 512), (2, 2048, 2048, 256), (8, 300, 200, 1000), (1, 4096, 128, 2048), (40, 512, 4096, 128)):
        bf = dict(device="cuda", dtype=torch.bfloat16)
        x, w, h = torch.randn(m, rows, width, **bf), torch.randn(m, 2 * hidden, width, **bf), torch.zeros(m, rows, hidden, **bf)
        kept, status = torch.zeros(m, rows, 2, hidden, device="cuda"), torch.zeros(8, device="cuda", dtype=torch.int32)
        d = PbtGatedDesc()
        d.members, d.rows, d.width, d.hidden, d.dtype = m, rows, width, hidden, 1
        d.x_row, d.x_member, d.weight_row, d.weight_member = width, rows * width, width, 2 * hidden * width
        for name, v in dict(x=x, weight=w, h=h, kept=kept, status_device=status).items():
            setattr(d, name, v.data_ptr())
        for _ in range(4):
            status.zero_()
            assert lib.pbt_gated_forward(C.byref(d), None, C.c_size_t(0), None) == 0
            torch.cuda.synchronize()
            words = status.tolist()
            assert words[4] in (0, 5) and words[:4] == [0] * 4, words
            seen += words[4] == 5
        assert lib.waits_that_ran_out_on_the_way_out() == 0
    assert seen >= {expected}, seen               # otherwise the waits did not run out, and this shows nothing
    assert (torch.ones(1000, device="cuda") * 2).sum().item() == 2000
'''
OUT = '''
extern "C" int waits_that_ran_out_on_the_way_out() {
  unsigned n = ~0u;
  cudaMemcpyFromSymbol(&n, pbt::tc::out_of_time, sizeof(n));
  return (int)n;
}
'''


@pytest.mark.gpu
@pytest.mark.parametrize("limit, expected", [(1, 6), (40, 0)])
def test_whatever_is_in_flight_lands_before_a_pair_ends(tmp_path, limit, expected):
    """Builds whose waits try once, or a few times: no wait on the way out runs out."""
    from paper_1711_09846_b200 import build
    for name in os.listdir(build.CSRC):
        if name.endswith(".cuh") or name in SOURCES or name in ("gemm_tcgen05.cu", "gemm_tcgen05_pair.cu"):
            shutil.copy(os.path.join(build.CSRC, name), tmp_path / name)
    common = tmp_path / "tc_common.cuh"
    text = common.read_text()
    spin, out = "constexpr uint32_t kSpinLimit = 1u << 22;", "__device__ __forceinline__ void mbar_wait_out("
    assert text.count(spin) == 1 and text.count(out) == 1
    at = text.index(out)
    end = text.index("\n}\n", at) + 3
    counted = '''static __device__ unsigned out_of_time;
__device__ __forceinline__ void mbar_wait_out(uint64_t* bar, uint32_t parity, uint32_t limit = 1u << 22) {
  uint32_t i = 0;
  for (; i < limit && !mbar_try_wait(bar, parity); ++i)
    if (i > 64) __nanosleep(64);
  if (i == limit) atomicAdd(&out_of_time, 1u);
}
'''
    common.write_text((text[:at] + counted + text[end:]).replace(spin, f"constexpr uint32_t kSpinLimit = {limit}u;"))
    tc = tmp_path / "gated_tc.cu"
    tc.write_text(tc.read_text() + OUT)
    (tmp_path / "stubs.cu").write_text(STUBS)

    def compile_one(name):
        flags = [f if f != build.CSRC else str(tmp_path) for f in build.NVCC_FLAGS]
        subprocess.run([build._nvcc(), *flags, "-c", str(tmp_path / name), "-o", str(tmp_path / name) + ".o"], check=True, capture_output=True)
        return str(tmp_path / name) + ".o"
    with ThreadPoolExecutor(4) as pool:
        objects = list(pool.map(compile_one, [*SOURCES, "gemm_tcgen05.cu", "gemm_tcgen05_pair.cu"]))
    library = str(tmp_path / "short_waits.so")
    subprocess.run([build._nvcc(), "-shared", "-o", library, *objects, "-gencode", "arch=compute_100a,code=sm_100a", "-lcudart"], check=True, capture_output=True)
    code = textwrap.dedent(RUN).format(root=ROOT, library=library, expected=expected)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
