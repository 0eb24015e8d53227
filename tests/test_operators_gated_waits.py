"""The gated units' bounded waits, made to run out: the kernels of a build whose waits try once give up in every role, wait for what they have in flight, and
leave PBT_ERR_TIMEOUT in the status words and a context that goes on."""
import os
import shutil
import subprocess
import sys
import textwrap
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STUBS = '''
#include "pbt_common.cuh"
namespace pbt {
void set_last_error(const char*) {}
bool serial_launches() { return true; }
}
'''

RUN = '''
    import ctypes as C, sys
    sys.path[:0] = [{root!r}, {tests!r}]
    import torch
    from paper_1711_09846_b200.binding import PbtGatedDesc
    lib = C.CDLL({library!r})
    ran_out = set()
    # few rows; tiles of one CTA, wide and narrow; pairs; a pass that keeps nothing
    for m, rows, width, hidden, keep in ((2, 3, 1024, 320, True), (3, 30, 2048, 128, True), (1, 100, 512, 256, True), (40, 120, 512, 512, True), (3, 600, 1024, 1024, True), (20, 512, 512, 512, False)):
        bf = dict(device="cuda", dtype=torch.bfloat16)
        x, w, dh = torch.randn(m, rows, width, **bf), torch.randn(m, 2 * hidden, width, **bf), torch.randn(m, rows, hidden, **bf)
        h, dx, dw = torch.zeros(m, rows, hidden, **bf), torch.zeros(m, rows, width, **bf), torch.zeros(m, 2 * hidden, width, **bf)
        kept, status = torch.zeros(m, rows, 2, hidden, device="cuda"), torch.zeros(8, device="cuda", dtype=torch.int32)
        d = PbtGatedDesc()
        d.members, d.rows, d.width, d.hidden, d.dtype = m, rows, width, hidden, 1
        d.x_row, d.x_member, d.weight_row, d.weight_member, d.dh_row, d.dh_member = width, rows * width, width, 2 * hidden * width, hidden, rows * hidden
        for name, v in dict(x=x, weight=w, dh=dh, h=h, dx=dx, dweight=dw, status_device=status, **(dict(kept=kept) if keep else dict())).items():
            setattr(d, name, v.data_ptr())
        for backward in (0, 1):
            status.zero_()
            size = C.c_size_t(0)
            assert lib.pbt_gated_query_workspace(C.byref(d), backward, C.byref(size)) == 0
            ws = torch.empty(max(size.value, 1), device="cuda", dtype=torch.uint8)
            call = lib.pbt_gated_backward if backward else lib.pbt_gated_forward
            assert call(C.byref(d), C.c_void_p(ws.data_ptr()), size, None) == 0
            torch.cuda.synchronize()
            words = status.tolist()
            assert words[4] in (0, 5) and words[:4] == [0] * 4, words
            if words[4]:
                ran_out.add((backward, words[5] // 10))
    assert {{k for k, _ in ran_out}} == {{0, 1}}, ran_out          # otherwise the waits did not run out, and this shows nothing
    assert (torch.ones(1000, device="cuda") * 2).sum().item() == 2000
'''
SOURCES = ("gated.cu", "gated_tc.cu", "gated_f32.cu", "dropout.cu", "stubs.cu")


@pytest.mark.gpu
def test_waits_that_run_out_leave_a_status_and_nothing_in_flight(tmp_path):
    """The products of the framework that a backward pass goes on with (gemm_tcgen05*.cu) keep their full limits."""
    from paper_1711_09846_b200 import build
    others = ("gemm_tcgen05.cu", "gemm_tcgen05_pair.cu")
    full = tmp_path / "full"
    full.mkdir()
    for name in os.listdir(build.CSRC):
        if name.endswith(".cuh"):
            shutil.copy(os.path.join(build.CSRC, name), tmp_path / name)
            shutil.copy(os.path.join(build.CSRC, name), full / name)
        elif name in SOURCES:
            shutil.copy(os.path.join(build.CSRC, name), tmp_path / name)
        elif name in others:
            shutil.copy(os.path.join(build.CSRC, name), full / name)
    common = tmp_path / "tc_common.cuh"
    text = common.read_text()
    assert text.count("constexpr uint32_t kSpinLimit = 1u << 22;") == 1
    common.write_text(text.replace("constexpr uint32_t kSpinLimit = 1u << 22;", "constexpr uint32_t kSpinLimit = 1u;"))
    (tmp_path / "stubs.cu").write_text(STUBS)

    def compile_one(path):
        flags = [f if f != build.CSRC else str(path.parent) for f in build.NVCC_FLAGS]
        subprocess.run([build._nvcc(), *flags, "-c", str(path), "-o", str(path) + ".o"], check=True, capture_output=True)
        return str(path) + ".o"
    with ThreadPoolExecutor(4) as pool:
        objects = list(pool.map(compile_one, [*(tmp_path / n for n in SOURCES), *(full / n for n in others)]))
    library = str(tmp_path / "short_waits.so")
    subprocess.run([build._nvcc(), "-shared", "-o", library, *objects, "-gencode", "arch=compute_100a,code=sm_100a", "-lcudart"], check=True, capture_output=True)
    code = textwrap.dedent(RUN).format(root=ROOT, tests=os.path.join(ROOT, "tests"), library=library)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
