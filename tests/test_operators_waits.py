"""The adapters' bounded waits, made to run out: the kernels of a build whose waits try once give up in every role, wait for what they have
in flight, and leave PBT_ERR_TIMEOUT in the status words and a context that goes on."""
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
    from paper_1711_09846_b200.binding import PbtAdapterDesc
    from test_operators_adapters import _case
    lib = C.CDLL({library!r})
    ran_out = set()
    for lengths, ids, k, n, rank, count in (([300, 41, 200], [1, 0, 1], 320, 264, 64, 2), ([2100, 3], [1, 0], 128, 72, 8, 2), ([128] * 5, [0, 1, 2, 3, 4], 256, 384, 16, 5),
                                            ([2] * 33, [j % 4 for j in range(33)], 33, 65, 1, 4), ([600, 400], [0, 1], 512, 512, 16, 2), ([700, 900], [0, 1], 1024, 4096, 48, 2)):
        for backward in (0, 1):
            c = _case("bfloat16", lengths, ids, k, n, rank, count)
            t = c["x"].shape[0]
            bf = dict(device="cuda", dtype=torch.bfloat16)
            y, s, dx = torch.zeros(t, n, **bf), torch.zeros(t, rank, device="cuda"), torch.zeros(t, k, **bf)
            d_a, d_b, status = torch.zeros(count, rank, k, device="cuda"), torch.zeros(count, n, rank, device="cuda"), torch.zeros(8, device="cuda", dtype=torch.int32)
            d = PbtAdapterDesc()
            d.rows, d.inputs, d.outputs, d.rank, d.n_adapters, d.n_segments, d.dtype = t, k, n, rank, count, len(ids), 1
            d.ld_weight, d.ld_x, d.ld_y, d.ld_dy, d.ld_dx = k, k, n, n, k
            for name, v in dict(c, y=y, s=s, dx=dx, dA=d_a, dB=d_b, status_device=status).items():
                if name != "segments":
                    setattr(d, name, v.data_ptr())
            size = C.c_size_t(0)
            assert lib.pbt_adapter_query_workspace(C.byref(d), backward, C.byref(size)) == 0
            ws = torch.empty(size.value, device="cuda", dtype=torch.uint8)
            call = lib.pbt_adapter_backward if backward else lib.pbt_adapter_forward
            assert call(C.byref(d), C.c_void_p(ws.data_ptr()), size, None) == 0
            torch.cuda.synchronize()
            words = status.tolist()
            assert words[4] in (0, 5) and words[:4] == [0] * 4, words
            if words[4]:
                ran_out.add(backward)
    assert ran_out == {{0, 1}}, ran_out          # otherwise the waits did not run out, and this shows nothing
    assert (torch.ones(1000, device="cuda") * 2).sum().item() == 2000
'''


@pytest.mark.gpu
def test_waits_that_run_out_leave_a_status_and_nothing_in_flight(tmp_path):
    from paper_1711_09846_b200 import build
    for name in os.listdir(build.CSRC):
        if name.endswith(".cuh") or name in ("adapters.cu", "adapters_tc.cu"):
            shutil.copy(os.path.join(build.CSRC, name), tmp_path / name)
    common = tmp_path / "tc_common.cuh"
    text = common.read_text()
    assert text.count("constexpr uint32_t kSpinLimit = 1u << 22;") == 1
    common.write_text(text.replace("constexpr uint32_t kSpinLimit = 1u << 22;", "constexpr uint32_t kSpinLimit = 1u;"))
    (tmp_path / "stubs.cu").write_text(STUBS)
    flags = [f if f != build.CSRC else str(tmp_path) for f in build.NVCC_FLAGS]

    def compile_one(name):
        subprocess.run([build._nvcc(), *flags, "-c", str(tmp_path / name), "-o", str(tmp_path / (name + ".o"))], check=True, capture_output=True)
        return str(tmp_path / (name + ".o"))
    with ThreadPoolExecutor(3) as pool:
        objects = list(pool.map(compile_one, ("adapters.cu", "adapters_tc.cu", "stubs.cu")))
    library = str(tmp_path / "short_waits.so")
    subprocess.run([build._nvcc(), "-shared", "-o", library, *objects, "-gencode", "arch=compute_100a,code=sm_100a", "-lcudart"], check=True, capture_output=True)
    code = textwrap.dedent(RUN).format(root=ROOT, tests=os.path.join(ROOT, "tests"), library=library)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
