"""Ways through the operators that the tests of the formulas do not take: long segment tables, operands beyond 32-bit offsets backwards,
transposed activations, several threads, captured graphs, and segment tables that make no sense between guarded buffers.  References and
tolerances are those of the formulas' tests."""
import ctypes as C
import os
import subprocess
import sys
import textwrap

import pytest

from test_operators_adapters import EPS32, _case, _verify

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# More segments than one list of the gradients' kernel holds (1024) and than one pass of the warps' search takes: adapters that occur in the
# first list only, in a later one only, in several, and not at all.
LONG_TABLES = {
    "single rows": ([1] * 2500, lambda k: 0 if k < 1000 else (k % 3) + 1 if k < 2100 else 4, 72, 136, 8, 6),
    "short segments": ([3, 1, 0, 5] * 400, lambda k: k % 7 - 1 if k < 1500 else 6, 264, 392, 12, 8),
    "wide": ([3] * 1300, lambda k: k % 2 if k < 1100 else 2, 1024, 512, 16, 3),
    "a long one behind many": ([1] * 1030 + [700], lambda k: int(k == 1030), 96, 200, 33, 2),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("name", sorted(LONG_TABLES))
def test_tables_of_more_than_a_thousand_segments(name, dtype):
    lengths, owner, *rest = LONG_TABLES[name]
    _verify(_case(dtype, lengths, [owner(k) for k in range(len(lengths))], *rest, seed=len(name), lead=2))


# The last rows of operands of more than 2^31 elements and 2^32 bytes.  fp32 sums of at most 2048 terms: 2048 eps of the magnitudes, which are
# below 64 times the largest value here; bf16 results carry their rounding, 2^-8.  dA and dB of the last adapter come from two rows.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("inputs, outputs", [(2048, 64), (64, 2048)])
def test_adapters_beyond_32_bit_offsets_both_ways(inputs, outputs, dtype):
    import torch
    import paper_1711_09846_b200 as pbt
    rows, dt = 1_100_000, getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(9)

    def normal(*shape, scale=1.0):
        return torch.empty(shape, device="cuda", dtype=dt).normal_(0.0, scale, generator=gen)

    x, dy, w = normal(rows, inputs), normal(rows, outputs), normal(outputs, inputs, scale=inputs ** -0.5)
    a, b = normal(2, 4, inputs, scale=inputs ** -0.5), normal(2, outputs, 4)
    where = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, rows - 2, rows], [0, 1])]
    layer = pbt.AdapterProjection(w, a, b, torch.tensor([1.0, 0.5], device="cuda"))
    y, kept = layer.forward(x, *where, keep=True)
    dx, d_a, d_b = layer.backward(dy, x, kept, *where)
    layer.check()
    xl, dl, w, a, b = (t.double().cpu() for t in (x[-2:], dy[-2:], w, a[1], b[1]))
    s, ds = xl @ a.T, 0.5 * dl @ b
    tol = 64 * 2048 * EPS32
    for name, got, want, rounding in (("y", y[-2:], xl @ w.T + 0.5 * s @ b.T, 1), ("dx", dx[-2:], dl @ w + ds @ a, 1), ("s", kept[-2:], s, 0),
                                      ("dA", d_a[1], ds.T @ xl, 0), ("dB", d_b[1], 0.5 * dl.T @ s, 0)):
        bound = (tol + (2.0 ** -8 if rounding and dtype == "bfloat16" else 0)) * want.abs().max()
        assert (got.double().cpu() - want).abs().max() <= bound, name


def _norm_run(d, dy, du):
    import paper_1711_09846_b200 as pbt
    kw = {k: d[k] for k in ("post_weight", "gate", "scale", "next_weight")}
    out = pbt.block_norm_forward(d["x"], d["block"], keep=True, **kw)
    g = pbt.block_norm_backward(dy, du, out.y, d["block"], rstd_block=out.rstd_block, rstd_next=out.rstd_next, **kw)
    return out, g


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("width", [7, 34, 64, 1001, 2048])
def test_norms_of_transposed_activations(width, dtype):
    """[rows, members, width] seen as [members, rows, width]: the row stride is larger than the member stride.  The same arithmetic as on
    contiguous activations, bit for bit."""
    import torch
    from test_operators_norm import _inputs
    d, dy, du = _inputs(3, 50, width, dtype, "full", seed=width)
    turn = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    flat = _norm_run(d, dy, du)
    turned = _norm_run({k: turn(v) if k in ("x", "block", "gate") else v for k, v in d.items()}, turn(dy), turn(du))
    for a, b in zip((*flat[0], *flat[1]), (*turned[0], *turned[1])):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["none", "vector", "full"])
@pytest.mark.parametrize("width", [7, 34, 64, 2048])
def test_norms_without_a_scale_are_those_with_ones(width, gate):
    import torch
    from test_operators_norm import _inputs
    d, dy, du = _inputs(2, 9, width, "bfloat16", gate, seed=width)
    with_ones = _norm_run({**d, "scale": torch.ones(2, device="cuda")}, dy, du)
    without = _norm_run({**d, "scale": None}, dy, du)
    assert without[1].dscale is None
    for a, b in zip((*with_ones[0], *with_ones[1][:-1]), (*without[0], *without[1][:-1])):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_threads_share_a_layer(dtype):
    import threading
    import torch
    import paper_1711_09846_b200 as pbt
    c = _case(dtype, [70, 1, 90], [0, 1, 1], 128, 200, 8, 2, seed=3)
    layer = pbt.AdapterProjection(c["weight"], c["A"], c["B"], c["scale"], bias=c["bias"])
    where = (c["row_offsets"], c["adapter_ids"])

    def step(x, dy, stream=None):
        y, kept = layer.forward(x, *where, keep=True, stream=stream)
        return (y, *layer.backward(dy, x, kept, *where, stream=stream))

    gen = torch.Generator(device="cuda").manual_seed(2)
    inputs = [[torch.randn(t.shape, generator=gen, device="cuda").to(t.dtype) for t in (c["x"], c["dy"])] for _ in range(4)]
    want = [step(*i) for i in inputs]
    torch.cuda.synchronize()
    got = [None] * 4

    def work(k):
        stream = torch.cuda.Stream()
        for _ in range(50):
            got[k] = step(*inputs[k], stream=stream)
        stream.synchronize()
    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    layer.check()
    for a, b in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.gpu
def test_the_first_calls_of_a_process_may_come_from_several_threads():
    code = '''
        import sys, threading
        sys.path[:0] = [{root!r}, {tests!r}]
        import torch
        import paper_1711_09846_b200 as pbt
        from test_operators_adapters import _case, _run, _reference, _close
        cases = [_case("bfloat16", [300, 200], [0, 1], 512, 512, 16, 2, seed=k) for k in range(6)]
        torch.cuda.synchronize()
        outs, together = [None] * 6, threading.Barrier(6)

        def work(k):
            together.wait()
            outs[k] = _run(cases[k])[1]
        threads = [threading.Thread(target=work, args=(k,)) for k in range(6)]
        for t in threads: t.start()
        for t in threads: t.join()
        for c, out in zip(cases, outs):
            ref = _reference(c)
            for name in ("y", "dx", "dA", "dB"):
                _close(name, out[name], ref, c)
        '''
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(code).format(root=ROOT, tests=os.path.join(ROOT, "tests"))], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_captured_graph_of_all_operators_replays_on_new_contents(dtype):
    import torch
    import paper_1711_09846_b200 as pbt
    from test_operators_norm import _inputs
    c = _case(dtype, [130, 1, 60, 9], [0, 1, 1, -1], 128, 200, 8, 2, seed=5)
    d, dy, du = _inputs(2, 50, 256, dtype, "vector", seed=6)
    grads = [torch.randn(n, device="cuda") for n in (70_001, 33, 4_000)]
    clipped = [torch.empty_like(g) for g in grads]
    layer = pbt.AdapterProjection(c["weight"], c["A"], c["B"], c["scale"], bias=c["bias"])
    clip = pbt.GradientClip(grads, [0, 1, 0], out=clipped)

    def step():
        where = (c["row_offsets"], c["adapter_ids"])
        y, kept = layer.forward(c["x"], *where, keep=True)
        out, g = _norm_run(d, dy, du)
        owned = kept[:131].clone()                      # (the rows that have an adapter)
        return [y, owned, *layer.backward(c["dy"], c["x"], kept, *where), *out, *g, clip.run(1.0), *clipped]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step()
    for seed in (1, 2):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for t in (c["x"], c["dy"], d["x"], d["block"], d["gate"], dy, du, *grads):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [r.clone() for r in results]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
    layer.check()


TABLES = [([0, 5000, 9000], [0, 1]), ([-7, 60, 150], [1, 99]), ([150, 20, 0], [0, 1]), ([-2 ** 31, 2 ** 31 - 1, -2 ** 31], [-2 ** 31, 2 ** 31 - 1]),
          ([0, 2 ** 31 - 1, 2 ** 31 - 1], [1, 1]), ([149, 150, 151], [0, 0]), ([0, 100, 50, 150, 20, 150], [0, 1, 0, 1, 0]), ([75] * 40, [k % 3 - 1 for k in range(39)]),
          ([(37 * k) % 151 for k in range(1201)], [k % 2 for k in range(1200)])]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("inputs, outputs, rank", [(128, 128, 8), (33, 65, 3), (512, 1024, 64)])
def test_no_segment_table_makes_a_kernel_write_beyond_its_results(inputs, outputs, rank, dtype):
    """Results and workspace lie between guards, inputs are compared: whatever the table holds, the calls write their results only."""
    import torch
    import paper_1711_09846_b200 as pbt
    from paper_1711_09846_b200.binding import PbtAdapterDesc
    lib, guard, pattern = pbt.load_library(), 4096, 0x5A
    c = _case(dtype, [90, 60], [0, 1], inputs, outputs, rank, 2)
    rows, element = 150, c["x"].element_size()
    status = torch.zeros(8, dtype=torch.int32, device="cuda")
    inputs_before = {k: c[k].clone() for k in ("x", "dy", "weight", "A", "B", "scale", "bias")}
    sizes = dict(y=rows * outputs * element, s=rows * rank * 4, dx=rows * inputs * element, dA=2 * rank * inputs * 4, dB=2 * rank * outputs * 4)

    def guarded(size):
        t = torch.full((size + 2 * guard + 512,), pattern, dtype=torch.uint8, device="cuda")
        lead = guard + -(t.data_ptr() + guard) % 256
        return t, lead, size

    for offsets, ids in TABLES:
        table = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (offsets, ids)]
        buffers = {k: guarded(v) for k, v in sizes.items()}
        d = PbtAdapterDesc()
        d.rows, d.inputs, d.outputs, d.rank, d.n_adapters, d.n_segments, d.dtype = rows, inputs, outputs, rank, 2, len(ids), int(dtype == "bfloat16")
        d.ld_weight, d.ld_x, d.ld_y, d.ld_dy, d.ld_dx = inputs, inputs, outputs, outputs, inputs
        for k in ("x", "dy", "weight", "A", "B", "scale", "bias"):
            setattr(d, k, c[k].data_ptr())
        for k, (t, lead, _) in buffers.items():
            setattr(d, k, t.data_ptr() + lead)
        d.row_offsets, d.adapter_ids, d.status_device = table[0].data_ptr(), table[1].data_ptr(), status.data_ptr()
        for backward, call in ((0, lib.pbt_adapter_forward), (1, lib.pbt_adapter_backward)):
            n = C.c_size_t(0)
            assert lib.pbt_adapter_query_workspace(C.byref(d), backward, C.byref(n)) == 0
            buffers[f"workspace {backward}"] = ws = guarded(n.value)
            assert call(C.byref(d), ws[0].data_ptr() + ws[1], n.value, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        for k, (t, lead, size) in buffers.items():
            assert (t[:lead] == pattern).all() and (t[lead + size:] == pattern).all(), (k, offsets)
        for k, v in inputs_before.items():
            assert torch.equal(c[k], v), (k, offsets)
        assert table[0].tolist() == list(offsets) and table[1].tolist() == list(ids)
        assert status.tolist() == [0] * 8
