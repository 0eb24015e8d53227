"""Low-rank adapters beside a shared projection (AdapterProjection / pbt_adapter_*) against the formulas in 64 bits.

Tolerances, from the magnitudes that the reference returns beside the values (the same sums over absolute values).
eps = 2^-24.  fp32 sums, whatever their order, of n terms are within n eps of the sum of magnitudes; the longest
sequential chain of any of the kernels is taken as (inputs + outputs) / 16 + rows / 4 + 64 terms.  A bf16 result is rounded
once (2^-8 of its value); its low-rank part may also hold S or dS rounded to bf16 before the second product (2^-8 of that
part's magnitude).  dA and dB are fp32 and are allowed the chain twice (dS or S, then the sum over rows)."""
import ctypes as C

import pytest

EPS32 = 2.0 ** -24


def _case(dtype, lengths, ids, inputs, outputs, rank, adapters, seed=0, pad=0, lead=0):
    """Inputs; `pad` gives rows a stride of their own, `lead` rows in front of the first segment have none."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = getattr(torch, dtype)
    rows = lead + sum(lengths)

    def draw(*shape, scale=1.0, wide=0):
        t = torch.randn(*shape[:-1], shape[-1] + wide, generator=gen).mul_(scale).to(dt).cuda()
        return t[..., :shape[-1]]
    at = [lead]
    for n in lengths:
        at.append(at[-1] + n)
    return dict(x=draw(rows, inputs, wide=pad), dy=draw(rows, outputs, scale=0.1, wide=pad),
                weight=draw(outputs, inputs, scale=inputs ** -0.5, wide=pad), A=draw(adapters, rank, inputs, scale=inputs ** -0.5),
                B=draw(adapters, outputs, rank, scale=rank ** -0.5), scale=(torch.rand(adapters, generator=gen) * 2 - 0.5).cuda(),
                bias=torch.randn(outputs, generator=gen).cuda(), row_offsets=torch.tensor(at, dtype=torch.int32).cuda(),
                adapter_ids=torch.tensor(ids, dtype=torch.int32).cuda(), segments=list(zip(at[:-1], at[1:], ids)))


def _reference(c, backward=True):
    """{name: (value, magnitude)} in 64 bits on the CPU; low: the magnitude of the low-rank part alone."""
    import torch
    f = {k: v.cpu().double() for k, v in c.items() if k != "segments"}
    x, w, a, b, s, dy = (f[k] for k in ("x", "weight", "A", "B", "scale", "dy"))
    y, ym = x @ w.T + f["bias"], x.abs() @ w.abs().T + f["bias"].abs()
    dx, dxm = dy @ w, dy.abs() @ w.abs()
    ylow, dxlow = torch.zeros_like(y), torch.zeros_like(dx)
    S, Sm = torch.zeros(x.shape[0], a.shape[1]).double(), torch.zeros(x.shape[0], a.shape[1]).double()
    dA, dAm, dB, dBm = (torch.zeros_like(t) for t in (a, a, b, b))
    for lo, hi, i in c["segments"]:
        if not 0 <= i < a.shape[0]:
            continue
        r, k = slice(lo, hi), s[i].abs()
        S[r], Sm[r] = x[r] @ a[i].T, x[r].abs() @ a[i].abs().T
        y[r] += s[i] * S[r] @ b[i].T
        ylow[r] = k * Sm[r] @ b[i].abs().T
        ds, dsm = s[i] * dy[r] @ b[i], k * dy[r].abs() @ b[i].abs()
        dx[r] += ds @ a[i]
        dxlow[r] = dsm @ a[i].abs()
        dA[i] += ds.T @ x[r]
        dAm[i] += dsm.T @ x[r].abs()
        dB[i] += s[i] * dy[r].T @ S[r]
        dBm[i] += k * dy[r].abs().T @ Sm[r]
    return dict(y=(y, ym + ylow, ylow), s=(S, Sm, None), dx=(dx, dxm + dxlow, dxlow), dA=(dA, dAm, None), dB=(dB, dBm, None))


def _close(name, got, ref, c, rows=None):
    import torch
    value, mag, low = ref[name]
    t, k = c["x"].shape
    chain = ((k + c["weight"].shape[0]) / 16 + t / 4 + 64) * EPS32
    tol = chain * (2 if name in ("dA", "dB") else 1) * mag
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (value.abs() + low) + 1e-38
    g = got.cpu().double()
    assert g.shape == value.shape
    if rows is not None:
        g, value, tol = g[rows], value[rows], tol[rows]
    bad = ~((g - value).abs() <= tol)
    assert not bad.any(), (name, ((g - value).abs() / tol.clamp_min(1e-300)).max().item(), int(bad.sum()))


def _owned(c):
    """Rows that have an adapter."""
    import torch
    m = torch.zeros(c["x"].shape[0], dtype=torch.bool)
    for lo, hi, i in c["segments"]:
        if 0 <= i < c["A"].shape[0]:
            m[lo:hi] = True
    return m


def _run(c, stream=None):
    import paper_1711_09846_b200 as pbt
    layer = pbt.AdapterProjection(c["weight"], c["A"], c["B"], c["scale"], bias=c["bias"])
    where = (c["row_offsets"], c["adapter_ids"])
    y, kept = layer.forward(c["x"], *where, keep=True, stream=stream)
    dx, d_a, d_b = layer.backward(c["dy"], c["x"], kept, *where, stream=stream)
    layer.check()
    return layer, dict(y=y, s=kept, dx=dx, dA=d_a, dB=d_b)


def _verify(c):
    import torch
    layer, out = _run(c)
    ref = _reference(c)
    for name in ("y", "dx", "dA", "dB"):
        _close(name, out[name], ref, c)
    _close("s", out["s"], ref, c, _owned(c))
    only = layer.forward(c["x"], c["row_offsets"], c["adapter_ids"])
    assert torch.equal(only, out["y"])         # keeping S changes nothing
    return out


# (segment lengths, adapter ids, inputs, outputs, rank, adapters)
CASES = {
    "one row": ([1], [0], 64, 64, 8, 1),
    "one column": ([3, 2], [1, 0], 1, 1, 1, 2),
    "tiny odd": ([2, 3, 1], [0, 1, 0], 7, 5, 3, 2),
    "no adapter at all": ([40, 30], [-1, -1], 64, 72, 8, 2),
    "single tokens": ([1] * 9, [2, -1, 0, 1, 2, 2, 0, 1, -1], 128, 136, 16, 3),
    "single tokens, many": ([1] * 70, [(7 * k) % 13 - 1 for k in range(70)], 264, 392, 8, 12),
    "empty segments": ([0, 5, 0, 0, 130, 0, 1, 0], [0, 1, 2, 0, 2, 1, 0, 2], 96, 160, 16, 3),
    "shared adapters": ([33, 64, 1, 127, 65], [1, 0, 1, 1, 0], 200, 256, 16, 4),
    "an id out of range": ([20, 20], [5, 1], 64, 64, 8, 2),
    "equal members": ([128] * 5, [0, 1, 2, 3, 4], 256, 384, 16, 5),
    "rank 64": ([300, 41], [1, 0], 320, 264, 64, 2),
    "rank 24": ([70, 200], [1, 0], 136, 520, 24, 2),
    "rank 4": ([257, 3], [0, 1], 784, 512, 4, 2),
    "odd widths": ([150, 77], [0, 1], 333, 259, 12, 2),
    "one odd width": ([150, 77], [1, 0], 512, 259, 16, 2),
    "long": ([1100, 300, 13], [0, 1, 0], 512, 640, 8, 2),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("name", list(CASES))
def test_forward_and_backward_match_the_formulas(name, dtype):
    _verify(_case(dtype, *CASES[name], seed=len(name)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad", [1, 8])
def test_row_strides_and_rows_outside_every_segment(pad, dtype):
    lengths, ids, *rest = CASES["shared adapters"]
    _verify(_case(dtype, lengths, ids, *rest, seed=pad, pad=pad, lead=5))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lengths", [[1] * 12, [130, 60, 3, 200]], ids=["tokens", "ragged"])
def test_a_diverged_adapter_reaches_no_other_row(lengths, dtype):
    import torch
    ids = [k % 3 for k in range(len(lengths))]
    c = _case(dtype, lengths, ids, 192, 256, 16, 3, seed=3)
    _, clean = _run(c)
    c["A"][1, 3, 7] = float("nan")
    c["B"][1, 5, 2] = float("inf")
    mine = torch.zeros(c["x"].shape[0], dtype=torch.bool)
    for lo, hi, i in c["segments"]:
        if i == 1:
            mine[lo:hi] = True
    _, out = _run(c)
    for name in ("y", "dx", "s"):
        assert torch.equal(out[name][~mine.cuda()], clean[name][~mine.cuda()]), name
    assert torch.isnan(out["y"][mine.cuda()]).any(1).all() and torch.isnan(out["dx"][mine.cuda()]).any(1).all()
    for name in ("dA", "dB"):
        assert torch.equal(out[name][[0, 2]], clean[name][[0, 2]]), name
    # and a row that holds NaN stays alone, in the gradients of the other adapters too
    c = _case(dtype, lengths, ids, 192, 256, 16, 3, seed=3)
    lo, hi, _ = c["segments"][1]
    c["x"][lo, 0] = float("nan")
    c["dy"][hi - 1, 3] = float("inf")
    _, out = _run(c)
    others = torch.ones(c["x"].shape[0], dtype=torch.bool)
    others[lo:hi] = False
    for name in ("y", "dx", "s"):
        assert torch.equal(out[name][others.cuda()], clean[name][others.cuda()]), name
    for name in ("dA", "dB"):
        assert torch.equal(out[name][[0, 2]], clean[name][[0, 2]]), name
        assert not torch.isfinite(out[name][1]).all(), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_no_rows(dtype):
    c = _case(dtype, [0, 0], [0, 1], 64, 64, 8, 2)
    _, out = _run(c)
    assert out["y"].shape == (0, 64) and out["dx"].shape == (0, 64)
    assert (out["dA"] == 0).all() and (out["dB"] == 0).all()


@pytest.mark.gpu
def test_segment_tables_that_make_no_sense_stay_inside_the_buffers():
    """Offsets beyond the rows and ids beyond the adapters are clamped (what the rows hold then is unspecified): the
    results' neighbours in memory stay as they were."""
    import torch
    import paper_1711_09846_b200 as pbt
    for dtype in ("float32", "bfloat16"):
        c = _case(dtype, [90, 60], [0, 1], 128, 128, 8, 2)
        for offsets, ids in (([0, 5000, 9000], [0, 1]), ([-7, 60, 150], [1, 99]), ([150, 20, 0], [0, 1])):
            layer = pbt.AdapterProjection(c["weight"], c["A"], c["B"], c["scale"])
            where = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (offsets, ids)]
            y, kept = layer.forward(c["x"], *where, keep=True)
            layer.backward(c["dy"], c["x"], torch.zeros_like(kept), *where)
        torch.cuda.synchronize()
        _verify(c)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_runs_are_reproducible_and_another_stream_gives_the_same_bits(dtype):
    import torch
    c = _case(dtype, [200, 1, 90, 300], [0, 1, 1, 0], 256, 320, 16, 2, seed=8)
    _, first = _run(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        _, out = _run(c, stream)
        torch.cuda.synchronize()
        for name in first:
            assert torch.equal(first[name], out[name]), name


@pytest.mark.gpu
def test_gradients_agree_with_differences_of_the_forward_pass():
    """Loss sum(y dy) in fp32: it is bilinear in (A, B) and linear in x, so a central difference along one tensor is exact
    up to the forward pass's rounding, about 1e-6 of a loss of order 100 over a step of 2: 2e-4 of the largest."""
    import torch
    import paper_1711_09846_b200 as pbt
    c = _case("float32", [30, 50, 20], [0, 1, 0], 48, 56, 8, 2, seed=2)
    _, out = _run(c)

    def loss(**kw):
        e = {**c, **kw}
        y = pbt.AdapterProjection(e["weight"], e["A"], e["B"], e["scale"], bias=e["bias"]).forward(e["x"], e["row_offsets"], e["adapter_ids"])
        return (y.double() * c["dy"].double()).sum().item()
    gen = torch.Generator(device="cuda").manual_seed(1)
    pairs = []
    for key, grad in (("x", "dx"), ("A", "dA"), ("B", "dB")):
        v = torch.randn(c[key].shape, generator=gen, device="cuda")
        diff = (loss(**{key: c[key] + v}) - loss(**{key: c[key] - v})) / 2
        pairs.append((key, diff, (out[grad].double() * v.double()).sum().item()))
    largest = max(abs(p[2]) for p in pairs)
    for key, diff, exact in pairs:
        assert abs(diff - exact) <= 2e-4 * max(largest, 100.0), pairs


def test_the_written_out_gradients_are_those_of_autograd(monkeypatch):
    """Pins the reference above (CPU, 64 bits) to automatic differentiation of the forward formula."""
    import torch
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self, *a, **k: self)
    c = _case("float32", [3, 0, 4], [1, 0, 1], 6, 5, 2, 2)
    f = {k: c[k].double().requires_grad_() for k in ("x", "A", "B")}
    y = f["x"] @ c["weight"].double().T + c["bias"].double()
    low = torch.zeros_like(y)
    for lo, hi, i in c["segments"]:
        low = low + torch.nn.functional.pad(c["scale"][i].double() * f["x"][lo:hi] @ f["A"][i].T @ f["B"][i].T, (0, 0, lo, y.shape[0] - hi))
    y = y + low
    (y * c["dy"].double()).sum().backward()
    ref = _reference(c)
    assert torch.allclose(ref["y"][0], y.detach())
    for name, key in (("dx", "x"), ("dA", "A"), ("dB", "B")):
        assert torch.allclose(ref[name][0], f[key].grad)


@pytest.mark.gpu
def test_adapter_refusals():
    import torch
    import paper_1711_09846_b200 as pbt
    c = _case("bfloat16", [4, 5], [0, 1], 32, 48, 8, 2)
    good = dict(weight=c["weight"], A=c["A"], B=c["B"], scale=c["scale"], bias=c["bias"])
    pbt.AdapterProjection(**good)
    for kw in (dict(weight=c["weight"].float()), dict(weight=c["weight"].cpu()), dict(weight=c["weight"].half()), dict(weight=c["weight"].T),
               dict(A=c["A"][:, :, :16]), dict(A=c["A"].transpose(0, 1)), dict(B=c["B"][:1]), dict(B=c["B"].float()),
               dict(scale=c["scale"].double()), dict(scale=c["scale"][:1]), dict(bias=c["bias"][:5])):
        with pytest.raises(ValueError):
            pbt.AdapterProjection(**{**good, **kw})
    wide = _case("bfloat16", [4], [0], 128, 128, 65, 1)
    with pytest.raises(pbt.PbtError):
        pbt.AdapterProjection(wide["weight"], wide["A"], wide["B"], wide["scale"])
    layer = pbt.AdapterProjection(**good)
    o, i = c["row_offsets"], c["adapter_ids"]
    for args in ((c["x"][:, :16], o, i), (c["x"].float(), o, i), (c["x"], o.long(), i), (c["x"], o[:-1], i), (c["x"], o, i.cpu()),
                 (c["x"][0], o, i), (torch.zeros(9, 64, device="cuda", dtype=torch.bfloat16)[:, ::2], o, i)):
        with pytest.raises(ValueError):
            layer.forward(*args)
    y, kept = layer.forward(c["x"], o, i, keep=True)
    for args in ((c["dy"][:3], c["x"], kept, o, i), (c["dy"].float(), c["x"], kept, o, i), (c["dy"], c["x"], kept[:, :4], o, i),
                 (c["dy"], c["x"], kept.bfloat16(), o, i)):
        with pytest.raises(ValueError):
            layer.backward(*args)


def test_adapter_arguments_are_checked_before_the_device_is_touched():
    import paper_1711_09846_b200 as pbt
    from paper_1711_09846_b200.binding import PbtAdapterDesc
    lib = pbt.load_library()
    n = C.c_size_t(0)

    def desc(**kw):
        d = PbtAdapterDesc()
        d.rows, d.inputs, d.outputs, d.rank, d.n_adapters, d.n_segments = 10, 32, 64, 8, 3, 2
        for name in ("weight", "A", "B", "scale", "row_offsets", "adapter_ids", "x", "y", "s", "dy", "dx", "dA", "dB"):
            setattr(d, name, 4096)
        d.ld_weight = d.ld_x = d.ld_dx = 32
        d.ld_y = d.ld_dy = 64
        for k, v in kw.items():
            setattr(d, k, v)
        return d
    for backward in (0, 1):
        assert lib.pbt_adapter_query_workspace(C.byref(desc()), backward, C.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    assert lib.pbt_adapter_query_workspace(C.byref(desc()), 0, None) == 1
    for kw, code in ((dict(rows=-1), 1), (dict(inputs=0), 1), (dict(outputs=0), 1), (dict(rank=0), 2), (dict(rank=65), 2), (dict(dtype=2), 2),
                     (dict(n_adapters=0), 1), (dict(n_segments=-1), 1), (dict(weight=None), 1), (dict(A=None), 1), (dict(B=None), 1),
                     (dict(dtype=1), 1), (dict(scale=None), 1), (dict(row_offsets=None), 1), (dict(adapter_ids=None), 1), (dict(ld_weight=31), 1)):
        assert lib.pbt_adapter_forward(C.byref(desc(**kw)), None, 0, None) == code, kw
        assert lib.pbt_adapter_backward(C.byref(desc(**kw)), None, 0, None) == code, kw
        assert lib.pbt_last_error(None)
    for kw in (dict(x=None), dict(y=None), dict(ld_x=31), dict(ld_y=63)):
        assert lib.pbt_adapter_forward(C.byref(desc(**kw)), None, 0, None) == 1, kw
    for kw in (dict(x=None), dict(s=None), dict(dy=None), dict(dx=None), dict(dA=None), dict(dB=None), dict(ld_dy=63), dict(ld_dx=31)):
        assert lib.pbt_adapter_backward(C.byref(desc(**kw)), None, 0, None) == 1, kw
    assert lib.pbt_adapter_forward(C.byref(desc()), None, 0, None) == 3
    assert lib.pbt_adapter_backward(C.byref(desc()), None, 0, None) == 3
    assert lib.pbt_adapter_forward(None, None, 0, None) == 1
    assert lib.pbt_adapter_forward(C.byref(desc(rows=0)), None, 0, None) == 0


# Every way through the kernels: several CTAs of rows in the few-rows kernel, wide and narrow fp32 tiles with many segments,
# rows split between CTAs in the gradients, ranks dealt to parts, all operands packed at once.
WAYS = {
    "single tokens, several row groups": ([1] * 150, [(5 * k) % 11 - 1 for k in range(150)], 264, 392, 16, 10),
    "single tokens, largest rank": ([1] * 40, [(3 * k) % 7 for k in range(40)], 136, 296, 64, 7),
    "short segments in wide tiles": ([5] * 140, [(3 * k) % 9 - 1 for k in range(140)], 96, 520, 12, 8),
    "one long adapter": ([2100, 3], [1, 0], 128, 72, 8, 2),
    "one long adapter, largest rank": ([1500, 70], [0, 1], 72, 136, 64, 2),
    "odd rank of many parts": ([90, 200], [1, 0], 80, 64, 61, 2),
    "everything unaligned": ([60, 1, 139], [2, 0, 1], 131, 77, 13, 3),
    "rank one, many segments": ([2] * 33, [k % 4 for k in range(33)], 33, 65, 1, 4),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("name", sorted(WAYS))
def test_every_way_through_the_kernels_matches_the_formulas(name, dtype):
    lengths, ids, inputs, outputs, rank, adapters = WAYS[name]
    for lead in (0, 3):
        _verify(_case(dtype, lengths, ids, inputs, outputs, rank, adapters, seed=len(name), lead=lead))


# The product kernel's low-rank operand: with W = 0 the result is the low-rank part alone, and its error is that of its own rounding to
# bf16.  An operand that is held to 2^-16 adds less than 2^-7 of that error, independently: 2^-15 of its root mean square; the fp32 sums add
# less.  One per cent covers both.  An operand of 8 bits, whose error is as large as the result's, adds about 40 %.
@pytest.mark.gpu
@pytest.mark.parametrize("rank", [4, 16, 29, 32, 33, 48, 64])
def test_the_low_rank_part_of_a_bf16_product_has_the_error_of_its_rounding(rank):
    import torch
    c = _case("bfloat16", [300, 30, 70], [1, 0, 1], 512, 512, rank, 2, seed=rank)      # (too many rows for the few-rows kernel)
    c["weight"].zero_()
    c["bias"].zero_()
    _, out = _run(c)
    ref = _reference(c)
    for name in ("y", "dx"):
        value = ref[name][0]
        got, rounded = ((t.cpu().double() - value).square().mean().sqrt().item() for t in (out[name], value.to(torch.bfloat16)))
        assert got <= 1.01 * rounded, (name, got / rounded)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [40, 400])
def test_a_low_rank_operand_at_the_end_of_the_range(rows):
    """S beyond the largest bf16 but not the largest float, and infinite S: the products are those of the formula."""
    import torch
    import paper_1711_09846_b200 as pbt
    k = n = 512
    x = torch.zeros(rows, k, device="cuda", dtype=torch.bfloat16)
    x[:, :2] = 1.0
    a = torch.zeros(1, 8, k, device="cuda", dtype=torch.bfloat16)
    a[0, 0, 0], a[0, 0, 1] = 3.3895313892515355e38, 1e36
    b = torch.zeros(1, n, 8, device="cuda", dtype=torch.bfloat16)
    b[0, :, 0] = 2.0 ** -126
    w = torch.zeros(n, k, device="cuda", dtype=torch.bfloat16)
    where = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, rows], [0])]
    layer = pbt.AdapterProjection(w, a, b, torch.ones(1, device="cuda"))
    y, kept = layer.forward(x, *where, keep=True)
    assert torch.isfinite(kept).all()
    want = (a[0, 0, 0].double() + a[0, 0, 1].double()) * 2.0 ** -126
    assert (y.double() / want - 1).abs().max() <= 2.0 ** -8
    dy = torch.zeros(rows, n, device="cuda", dtype=torch.bfloat16)
    dy[0, 0] = 2.0 ** -10
    _, _, d_b = layer.backward(dy, x, kept, *where)
    assert torch.isfinite(d_b).all() and abs(d_b[0, 0, 0].double() / (kept[0, 0].double() * 2.0 ** -10) - 1) <= 2.0 ** -20
    a[0, 0, 1] = 3.3895313892515355e38
    y, kept = layer.forward(x, *where, keep=True)
    assert torch.isinf(kept[:, 0]).all() and torch.isinf(y).all()
    layer.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rank", [4, 16, 13])
def test_calls_that_follow_one_another_read_their_own_low_rank_rows(rank, dtype):
    """Calls without a pause share a workspace, and the product begins while the shrink writes it: bit for bit what a call alone gives."""
    import torch
    import paper_1711_09846_b200 as pbt
    n = 60
    c = _case(dtype, [1] * n, [(3 * k) % 11 - 1 for k in range(n)], 72, 200, rank, 10, seed=rank)
    layer = pbt.AdapterProjection(c["weight"], c["A"], c["B"], c["scale"], bias=c["bias"])
    gen = torch.Generator(device="cuda").manual_seed(1)
    xs = [torch.randn(c["x"].shape, generator=gen, device="cuda").to(c["x"].dtype) for _ in range(40)]
    alone = []
    for x in xs:
        alone.append(layer.forward(x, c["row_offsets"], c["adapter_ids"]))
        torch.cuda.synchronize()
    together = [layer.forward(x, c["row_offsets"], c["adapter_ids"]) for x in xs]
    layer.check()
    assert all(torch.equal(a, b) for a, b in zip(alone, together))


@pytest.mark.gpu
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("current", [False, True])
def test_the_status_words_outlive_a_call_on_another_stream(current, backward):
    """The kernels hold their address: with the layer gone, its words are nobody else's memory before the other stream is done."""
    import torch
    import paper_1711_09846_b200 as pbt
    c = _case("bfloat16", [40, 60], [0, 1], 64, 64, 8, 2)
    where = (c["row_offsets"], c["adapter_ids"])
    layer = pbt.AdapterProjection(c["weight"], c["A"], c["B"], c["scale"])
    _, kept = layer.forward(c["x"], *where, keep=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)       # a tenth of a second
    with torch.cuda.stream(side if current else None):
        stream = None if current else side
        if backward:
            layer.backward(c["dy"], c["x"], kept, *where, stream=stream)
        else:
            layer.forward(c["x"], *where, stream=stream)
    at = layer._status.data_ptr()
    del layer
    others = [torch.zeros(8, dtype=torch.int32, device="cuda") for _ in range(200)]
    assert not side.query()
    assert at not in [t.data_ptr() for t in others]
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("inputs, outputs", [(1, 40), (24, 1), (1, 1)])
def test_a_weight_of_one_row_or_column_may_have_any_stride_across_it(inputs, outputs, dtype):
    import torch
    c = _case(dtype, [30, 50], [1, 0], inputs, outputs, 4, 2, seed=inputs)
    w = c["weight"]
    _, whole = _run(c)
    for strides in (((1, 7), (3, 5)) if inputs == 1 else ((0, 1), (1, 1))):
        c["weight"] = torch.empty(4096, device="cuda", dtype=w.dtype).as_strided((outputs, inputs), strides).copy_(w)
        _, out = _run(c)
        assert all(torch.equal(out[name], whole[name]) for name in whole)
