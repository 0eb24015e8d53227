"""Gated units (GatedUnit) against the formulas in 64 bits.

Tolerances.  eps = 2^-24.  A product of n terms is off by at most (n + 16) eps of the sum of its terms' magnitudes, in whatever order it is
added, on the ALUs or the tensor cores (which cut 2^-23 of a partial sum once for every 16 terms).  act and act' come from an
exponential whose relative error is (|g| + 4) 2^-22 or an error function good to some ulp: off by at most 64 eps (1 + |g|) for arguments like
these (|g| < 10), and by their slopes, at most 1.13 (act) and 1 (act'), times the error of g.  relu's slope may be either one where g is
nearer to 0 than its error.  A bf16 result adds its rounding, 2^-8 of the value; dg and du of a bf16 pass are rounded the same way before they are multiplied."""
import ctypes as C

import pytest

from test_operators_dropout import scales

EPS32 = 2.0 ** -24
SEED = 0x123456789ABCDEF0


def _case(m, rows, width, hidden, dtype, pad=0, drop=True, shared=False, seed=0):
    import torch
    import paper_1711_09846_b200 as pbt
    gen = torch.Generator().manual_seed(seed)
    dt = getattr(torch, dtype)

    def rand(a, b, c, scale=1.0):
        t = torch.randn(a, b + (1 if pad else 0), c + pad, generator=gen).mul_(scale).to(dt).cuda()
        return t[:, :b, :c]                    # strides of their own when padded
    weight = rand(1 if shared else m, 2 * hidden, width, 1.5 * width ** -0.5)
    c = dict(x=rand(m, rows, width), weight=weight.expand(m, -1, -1) if shared else weight, dh=rand(m, rows, hidden, 0.1), dropout=None, scale=None)
    if drop:
        rate, step = (torch.rand(m, generator=gen) * 0.6).cuda(), torch.randint(0, 1 << 31, (m,), generator=gen).cuda()
        c["dropout"] = pbt.Dropout(rate, SEED, step, site=1, first_member=2)
        c["scale"] = torch.from_numpy(scales(m, rows, hidden, rate.cpu().numpy(), SEED, step.cpu().numpy(), 1, 2)).cuda()
    return c


def _act(kind, g):
    """act(g) and act'(g) in 64 bits."""
    import torch
    if kind == "relu":
        return g.clamp_min(0), (g > 0).double()
    if kind == "gelu":
        cdf = torch.special.ndtr(g)
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / (2 * torch.pi) ** 0.5
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if kind == "sigmoid" else (g * s, s + g * s * (1 - s))


def formulas(c, kind):
    """{name: (value, tolerance without the result's own rounding)} of h, dx and dweight."""
    import torch
    x, w, dh = (c[k].double() for k in ("x", "weight", "dh"))
    f = torch.ones((), device=x.device, dtype=torch.float64) if c["scale"] is None else c["scale"]
    bf = 2.0 ** -8 if c["x"].dtype == torch.bfloat16 else 0.0
    width, hidden = x.shape[2], w.shape[1] // 2
    g, u = (x @ w.transpose(1, 2)).chunk(2, -1)
    eg, eu = ((width + 16) * EPS32 * (x.abs() @ w.abs().transpose(1, 2))).chunk(2, -1)
    act, slope = _act(kind, g)
    own = 64 * EPS32 * (1 + g.abs())
    ea = 1.13 * eg + own
    es = eg + own + ((g.abs() <= eg).double() if kind == "relu" else 0.0)
    near = 16 * EPS32
    out = {"h": (f * act * u, f * (ea * u.abs() + (act.abs() + ea) * eu + near * (act * u).abs()))}
    d = f * dh
    dz = torch.cat([d * u * slope, d * act], -1)
    ez = torch.cat([d.abs() * (es * u.abs() + (slope.abs() + es) * eu), d.abs() * ea], -1) + near * dz.abs()
    ez = ez + bf * (dz.abs() + ez)
    out["dx"] = (dz @ w, ez @ w.abs() + (2 * hidden + 16) * EPS32 * ((dz.abs() + ez) @ w.abs()))
    out["dweight"] = (dz.transpose(1, 2) @ x, ez.transpose(1, 2) @ x.abs() + (x.shape[1] + 16) * EPS32 * ((dz.abs() + ez).transpose(1, 2) @ x.abs()))
    return out


def _run(c, kind, keep=True, layer=None, **kw):
    import paper_1711_09846_b200 as pbt
    layer = layer or pbt.GatedUnit(c["weight"], kind)
    h = layer.forward(c["x"], dropout=c["dropout"], keep=keep, **kw)
    h, kept = h if keep else (h, None)
    dx, dweight = layer.backward(c["dh"], c["x"], kept, dropout=c["dropout"], **kw)
    return {"h": h, "dx": dx, "dweight": dweight}, layer


def _verify(c, kind, got=None):
    import torch
    want = formulas(c, kind)
    layer = None
    if got is None:
        got, layer = _run(c, kind)
    for name, (value, tol) in want.items():
        r = got[name]
        assert r.shape == value.shape and r.is_contiguous() and r.dtype == c["x"].dtype
        if r.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (value.abs() + tol)
        off = (r.double() - value).abs()
        assert (off <= tol + 1e-38).all(), (name, (off / (tol + 1e-38)).max().item())
    if c["scale"] is not None and kind != "relu":
        assert (got["h"][c["scale"] == 0] == 0).all()
    if layer is not None:
        layer.check()
    return got


SHAPES = [(1, 1, 1, 1), (1, 1, 8, 8), (2, 3, 7, 5), (1, 5, 64, 64), (3, 17, 100, 33), (1, 64, 256, 128), (1, 65, 256, 136), (2, 130, 72, 200), (5, 9, 1000, 264),
          (1, 300, 130, 515), (2, 257, 64, 129), (1, 513, 784, 256), (70, 3, 48, 40), (3, 128, 2048, 64), (1, 1000, 512, 1024), (2, 33, 1001, 72), (1, 31, 2056, 7),
          (2, 520, 128, 320), (9, 256, 384, 256), (1, 2, 8192, 16), (4, 24, 520, 1048)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_both_directions_match_the_formulas(shape, dtype):
    kinds = ["silu", "gelu", "relu", "sigmoid"]
    for k, (pad, drop) in enumerate(((0, True), (0, False), (8, True), (3, False), (1, True))):
        c = _case(*shape, dtype, pad, drop, seed=sum(shape) + k)
        _verify(c, kinds[(k + sum(shape)) % 4])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("kind", ["silu", "gelu", "relu", "sigmoid"])
def test_every_activation_through_every_size_class(kind, dtype):
    for m, rows, width, hidden in ((3, 7, 96, 80), (2, 100, 96, 72), (1, 400, 200, 264)):
        _verify(_case(m, rows, width, hidden, dtype, seed=rows), kind)


def test_the_written_out_gradients_are_those_of_autograd():
    """Pins the reference above (CPU, 64 bits) to automatic differentiation of the definition."""
    import torch
    torch.manual_seed(1)
    for kind, act in (("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu), ("relu", torch.relu), ("sigmoid", torch.sigmoid)):
        c = dict(x=torch.randn(2, 5, 7), weight=torch.randn(2, 6, 7), dh=torch.randn(2, 5, 3), scale=torch.rand(2, 5, 3).double())
        x, w = (c[k].double().requires_grad_() for k in ("x", "weight"))
        h = c["scale"] * act(x @ w[:, :3].transpose(1, 2)) * (x @ w[:, 3:].transpose(1, 2))
        dx, dw = torch.autograd.grad(h, (x, w), c["dh"].double())
        ref = formulas(c, kind)
        for name, value in (("h", h), ("dx", dx), ("dweight", dw)):
            assert torch.allclose(ref[name][0], value, rtol=1e-12, atol=1e-12), (kind, name)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["silu", "gelu", "sigmoid"])
@pytest.mark.parametrize("drop", [False, True])
def test_backward_agrees_with_differences_of_the_forward_pass(kind, drop):
    """Directional differences of the forward kernel in fp32.  Step 2^-6 along directions of size 1: the second-order term of a central
    difference is below 2e-3 of the gradient, the forward pass's rounding, 1e-6 of a loss of order 30 over a step of 3e-2, below
    2e-3: 1e-2 of the larger derivative covers both."""
    import torch
    import paper_1711_09846_b200 as pbt
    c = _case(2, 6, 40, 24, "float32", drop=drop, seed=5)
    dh = c["dh"] = c["dh"] * 10

    def loss(x, w):
        return (pbt.GatedUnit(w, kind).forward(x, dropout=c["dropout"]).double() * dh.double()).sum().item()
    g, _ = _run(c, kind)
    gen = torch.Generator(device="cuda").manual_seed(2)
    pairs = []
    for k, name in enumerate(("dx", "dweight")):
        v = torch.randn(g[name].shape, generator=gen, device="cuda")
        v /= v.norm()
        e = 2.0 ** -6
        up, down = ([c["x"] + s * e * v, c["weight"]] if k == 0 else [c["x"], c["weight"] + s * e * v] for s in (1, -1))
        pairs.append(((loss(*up) - loss(*down)) / (2 * e), (g[name].double() * v.double()).sum().item()))
    top = max(abs(b) for _, b in pairs)
    for diff, exact in pairs:
        assert abs(diff - exact) <= 1e-2 * top, pairs


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 3, 64, 40), (3, 70, 72, 33), (2, 300, 256, 128), (1, 40, 33, 24)], ids=str)
def test_a_pass_that_keeps_nothing_gives_the_same_bits(shape, dtype):
    import torch
    c = _case(*shape, dtype, seed=3)
    (a, _), (b, _) = _run(c, "silu"), _run(c, "silu", keep=False)
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [4, 100, 300])
def test_shared_weights_transposed_rows_and_any_alignment(rows, dtype):
    """One weight for all members; activations [rows, members, width] seen as [members, rows, width]; a shared x; bases off a vector's boundary."""
    import torch
    _verify(_case(3, rows, 72, 40, dtype, shared=True, seed=1), "silu")
    turn = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    c = _case(3, rows, 72, 40, dtype, seed=2)
    _verify({**c, "x": turn(c["x"]), "dh": turn(c["dh"])}, "silu")
    _verify({**c, "x": c["x"][:1].expand(3, -1, -1), "dh": c["dh"][:1].expand(3, -1, -1)}, "gelu")

    def moved(t, by):
        flat = torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")
        flat[by:by + t.numel()] = t.reshape(-1)
        return flat[by:by + t.numel()].view(t.shape)
    for by in (1, 4):
        for name in ("x", "weight", "dh"):
            _verify({**c, name: moved(c[name], by)}, "silu")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [6, 140, 300])
def test_a_diverged_row_or_member_stays_where_it_is(rows, dtype):
    import torch
    c = _case(3, rows, 72, 40, dtype, drop=False, seed=9)
    clean, _ = _run(c, "silu")
    dirty = {**c, "x": c["x"].clone(), "weight": c["weight"].clone(), "dh": c["dh"].clone()}
    dirty["x"][1, 2, 5] = float("nan")
    dirty["weight"][2] = float("nan")
    dirty["dh"][1, 4, 3] = float("inf")
    got, _ = _run(dirty, "silu")
    ok = torch.ones(3, rows, dtype=torch.bool)
    ok[2] = ok[1, 2] = False
    assert torch.equal(got["h"][ok], clean["h"][ok]) and torch.isnan(got["h"][~ok]).all()
    ok[1, 4] = False
    assert torch.equal(got["dx"][ok], clean["dx"][ok]) and torch.isnan(got["dx"][1, 2]).all() and torch.isnan(got["dx"][2]).all()
    assert not torch.isfinite(got["dx"][1, 4]).any()
    assert torch.equal(got["dweight"][0], clean["dweight"][0]) and not torch.isfinite(got["dweight"][1, 3]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [6, 140, 300])
def test_a_dropped_unit_is_zero_whatever_it_was(rows, dtype):
    import torch
    c = _case(2, rows, 72, 40, dtype, seed=4)
    off = c["scale"] == 0
    c["dh"][off] = float("nan")
    got = _verify({**c, "dh": torch.where(off, 0.0, c["dh"])}, "silu", _run(c, "silu")[0])
    c["weight"][:, 7] = float("nan")                    # one hidden unit of the gate
    got, _ = _run(c, "silu")
    assert (got["h"][:, :, 7][off[:, :, 7]] == 0).all() and torch.isnan(got["h"][:, :, 7][~off[:, :, 7]]).all()


@pytest.mark.gpu
def test_large_arguments_have_the_limits_of_the_activations():
    """g of 0, +-30, +-200 and +-1e30 (u = 1, dh = 1): act and act' of the definition, no NaN from an overflowing exponential."""
    import torch
    import paper_1711_09846_b200 as pbt
    values = torch.tensor([0.0, 30, -30, 200, -200, 1e30, -1e30], device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        for rows in (7, 77, 301):
            x = torch.zeros(1, rows, 2, device="cuda", dtype=dtype)
            x[0, :, 0], x[0, :, 1] = values.repeat(rows // 7 + 1)[:rows].to(dtype), 1
            w = torch.tensor([[[1.0, 0.0], [0.0, 1.0]]], device="cuda", dtype=dtype)
            for kind in ("silu", "gelu", "relu", "sigmoid"):
                h, kept = pbt.GatedUnit(w, kind).forward(x, keep=True)
                dx, _ = pbt.GatedUnit(w, kind).backward(torch.ones_like(h), x, kept)
                act, slope = _act(kind, x[0, :, 0].double())
                if kind == "gelu":
                    slope = torch.where(x[0, :, 0].abs() > 100, (x[0, :, 0] > 0).double(), slope)     # (inf * 0 in the formula)
                for got, want in ((h[0, :, 0], act), (dx[0, :, 0], slope), (dx[0, :, 1], act)):
                    assert ((got.double() - want).abs() <= (2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -18) * want.abs() + 1e-8).all(), kind


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_operands_beyond_32_bit_offsets(dtype):
    """x and dx of more than 2^31 elements (the last rows are looked at), and a weight like that."""
    import torch
    import paper_1711_09846_b200 as pbt
    dt = getattr(torch, dtype)

    def normal(*shape, scale=1.0):
        return torch.empty(shape, device="cuda", dtype=dt).normal_(0.0, scale)
    x, w = normal(5, 220_000, 2048), normal(5, 32, 2048, scale=2048 ** -0.5)
    dh = normal(5, 220_000, 16, scale=0.1)
    layer = pbt.GatedUnit(w)
    h, kept = layer.forward(x, keep=True)
    dx, _ = layer.backward(dh, x, kept)
    last = dict(x=x[4:, -3:], weight=w[4:], dh=dh[4:, -3:], scale=None, dropout=None)
    want = formulas(last, "silu")
    for got, name in ((h, "h"), (dx, "dx")):
        value, tol = want[name]
        assert ((got[4:, -3:].double() - value).abs() <= tol + (2.0 ** -8 if dt == torch.bfloat16 else 0) * (value.abs() + tol)).all(), name
    layer.check()
    del x, dx, h, kept, dh
    x, w = normal(70, 3, 4096), normal(70, 8200, 4096, scale=4096 ** -0.5)
    h = pbt.GatedUnit(w).forward(x)
    value, tol = formulas(dict(x=x[69:], weight=w[69:], dh=normal(1, 3, 4100), scale=None, dropout=None), "silu")["h"]
    assert ((h[69:].double() - value).abs() <= tol + (2.0 ** -8 if dt == torch.bfloat16 else 0) * (value.abs() + tol)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_streams_graphs_and_threads(dtype):
    import threading
    import torch
    import paper_1711_09846_b200 as pbt
    cases = [_case(2, rows, 72, 40, dtype, seed=rows) for rows in (5, 90, 300)]
    layer = pbt.GatedUnit(cases[0]["weight"])
    cases = [{**c, "weight": cases[0]["weight"]} for c in cases]
    want = [_run(c, "silu", layer=layer)[0] for c in cases]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [_run(c, "silu", layer=layer, stream=side)[0] for c in cases]
    side.synchronize()
    step = cases[1]["dropout"].step
    graphs = []
    for c in cases:                                    # two graphs of one layer share nothing that a replay writes
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, _run(c, "silu", layer=layer)[0]))
    results = [None] * 6

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                results[k] = _run(cases[k % 3], "silu", layer=layer)[0]
            torch.cuda.current_stream().synchronize()
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(k,)) for k in range(6)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for g, _ in graphs * 2:
        g.replay()
    torch.cuda.synchronize()
    for k, c in enumerate(cases):
        for other in (got[k], graphs[k][1], results[k], results[k + 3]):
            for name in want[k]:
                assert torch.equal(want[k][name], other[name]), name
    step += 1                                          # a replay draws anew for the steps that it finds
    graphs[1][0].replay()
    fresh, _ = _run(cases[1], "silu", layer=layer)
    torch.cuda.synchronize()
    assert torch.equal(graphs[1][1]["h"], fresh["h"]) and not torch.equal(fresh["h"], want[1]["h"])
    layer.check()


@pytest.mark.gpu
def test_the_units_dropout_is_the_operators():
    """The hidden units that a gated unit drops are those that dropout_forward drops for the same rule."""
    import torch
    import paper_1711_09846_b200 as pbt
    for rows in (3, 100, 400):
        c = _case(2, rows, 64, 200, "bfloat16", seed=rows)
        h = pbt.GatedUnit(c["weight"], "sigmoid").forward(torch.ones_like(c["x"]), dropout=c["dropout"])
        assert torch.equal(h == 0, pbt.dropout_forward(torch.ones_like(h), c["dropout"]) == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 3, 64, 40), (2, 70, 72, 33), (2, 300, 264, 136), (1, 129, 33, 24)], ids=str)
def test_nothing_is_written_beside_the_results(shape, dtype):
    """The C calls on results that lie between guarded bytes, with a workspace of exactly the size that is asked for."""
    import torch
    import paper_1711_09846_b200 as pbt
    m, rows, width, hidden = shape
    c = _case(*shape, dtype, seed=6)
    want, layer = _run(c, "silu")
    lib, size = pbt.load_library(), c["x"].element_size()
    guard = 4096

    def between(n):
        t = torch.full((n + 2 * guard,), 0x5A, dtype=torch.uint8, device="cuda")
        return t, t[guard:guard + n]
    sizes = dict(h=m * rows * hidden * size, kept=m * rows * 2 * ((hidden + 7) // 8 * 8) * 4, dx=m * rows * width * size, dweight=m * 2 * hidden * width * size)
    places = {k: between(n) for k, n in sizes.items()}
    d = layer._call(layer._describe(c["x"], c["dh"]), c["x"], c["dropout"])
    d.dh = c["dh"].data_ptr()
    for k, (_, t) in places.items():
        setattr(d, k, t.data_ptr())
    n = C.c_size_t(0)
    s = torch.cuda.current_stream().cuda_stream
    for backward, call in ((0, lib.pbt_gated_forward), (1, lib.pbt_gated_backward)):
        assert lib.pbt_gated_query_workspace(C.byref(d), backward, C.byref(n)) == 0
        whole, ws = between(n.value)
        places[f"workspace {backward}"] = (whole, ws)
        assert call(C.byref(d), ws.data_ptr(), n.value, s) == 0
        if n.value:
            assert call(C.byref(d), ws.data_ptr(), n.value - 1, s) == 3 and call(C.byref(d), ws.data_ptr() + 16, n.value, s) == 3
            assert call(C.byref(d), None, n.value, s) == 3
    torch.cuda.synchronize()
    for k, (whole, t) in places.items():
        assert (whole[:guard] == 0x5A).all() and (whole[-guard:] == 0x5A).all(), k
    for k in want:
        assert torch.equal(places[k][1].view(want[k].dtype).view(want[k].shape), want[k]), k


def test_the_c_calls_refuse_what_they_cannot_do():
    import paper_1711_09846_b200 as pbt
    from paper_1711_09846_b200.binding import PbtDropRule, PbtGatedDesc
    lib, n = pbt.load_library(), C.c_size_t(0)

    def desc(**kw):
        d = PbtGatedDesc()
        d.members, d.rows, d.width, d.hidden, d.dtype = 1, 4, 8, 8, 1
        for name in ("x", "weight", "h", "kept", "dh", "dx", "dweight", "status_device"):
            setattr(d, name, 4096)
        d.x_row = d.weight_row = d.dh_row = 8
        for k, v in kw.items():
            setattr(d, k, v)
        return d
    assert lib.pbt_gated_query_workspace(None, 0, C.byref(n)) == 1 and lib.pbt_gated_query_workspace(C.byref(desc()), 0, None) == 1
    assert lib.pbt_gated_forward(None, None, 0, None) == 1 and lib.pbt_gated_backward(None, None, 0, None) == 1
    rule = PbtDropRule()
    rule.rate_all = 2.0
    common = [(1, dict(members=0)), (1, dict(rows=-1)), (1, dict(width=0)), (1, dict(hidden=0)), (2, dict(members=65536)), (2, dict(rows=1 << 22)),
              (2, dict(width=1 << 22)), (2, dict(hidden=1 << 21)), (2, dict(members=65535, rows=1 << 20, hidden=1 << 20, width=1 << 20, x_row=1 << 20, weight_row=1 << 20)),
              (2, dict(dtype=2)), (2, dict(activation=4)), (2, dict(activation=-1)), (1, dict(weight=None)), (1, dict(weight_row=7)), (1, dict(weight_member=-8)),
              (1, dict(x=None)), (1, dict(x_row=7)), (1, dict(x_member=-1)), (1, dict(status_device=None)), (1, dict(drop=C.addressof(rule))), (1, dict(kept=4100)), (2, dict(rows=1 << 21, members=1 << 10, width=33, x_row=33, weight_row=40)),
              (2, dict(rows=40, hidden=1 << 20, members=1 << 10, width=65, x_row=72, weight_row=65, x_member=72, weight_member=1))]
    for code, kw in common:
        for backward in (0, 1):
            assert lib.pbt_gated_query_workspace(C.byref(desc(**kw)), backward, C.byref(n)) == code, kw
        assert lib.pbt_gated_forward(C.byref(desc(**kw)), 4096, 1 << 60, None) == code and lib.pbt_gated_backward(C.byref(desc(**kw)), 4096, 1 << 60, None) == code
        assert lib.pbt_last_error(None)
    assert lib.pbt_gated_forward(C.byref(desc(h=None)), 4096, 1 << 60, None) == 1
    for kw in (dict(dh=None), dict(dx=None), dict(dweight=None), dict(dh_row=7), dict(dh_member=-1)):
        assert lib.pbt_gated_backward(C.byref(desc(**kw)), 4096, 1 << 60, None) == 1, kw
    assert lib.pbt_gated_forward(C.byref(desc(rows=0, x=None, h=None)), None, 0, None) == 0         # nothing to do
    for kw in (dict(x=4098), dict(weight_row=9)):       # these need one
        assert lib.pbt_gated_query_workspace(C.byref(desc(**kw)), 0, C.byref(n)) == 0 and n.value > 0
        assert lib.pbt_gated_forward(C.byref(desc(**kw)), None, 1 << 20, None) == 3 and lib.pbt_gated_backward(C.byref(desc(**kw)), None, 1 << 20, None) == 3
    for dtype in (0, 1):
        assert lib.pbt_gated_query_workspace(C.byref(desc(dtype=dtype)), 0, C.byref(n)) == 0 and n.value == 0
    assert lib.pbt_gated_query_workspace(C.byref(desc(x_row=9, dtype=0)), 0, C.byref(n)) == 0 and n.value == 0


@pytest.mark.gpu
def test_refusals_and_empty_batches():
    import torch
    import paper_1711_09846_b200 as pbt
    w = torch.randn(2, 16, 24, device="cuda")
    layer = pbt.GatedUnit(w)
    x, dh = torch.randn(2, 3, 24, device="cuda"), torch.randn(2, 3, 8, device="cuda")
    h, kept = layer.forward(x, keep=True)
    for bad in (w.cpu(), w[0], w.double(), w[:, :15], w[:, :0], w.transpose(1, 2)):
        with pytest.raises(ValueError):
            pbt.GatedUnit(bad)
    with pytest.raises(ValueError):
        pbt.GatedUnit(w, "tanh")
    for bad in (x.cpu(), x[0], x.bfloat16(), x[:1], x[:, :, :23], x.transpose(0, 1).transpose(1, 2)):
        with pytest.raises(ValueError):
            layer.forward(bad)
    for bad in (dh.cpu(), dh.bfloat16(), dh[:, :2], dh[..., :7], dh.transpose(1, 2)):
        with pytest.raises(ValueError):
            layer.backward(bad, x, kept)
    for bad in (kept[:, :2], kept.bfloat16(), kept.transpose(1, 2), kept.cpu()):
        with pytest.raises(ValueError):
            layer.backward(dh, x, bad)
    with pytest.raises(ValueError):
        layer.forward(x, dropout=pbt.Dropout(torch.ones(3, device="cuda"), 1, 2))
    with pytest.raises(pbt.PbtError):
        layer.forward(x, dropout=pbt.Dropout(0.5, 1, 2, first_member=0x7FFFFFFF))
    with pytest.raises(pbt.PbtError):
        layer.forward(x[:, :1].expand(2, 3, 24))       # rows that lie on one another
    many = torch.empty(2, 1, 24, device="cuda").expand(2, 2 ** 32 + 3, 24)
    with pytest.raises(ValueError):
        layer.forward(many)
    h0, k0 = layer.forward(x[:, :0], keep=True)
    dx, dw = layer.backward(dh[:, :0], x[:, :0], k0)
    assert h0.shape == (2, 0, 8) and dx.shape == (2, 0, 24) and (dw == 0).all()
