"""Block norms (block_norm_forward / block_norm_backward) against the formulas in 64 bits, differentiated by autograd.

Tolerances.  eps = 2^-24.  A result is a product of at most a dozen fp32 factors, among them a reciprocal root (2 ulp), a
sigmoid (its exponential's relative error is about (|z| + 2) 2^-22: |z| < 6 in these inputs, 32 eps) and a mean of n <=
8192 terms added by threads (at most 64 each) and a tree (10 levels): below 128 eps of the sum of the terms' magnitudes;
96 + 128 eps of max(|value|, rms of its row) covers them: 1.4e-5.  A bf16 result adds its rounding, 2^-8 of the value.
A column sum of R rows adds (R + 16) eps of the sum of its terms' magnitudes, which the reference returns."""
import ctypes as C

import pytest

EPS32 = 2.0 ** -24
VALUE = 224 * EPS32


def _inputs(m, rows, width, dtype, gate, seed, pad=0, block=True, nxt=True):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = getattr(torch, dtype)

    def act(scale=1.0):
        t = torch.randn(m, rows + (1 if pad else 0), width + pad, generator=gen).mul_(scale).to(dt).cuda()
        return t[:, :rows, :width]            # strides of their own when padded

    d = dict(x=act(), block=act(0.7) if block else None, gate=None, post_weight=None, scale=None, next_weight=None)
    if block:
        d["post_weight"] = (torch.rand(m, width, generator=gen) + 0.5).cuda()
        d["scale"] = (torch.rand(m, generator=gen) - 0.3).cuda()
        if gate == "full":
            d["gate"] = act(1.2)
        elif gate == "vector":
            d["gate"] = torch.randn(m, width, generator=gen).to(dt).cuda()
    if nxt:
        d["next_weight"] = (torch.rand(m, width, generator=gen) + 0.5).cuda()
    return d, act(0.1), act(0.1)


def _formula(d, eps):
    """(y, u) in 64 bits, differentiable."""
    import torch
    y = d["x"]
    if d["block"] is not None:
        v = d["block"] / torch.sqrt(d["block"].square().mean(-1, keepdim=True) + eps)
        n = v * d["post_weight"][:, None]
        if d["gate"] is not None:
            g = torch.sigmoid(d["gate"])
            n = n * (g if g.dim() == 3 else g[:, None])
        y = y + n * (1.0 if d["scale"] is None else d["scale"].view(-1, 1, 1))
    u = None
    if d["next_weight"] is not None:
        u = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * d["next_weight"][:, None]
    return y, u


def _double(d):
    return {k: None if v is None else v.detach().cpu().double() for k, v in d.items()}


def _close(got, want, extra=0.0):
    """|got - want| <= VALUE max(|want|, rms of the row) + bf16 rounding + extra."""
    import torch
    if want.numel() == 0:
        assert got.shape == want.shape
        return
    g = got.detach().cpu().double()
    rms = want.square().mean(-1, keepdim=True).sqrt()
    tol = VALUE * torch.maximum(want.abs(), rms) + extra
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs() + 1e-38
    bad = ~((g - want).abs() <= tol)
    assert not bad.any(), ((g - want).abs() / tol).max()


SHAPES = [(1, 1, 1), (1, 1, 8), (2, 3, 7), (1, 5, 64), (3, 17, 100), (2, 33, 256), (1, 4, 1001), (5, 9, 1000), (2, 40, 2048),
          (1, 3, 2056), (2, 2, 4096), (1, 3, 4100), (1, 2, 8192), (1, 2, 8191), (70, 3, 48), (1, 600, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gate", ["none", "vector", "full"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_backward_match_the_formulas(shape, gate, dtype):
    import torch
    import paper_1711_09846_b200 as pbt
    m, rows, width = shape
    eps = 1e-5
    for pad, block, nxt in ((0, True, True), (8, True, True), (3, True, True), (0, True, False), (0, False, True)):
        if not block and gate != "none":
            continue
        d, dy, du = _inputs(m, rows, width, dtype, gate, seed=sum(shape) + pad, pad=pad, block=block, nxt=nxt)
        kw = {k: d[k] for k in ("post_weight", "gate", "scale", "next_weight")}
        out = pbt.block_norm_forward(d["x"], d["block"], eps=eps, keep=True, **kw)
        want_y, want_u = _formula(_double(d), eps)
        if block:
            _close(out.y, want_y)
            r = (_double(d)["block"].square().mean(-1) + eps).rsqrt()
            assert torch.allclose(out.rstd_block.cpu().double(), r, rtol=VALUE)
        else:
            assert out.y is d["x"]
        plain = pbt.block_norm_forward(d["x"], d["block"], eps=eps, **kw)
        assert torch.equal(plain.y, out.y) and (plain.u is None or torch.equal(plain.u, out.u)) and plain.rstd_block is plain.rstd_next is None
        if nxt:
            _close(out.u, want_u)
            r = (want_y.square().mean(-1) + eps).rsqrt()
            assert torch.allclose(out.rstd_next.cpu().double(), r, rtol=VALUE)
        # the backward pass is a function of the stored y: the reference takes the same values for y and the roots
        grads = pbt.block_norm_backward(dy, du if nxt else None, out.y, d["block"], rstd_block=out.rstd_block,
                                        rstd_next=out.rstd_next, **kw)
        ref, mags = _reference_backward(d, dy, du if nxt else None, out)
        bf = (rows + 16) * EPS32
        _close(grads.dx, ref["dx"])
        if block:
            _close(grads.dblock, ref["dblock"])
            _close(grads.dpost_weight, ref["dpost"], bf * mags["dpost"])
            assert abs(grads.dscale.cpu().double() - ref["dscale"]).le((VALUE + (rows * 4 + 64) * EPS32) * mags["dscale"] + 1e-30).all()
            if gate == "full":
                _close(grads.dgate, ref["dgate"])
            elif gate == "vector":
                _close(grads.dgate, ref["dgate"], bf * mags["dgate"])
            else:
                assert grads.dgate is None
        else:
            assert grads.dblock is None and grads.dpost_weight is None and grads.dscale is None
        if nxt:
            _close(grads.dnext_weight, ref["dnext"], bf * mags["dnext"])
        else:
            assert grads.dnext_weight is None


def _reference_backward(d, dy, du, out):
    """The gradients written out in 64 bits from the stored y and reciprocal roots, and the sums of magnitudes."""
    import torch
    f = _double(d)
    dy, y = dy.cpu().double(), out.y.cpu().double()
    ref, mags = {}, {}
    dx = dy
    if du is not None:
        du = du.cpu().double()
        r = out.rstd_next.cpu().double()[..., None]
        yh, dh = y * r, du * f["next_weight"][:, None]
        dx = dy + r * (dh - yh * (dh * yh).mean(-1, keepdim=True))
        ref["dnext"], mags["dnext"] = (du * yh).sum(1), (du * yh).abs().sum(1)
    ref["dx"] = dx
    if f["block"] is not None:
        r = out.rstd_block.cpu().double()[..., None]
        v, w, c = f["block"] * r, f["post_weight"][:, None], f["scale"].view(-1, 1, 1)
        g = torch.ones_like(v)
        if f["gate"] is not None:
            g = torch.sigmoid(f["gate"])
            g = g if g.dim() == 3 else g[:, None].expand_as(v)
        dn = c * g * dx
        ref["dblock"] = r * (dn * w - v * (dn * w * v).mean(-1, keepdim=True))
        ref["dpost"], mags["dpost"] = (dn * v).sum(1), (dn * v).abs().sum(1)
        o = dx * v * w * g
        ref["dscale"], mags["dscale"] = o.sum((1, 2)), o.abs().sum((1, 2))
        dz = c * o * (1 - g)
        ref["dgate"] = dz if f["gate"] is None or f["gate"].dim() == 3 else dz.sum(1)
        mags["dgate"] = dz.abs().sum(1)
    return ref, mags


@pytest.mark.parametrize("gate", ["none", "vector", "full"])
def test_the_written_out_gradients_are_those_of_autograd(gate):
    """Pins the reference above (CPU, 64 bits) to automatic differentiation of the formula."""
    import torch
    torch.manual_seed(1)
    m, rows, width, eps = 2, 5, 12, 1e-5
    d = dict(x=torch.randn(m, rows, width), block=torch.randn(m, rows, width), post_weight=torch.rand(m, width) + 0.5,
             scale=torch.rand(m), next_weight=torch.rand(m, width) + 0.5,
             gate=None if gate == "none" else torch.randn(*((m, rows, width) if gate == "full" else (m, width))))
    f = {k: None if v is None else v.double().requires_grad_() for k, v in d.items()}
    y, u = _formula(f, eps)
    dy, du = torch.randn(m, rows, width).double(), torch.randn(m, rows, width).double()
    ((y * dy).sum() + (u * du).sum()).backward()

    class Out:
        pass
    Out.y = y.detach()
    Out.rstd_block = (f["block"].detach().square().mean(-1) + eps).rsqrt()
    Out.rstd_next = (y.detach().square().mean(-1) + eps).rsqrt()
    ref, _ = _reference_backward(d, dy, du, Out)
    for name, key in (("dx", "x"), ("dblock", "block"), ("dpost", "post_weight"), ("dnext", "next_weight"), ("dscale", "scale"),
                      ("dgate", "gate")):
        if f[key] is not None:
            assert torch.allclose(ref[name], f[key].grad, rtol=1e-6, atol=1e-6), name


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["none", "vector", "full"])
def test_backward_agrees_with_differences_of_the_forward_pass(gate):
    """Directional differences of the forward kernel in fp32.  Step 2^-6 along directions of size 1: the second-order term
    of a central difference is below 2e-3 of the gradient, the forward pass's rounding, 1e-6 of a loss of order 30 over a
    step of 3e-2, below 2e-3: 1e-2 of the largest derivative in the set covers both."""
    import torch
    import paper_1711_09846_b200 as pbt
    d, dy, du = _inputs(2, 6, 40, "float32", gate, seed=5)
    dy, du = dy * 10, du * 10
    names = [k for k in ("x", "block", "post_weight", "gate", "scale", "next_weight") if d[k] is not None]

    def run(e):
        kw = {k: e[k] for k in ("post_weight", "gate", "scale", "next_weight")}
        return pbt.block_norm_forward(e["x"], e["block"], keep=True, **kw), kw

    def loss(e):
        out, _ = run(e)
        return ((out.y.double() * dy.double()).sum() + (out.u.double() * du.double()).sum()).item()

    out, kw = run(d)
    g = pbt.block_norm_backward(dy, du, out.y, d["block"], rstd_block=out.rstd_block, rstd_next=out.rstd_next, **kw)
    grads = dict(x=g.dx, block=g.dblock, post_weight=g.dpost_weight, gate=g.dgate, scale=g.dscale, next_weight=g.dnext_weight)
    gen = torch.Generator(device="cuda").manual_seed(2)
    pairs = []
    for k in names:
        v = torch.randn(d[k].shape, generator=gen, device="cuda")
        v /= v.norm()
        h = 2.0 ** -6
        diff = (loss({**d, k: d[k] + h * v}) - loss({**d, k: d[k] - h * v})) / (2 * h)
        pairs.append((k, diff, (grads[k].double() * v.double()).sum().item()))
    scale = max(abs(b) for _, _, b in pairs)
    for k, diff, exact in pairs:
        assert abs(diff - exact) <= 1e-2 * scale, pairs


@pytest.mark.gpu
def test_a_diverged_row_stays_in_its_row_and_member():
    import torch
    import paper_1711_09846_b200 as pbt
    d, dy, du = _inputs(3, 8, 72, "bfloat16", "full", seed=9)
    kw = {k: d[k] for k in ("post_weight", "gate", "scale", "next_weight")}
    clean = pbt.block_norm_forward(d["x"], d["block"], **kw)
    dirty = {k: v.clone() for k, v in d.items()}
    dirty["block"][1, 2, 5] = float("nan")
    dirty["x"][1, 4, 0] = float("inf")
    dirty["gate"][0, 3, :] = float("-inf")          # a closed gate: y is x there, exactly
    kd = {k: dirty[k] for k in kw}
    out = pbt.block_norm_forward(dirty["x"], dirty["block"], keep=True, **kd)
    assert torch.equal(out.y[0, 3], d["x"][0, 3])
    ok = torch.ones(3, 8, dtype=torch.bool)
    ok[1, 2] = ok[1, 4] = ok[0, 3] = False
    assert torch.equal(out.y[ok], clean.y[ok]) and torch.equal(out.u[ok], clean.u[ok])
    assert torch.isnan(out.y[1, 2]).all()
    g = pbt.block_norm_backward(dy, du, out.y, dirty["block"], rstd_block=out.rstd_block, rstd_next=out.rstd_next, **kd)
    assert torch.isnan(g.dx[1, 2]).all() and torch.isfinite(g.dx[ok]).all()
    assert torch.isfinite(g.dpost_weight[[0, 2]]).all() and torch.isfinite(g.dscale[[0, 2]]).all()
    assert (g.dgate[0, 3] == 0).all()


@pytest.mark.gpu
def test_zero_rows_and_rows_of_zeros():
    import torch
    import paper_1711_09846_b200 as pbt
    d, dy, du = _inputs(2, 0, 64, "float32", "vector", seed=1)
    kw = {k: d[k] for k in ("post_weight", "gate", "scale", "next_weight")}
    out = pbt.block_norm_forward(d["x"], d["block"], keep=True, **kw)
    assert out.y.shape == (2, 0, 64) and out.u.shape == (2, 0, 64)
    g = pbt.block_norm_backward(dy, du, out.y, d["block"], rstd_block=out.rstd_block, rstd_next=out.rstd_next, **kw)
    for t in (g.dgate, g.dpost_weight, g.dnext_weight, g.dscale):
        assert (t == 0).all()
    z = torch.zeros(1, 2, 64, device="cuda")
    w = torch.ones(1, 64, device="cuda")
    out = pbt.block_norm_forward(z, z, post_weight=w, next_weight=w, keep=True)
    assert (out.y == 0).all() and (out.u == 0).all() and torch.allclose(out.rstd_next, torch.full((1, 2), 1e3, device="cuda"))


@pytest.mark.gpu
def test_another_stream_gives_the_same_bits():
    import torch
    import paper_1711_09846_b200 as pbt
    d, dy, du = _inputs(3, 50, 512, "bfloat16", "full", seed=4)
    kw = {k: d[k] for k in ("post_weight", "gate", "scale", "next_weight")}
    out = pbt.block_norm_forward(d["x"], d["block"], keep=True, **kw)
    g = pbt.block_norm_backward(dy, du, out.y, d["block"], rstd_block=out.rstd_block, rstd_next=out.rstd_next, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out2 = pbt.block_norm_forward(d["x"], d["block"], stream=side, keep=True, **kw)
    g2 = pbt.block_norm_backward(dy, du, out2.y, d["block"], rstd_block=out2.rstd_block, rstd_next=out2.rstd_next, stream=side, **kw)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((*out, *g), (*out2, *g2)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_norm_refusals():
    import torch
    import paper_1711_09846_b200 as pbt
    x, w, c = torch.zeros(2, 3, 16, device="cuda"), torch.ones(2, 16, device="cuda"), torch.ones(2, device="cuda")
    bad = [dict(), dict(block=x), dict(block=x, post_weight=w.half()), dict(block=x[:, :2], post_weight=w),
           dict(block=x.bfloat16(), post_weight=w), dict(block=x, post_weight=w[:1]), dict(gate=x, next_weight=w),
           dict(block=x, post_weight=w, gate=w.bfloat16()), dict(block=x, post_weight=w, scale=torch.ones(3, device="cuda")),
           dict(next_weight=w.t().contiguous().t()), dict(next_weight=w.cpu())]
    for kw in bad:
        kw = dict(kw)
        with pytest.raises(ValueError):
            pbt.block_norm_forward(x, kw.pop("block", None), **kw)
    for y in (x[0], x.half(), x.cpu(), torch.zeros(2, 3, 32, device="cuda")[..., ::2]):
        with pytest.raises(ValueError):
            pbt.block_norm_forward(y, next_weight=w)
    with pytest.raises(pbt.PbtError):
        pbt.block_norm_forward(torch.zeros(1, 1, 8200, device="cuda"), next_weight=torch.ones(1, 8200, device="cuda"))
    with pytest.raises(pbt.PbtError):
        pbt.block_norm_forward(x, next_weight=w, eps=-1.0)
    with pytest.raises(ValueError):
        pbt.block_norm_backward(x, None, x)
    with pytest.raises(ValueError):
        pbt.block_norm_backward(x, x, x, next_weight=w)


def test_norm_arguments_are_checked_before_the_device_is_touched():
    import paper_1711_09846_b200 as pbt
    from paper_1711_09846_b200.binding import PbtBlockNormDesc
    lib = pbt.load_library()
    n = C.c_size_t(0)

    def desc(**kw):
        d = PbtBlockNormDesc()
        d.members, d.rows, d.width, d.eps = 2, 3, 16, 1e-6
        d.x, d.u, d.next_weight = 4096, 8192, 16384
        for k, v in kw.items():
            setattr(d, k, v)
        return d
    for kw, code in ((dict(members=0), 1), (dict(rows=-1), 1), (dict(width=0), 1), (dict(dtype=5), 2), (dict(width=9000), 2),
                     (dict(x=None), 1), (dict(u=None), 1), (dict(next_weight=None), 1), (dict(gate=64), 1), (dict(block=64), 1),
                     (dict(eps=float("nan")), 1)):
        assert lib.pbt_block_norm_forward(C.byref(desc(**kw)), None) == code, kw
        assert lib.pbt_last_error(None)
    assert lib.pbt_block_norm_forward(None, None) == 1
    assert lib.pbt_block_norm_query_workspace(C.byref(desc(du=64)), C.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    ok = dict(du=64, dnext_weight=64, dx=64, rstd_next=64)
    assert lib.pbt_block_norm_backward(C.byref(desc(**ok)), None, 0, None) == 3
    for kw in (dict(du=None), dict(dnext_weight=None), dict(dx=None), dict(rstd_next=None)):
        assert lib.pbt_block_norm_backward(C.byref(desc(**{**ok, **kw})), None, 0, None) == 1, kw


# Even widths whose rows are no multiples of 16 bytes, around the limits of the widths that a warp, a block and a thread take.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gate", ["none", "vector", "full"])
@pytest.mark.parametrize("shape", [(2, 5, 30), (2, 5, 34), (3, 40, 66), (2, 7, 514), (4, 50, 1002), (2, 30, 2050), (1, 9, 4098), (1, 3, 8190)], ids=str)
def test_rows_of_even_width_match_the_formulas(shape, gate, dtype):
    test_forward_and_backward_match_the_formulas(shape, gate, dtype)


# The gradient of gates that are nearly open or nearly closed, element by element.  Without a next norm dx is dy, so dz = c dy v w g (1 - g)
# is a product of seven factors: 16 eps, and twice the sigmoid's (|z| + 3) 2^-22, relative to the element itself (which is no
# difference of larger numbers); bf16 adds its rounding, a gate vector the sum over its rows.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gate", ["vector", "full"])
@pytest.mark.parametrize("shape", [(2, 3, 7), (2, 3, 8), (1, 4, 64), (2, 3, 34), (1, 2, 33), (1, 3, 2048), (1, 2, 4104), (1, 2, 4099)], ids=str)
def test_the_gradient_of_a_saturated_gate_is_exact_to_rounding(shape, gate, dtype):
    import torch
    import paper_1711_09846_b200 as pbt
    m, rows, width = shape
    d, dy, _ = _inputs(m, rows, width, dtype, gate, seed=sum(shape), nxt=False)
    at = torch.tensor([8.0, -8.0, 12.0, -12.0, 16.0, -16.0, 20.0, -20.0, 60.0, -60.0, 0.0], device="cuda")
    d["gate"].copy_(at[torch.arange(d["gate"].numel(), device="cuda").view(d["gate"].shape) % 11])
    kw = {k: d[k] for k in ("post_weight", "gate", "scale")}
    out = pbt.block_norm_forward(d["x"], d["block"], keep=True, **kw)
    got = pbt.block_norm_backward(dy, None, out.y, d["block"], rstd_block=out.rstd_block, **kw).dgate.cpu().double()
    f = _double(d)
    z = f["gate"] if gate == "full" else f["gate"][:, None]
    dz = f["scale"].view(-1, 1, 1) * dy.cpu().double() * f["block"] * out.rstd_block.cpu().double()[..., None] * f["post_weight"][:, None] \
        * torch.sigmoid(z) * torch.sigmoid(-z)
    tol = (16 * EPS32 + 2 * (z.abs() + 3) * 2.0 ** -22) * dz.abs()
    if gate == "vector":
        dz, tol = dz.sum(1), (tol + (rows + 16) * EPS32 * dz.abs()).sum(1)
    if dtype == "bfloat16":
        tol = tol + 2.0 ** -8 * dz.abs()
    assert ((got - dz).abs() <= tol + 1e-37).all(), ((got - dz).abs() / (tol + 1e-37)).max()
