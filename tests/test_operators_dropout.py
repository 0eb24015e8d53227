"""Dropout (dropout_forward / dropout_backward) against the definition, with masks from the oracle's generator.

Tolerances.  eps = 2^-24.  A kept element is x times a scale, which is one division's rounding away from its definition, and the
product's: 2 eps of it; the residual's addition rounds once more, eps of the result.  A bf16 result adds its rounding, 2^-8 of the value.
Which elements are dropped has no tolerance."""
import ctypes as C

import numpy as np
import pytest

from oracle.philox import philox4x32_10, philox4x32_10_np

EPS32 = 2.0 ** -24
SEED = 0xDEADBEEF12345678


def scales(members, rows, width, rate, seed, step, site=0, first_member=0):
    """What every element is multiplied by, float64 [members, rows, width], from the definition; rate and step: a value for every member."""
    groups = (width + 7) // 8
    block = np.arange(rows * groups, dtype=np.uint64)
    out = np.zeros((members, rows, width))
    for m in range(members):
        words = philox4x32_10_np(np.uint64(first_member + m), np.uint64(int(step[m]) & 0xFFFFFFFF), np.uint64(5 + site), block, seed)
        bits = np.stack([w >> s & np.uint32(0xFFFF) for w in words for s in (np.uint32(0), np.uint32(16))], -1)
        r = np.float32(rate[m])
        t = 0 if np.isnan(r) else int(np.rint(min(max(float(r), 0.0), 1.0) * 65536))
        kept = bits.reshape(rows, groups * 8)[:, :width] >= t
        out[m] = np.where(kept, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)
    return out


def _case(m, rows, width, dtype, pad=0, residual=True, seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = getattr(torch, dtype)

    def act():
        t = torch.randn(m, rows + (1 if pad else 0), width + pad, generator=gen)
        return torch.where(t == 0, 1.0, t).to(dt).cuda()[:, :rows, :width]
    rate = torch.rand(m, generator=gen).cuda()
    step = torch.randint(0, 1 << 40, (m,), generator=gen).cuda()       # (the lower 32 bits count)
    return act(), act() if residual else None, rate, step


def _verify(got, x, residual, scale):
    import torch
    f = torch.from_numpy(scale)
    x, y = x.cpu().double(), got.cpu().double()
    part = torch.where(f == 0, 0.0, x * f)
    want = part if residual is None else part + residual.cpu().double()
    tol = 2 * EPS32 * part.abs() + EPS32 * want.abs() + 1e-40
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs()
    assert got.is_contiguous() and got.shape == x.shape
    assert ((y - want).abs() <= tol).all()
    if residual is None:
        assert torch.equal(y == 0, f == 0)
    else:                                              # what is dropped leaves the residual as it is
        assert torch.equal(y[f == 0], residual.cpu().double()[f == 0])


def test_the_oracle_of_the_masks_is_the_generator():
    """One element by hand: member 7 of the population, step 3, site 2, row 4 and column 13 of 21."""
    words = philox4x32_10((7, 3, 7, 4 * 3 + 1), (SEED & 0xFFFFFFFF, SEED >> 32))
    bits = words[2] >> 16                              # column 13 is the sixth of its group: the upper half of word 2
    s = [scales(2, 5, 21, [0.0, t / 65536], SEED, [9, 3], site=2, first_member=6)[1, 4, 13] for t in (bits, bits + 1)]
    assert s == [65536 / (65536 - bits), 0.0]


# (the last ones: vectors that reach over rows and members, in small calls and in those that fill the GPU)
SHAPES = [(1, 1, 1), (1, 1, 8), (2, 3, 7), (1, 5, 64), (3, 17, 100), (2, 33, 256), (1, 4, 1001), (5, 9, 1000), (2, 40, 2048), (1, 3, 2052),
          (1, 2, 8191), (70, 3, 48), (1, 6000, 24), (300, 1, 9), (400, 1, 13), (7, 1, 8), (9, 3, 11),
          (600, 9, 1003), (5000, 1, 1001), (2, 20000, 139)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_both_directions_match_the_definition(shape, dtype):
    import paper_1711_09846_b200 as pbt
    for pad, residual in ((0, True), (0, False), (8, True), (3, True), (3, False), (4, True), (1, False)):
        x, r, rate, step = _case(*shape, dtype, pad, residual, seed=sum(shape) + pad)
        drop = pbt.Dropout(rate, SEED, step, site=3, first_member=11)
        f = scales(*shape, rate.cpu().numpy(), SEED, step.cpu().numpy(), 3, 11)
        _verify(pbt.dropout_forward(x, drop, residual=r), x, r, f)
        _verify(pbt.dropout_backward(x, drop), x, None, f)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset", [1, 2, 4, 7])
@pytest.mark.parametrize("width", [24, 1000, 1001])
def test_bases_and_strides_of_any_alignment(width, offset, dtype):
    """x and residual at different distances from a vector's boundary, members closer together than rows (transposed)."""
    import torch
    import paper_1711_09846_b200 as pbt
    dt = getattr(torch, dtype)
    flat = torch.randn(2, 5 * 3 * width + 16, device="cuda").to(dt)
    x = flat[0, offset:offset + 15 * width].view(5, 3, width).transpose(0, 1)
    r = flat[1, 8 - offset:8 - offset + 15 * width].view(3, 5, width)
    f = scales(3, 5, width, [0.3] * 3, SEED, [5] * 3)
    drop = pbt.Dropout(0.3, SEED, 5)
    _verify(pbt.dropout_forward(x, drop, residual=r), x, r, f)
    _verify(pbt.dropout_forward(r, drop, residual=x), r, x, f)
    shared = r[:1].expand(3, 5, width)                 # one input for all members
    _verify(pbt.dropout_forward(shared, drop, residual=x), shared, x, f)
    repeated = r[:, :1].expand(3, 5, width)            # one row for all rows
    _verify(pbt.dropout_forward(repeated, drop), repeated, None, f)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rates_at_and_beyond_their_ends(dtype):
    import torch
    import paper_1711_09846_b200 as pbt
    values = [0.0, 1e-9, 2.0 ** -17, 1.5 * 2.0 ** -16, 2.5 * 2.0 ** -16, 0.5, 1 - 2.0 ** -16, 1 - 2.0 ** -18, 1.0, 1.5, -0.25, float("nan"), float("inf"),
              -float("inf")]
    rate = torch.tensor(values, device="cuda")
    m = len(values)
    x = torch.randn(m, 64, 1000, device="cuda").to(getattr(torch, dtype))
    x[x == 0] = 1
    f = scales(m, 64, 1000, values, 1, [0] * m)
    got = pbt.dropout_forward(x, pbt.Dropout(rate, 1, 0))
    _verify(got, x, None, f)
    for k in (0, 1, 10, 11, 13):
        assert torch.equal(got[k], x[k])
    for k in (7, 8, 9, 12):
        assert (got[k] == 0).all()
    assert torch.equal(pbt.dropout_forward(x, pbt.Dropout(0.0, 1, 0)), x) and (pbt.dropout_forward(x, pbt.Dropout(1, 1, 0)) == 0).all()


@pytest.mark.gpu
def test_what_is_dropped_is_zero_whatever_it_was():
    import torch
    import paper_1711_09846_b200 as pbt
    x = torch.ones(2, 9, 72, device="cuda", dtype=torch.bfloat16)
    drop = pbt.Dropout(0.5, 3, 4)
    zero = pbt.dropout_forward(x, drop) == 0
    for bad in (float("nan"), float("inf"), -float("inf")):
        for y in (pbt.dropout_forward(x * bad, drop), pbt.dropout_forward(x * bad, drop, residual=x)):
            assert torch.isfinite(y[zero]).all() and not torch.isfinite(y[~zero]).any()


@pytest.mark.gpu
def test_draws_follow_member_step_site_and_seed():
    """A shard draws what the whole population draws; steps beyond 32 bits count modulo 2^32; everything else that differs draws
    independently: two masks at rate 1/2 agree in half of n elements, give or take 6 sqrt(n) / 2."""
    import torch
    import paper_1711_09846_b200 as pbt
    x = torch.ones(6, 50, 333, device="cuda")
    step = torch.tensor([5, 6, 7, 2 ** 32 + 5, 9, 5], device="cuda")
    rate = torch.tensor([0.1, 0.2, 0.3, 0.5, 0.6, 0.9], device="cuda")
    whole = pbt.dropout_forward(x, pbt.Dropout(rate, SEED, step, 1))
    part = pbt.dropout_forward(x[2:5], pbt.Dropout(rate[2:5], SEED, step[2:5], 1, first_member=2))
    assert torch.equal(whole[2:5], part)
    one = pbt.dropout_forward(x[:1], pbt.Dropout(0.5, SEED, 5, 1, first_member=3))
    assert torch.equal(one[0], whole[3])
    base = pbt.dropout_forward(x, pbt.Dropout(0.5, SEED, 5)) == 0
    n, half = base[0].numel(), base.numel() / 2
    for other in (pbt.Dropout(0.5, SEED, 6), pbt.Dropout(0.5, SEED, 5, 1), pbt.Dropout(0.5, SEED + 1, 5), pbt.Dropout(0.5, SEED ^ 1 << 63, 5),
                  pbt.Dropout(0.5, SEED, 5, first_member=1)):
        agree = ((pbt.dropout_forward(x, other) == 0) == base)
        same = agree[:-1] if other.first_member else agree
        assert abs(same.sum().item() - same.numel() / 2) < 3 * same.numel() ** 0.5
    assert abs(base.sum().item() - half) < 3 * base.numel() ** 0.5 and abs((base[0] == base[1]).sum().item() - n / 2) < 3 * n ** 0.5
    # every column of a group is drawn by itself: over 300 rows the fractions of neighbours' agreement stay within 6 sigma
    cols = (pbt.dropout_forward(torch.ones(1, 4000, 16, device="cuda"), pbt.Dropout(0.5, 8, 9)) == 0)[0].double()
    agreement = (cols.T @ cols + (1 - cols).T @ (1 - cols)) / 4000
    agreement.fill_diagonal_(0.5)
    assert (agreement - 0.5).abs().max() < 3 / 4000 ** 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("width", [2047, 2048])
def test_activations_beyond_32_bit_offsets(width, dtype):
    """The last rows of more than 2^31 elements, in one member and as members that lie far apart."""
    import torch
    import paper_1711_09846_b200 as pbt
    rows = 1_100_000
    x = torch.empty(1, rows, width, device="cuda", dtype=getattr(torch, dtype)).fill_(1.5)
    y = pbt.dropout_forward(x, pbt.Dropout(0.25, 7, 8), residual=x)[0, -2:].clone()
    block = (np.arange(2, dtype=np.uint64)[:, None] + np.uint64(rows - 2)) * np.uint64(256) + np.arange(256, dtype=np.uint64)
    words = philox4x32_10_np(np.uint64(0), np.uint64(8), np.uint64(5), block, 7)
    bits = np.stack([w >> s & np.uint32(0xFFFF) for w in words for s in (np.uint32(0), np.uint32(16))], -1).reshape(2, 2048)[:, :width]
    assert torch.equal(y.cpu().double(), torch.from_numpy(np.where(bits >= 16384, 1.5 / 0.75, 0.0) + 1.5))
    far = x.view(-1)[:2 * rows * 1000].view(2, rows, 1000)[:, :3]       # (the second member 1.1e9 elements on)
    _verify(pbt.dropout_forward(far, pbt.Dropout(0.25, 7, 8)), far, None, scales(2, 3, 1000, [0.25] * 2, 7, [8] * 2))


@pytest.mark.gpu
def test_streams_and_graphs():
    import torch
    import paper_1711_09846_b200 as pbt
    x, r, rate, step = _case(3, 40, 200, "bfloat16")
    drop = pbt.Dropout(rate, SEED, step)
    want = pbt.dropout_forward(x, drop, residual=r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pbt.dropout_forward(x, drop, residual=r, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = pbt.dropout_forward(x, drop, residual=r)
        step += 1
    first = step.clone()
    for k in range(3):                                 # a replay draws for the steps and rates that it finds
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(step, first + k + 1)
        assert torch.equal(y, pbt.dropout_forward(x, pbt.Dropout(rate, SEED, first + k), residual=r))


def test_the_c_call_refuses_what_it_cannot_do():
    import paper_1711_09846_b200 as pbt
    from paper_1711_09846_b200.binding import PbtDropoutDesc
    lib = pbt.load_library()

    def call(**kw):
        d = PbtDropoutDesc()
        d.members, d.rows, d.width, d.dtype, d.x, d.x_row, d.y = 1, 0, 8, 1, 4096, 8, 8192
        d.rule.rate_all = 0.5
        for k, v in kw.items():
            setattr(d.rule if hasattr(d.rule, k) else d, k, v)
        return lib.pbt_dropout(C.byref(d), None)
    assert lib.pbt_dropout(None, None) == 1
    assert call() == 0                                 # no rows: nothing to do, nothing launched
    for code, kw in ((1, dict(members=0)), (1, dict(rows=-1)), (1, dict(width=0)), (2, dict(members=65536)), (2, dict(dtype=2)), (1, dict(site=-1)),
                     (1, dict(site=(1 << 30) + 1)), (1, dict(first_member=-1)), (1, dict(first_member=0x7FFFFFFF)), (1, dict(rate_all=1.25)),
                     (1, dict(rate_all=-0.5)), (1, dict(rate_all=float("nan"))), (2, dict(rows=1 << 22, width=1 << 13)), (1, dict(rows=1, x=None)),
                     (1, dict(rows=1, y=None))):
        assert call(**kw) == code, kw
        assert lib.pbt_last_error(None)


@pytest.mark.gpu
def test_refusals_and_empty_batches():
    import torch
    import paper_1711_09846_b200 as pbt
    x = torch.ones(2, 3, 16, device="cuda")
    ok = pbt.Dropout(0.5, 1, 2)
    assert pbt.dropout_forward(x[:, :0], ok).shape == (2, 0, 16)
    for a, r in ((x.cpu(), None), (x[0], None), (x.double(), None), (x, x.bfloat16()), (x, x[:1]), (x, x.cpu()), (x.transpose(1, 2), None), (x, x.transpose(1, 2))):
        with pytest.raises(ValueError):
            pbt.dropout_forward(a, ok, residual=r)
    two, three = torch.ones(2, device="cuda"), torch.ones(3, device="cuda")
    for drop in (pbt.Dropout(three, 1, 2), pbt.Dropout(0.5, 1, three.long())):           # of another number of members
        with pytest.raises(ValueError):
            pbt.dropout_forward(x, drop)
    for args in (dict(rate=two.cpu()), dict(rate=two.double()), dict(rate=torch.ones(4, device="cuda")[::2]), dict(rate=x[0]), dict(step=two), dict(step=two.long().cpu()),
                 dict(rate=two, step=three.long()), dict(step=-1), dict(step=1 << 63), dict(seed=-1), dict(seed=1 << 64), dict(site=-1), dict(site=1 << 31),
                 dict(first_member=-1), dict(first_member=1 << 32), dict(rate=1.5), dict(rate=-0.1), dict(rate=float("nan"))):
        with pytest.raises(ValueError):
            pbt.Dropout(**{**dict(rate=0.5, seed=1, step=2), **args})
    with pytest.raises(pbt.PbtError):
        pbt.dropout_forward(x, pbt.Dropout(0.5, 1, 2, first_member=0x7FFFFFFF))
