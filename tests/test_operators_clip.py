"""Gradient clipping (GradientClip / pbt_clip_*) against the definition in 64 bits.

Tolerances.  A chunk's squares are summed in fp32 by 256 threads, at most 64 terms each, then in a
tree, and the chunks' sums in fp64: relative error of the sum of squares below (64 + 8) 2^-24, of the norm half of that,
plus one rounding: 40 2^-24 = 2.4e-6.  A clipped element has the norm's error, one division and one multiplication on top:
2.6e-6 in fp32; in bf16 its rounding (2^-8) dominates."""
import ctypes as C
import math

import pytest

NORM_TOL = 40 * 2.0 ** -24
OUT_TOL = {"float32": 44 * 2.0 ** -24, "bfloat16": 2.0 ** -8 + 44 * 2.0 ** -24}


def _reference(grads, groups, n_groups, limits):
    import torch
    total = torch.zeros(n_groups, dtype=torch.float64)
    for g, k in zip(grads, groups):
        total[k] += (g.detach().cpu().double() ** 2).sum()
    norms = total.sqrt()
    out = []
    for g, k in zip(grads, groups):
        n, lim = norms[k].item(), float(limits[k])
        f = 1.0 if (math.isinf(lim) or n <= lim) else (lim / n if n == n else math.nan)
        out.append(g.detach().cpu().double() * f)
    return norms, out


def _check(norms, out, ref_norms, ref_out):
    import torch
    got = norms.cpu().double()
    assert torch.allclose(got, ref_norms, rtol=NORM_TOL, atol=0, equal_nan=True), (got, ref_norms)
    for o, r in zip(out, ref_out):
        tol = OUT_TOL[str(o.dtype).replace("torch.", "")]
        assert torch.allclose(o.cpu().double(), r, rtol=tol, atol=1e-38, equal_nan=True)


SIZES = {
    "one element": [1],
    "odd, unaligned": [1, 7, 8, 9, 31, 33, 255, 1023, 4097],
    "around a chunk": [16383, 16384, 16385, 32768 + 5, 3],
    "empty among them": [0, 5, 0, 129, 0],
    "large": [3_000_001, 1_000_003],
    "beyond the shared memory of all SMs": [17_000_003, 33, 5, 70_001],
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", sorted(SIZES))
def test_clip_matches_the_definition(case, dtype, in_place):
    import torch
    import paper_1711_09846_b200 as pbt
    gen = torch.Generator(device="cuda").manual_seed(len(case))
    sizes = SIZES[case]
    for lead in (0, 1, 3):                # the packed tensors start at every alignment, source and destination differently
        flat = torch.randn(sum(sizes) + lead, generator=gen, device="cuda").mul_(0.1).to(getattr(torch, dtype))
        grads = list(flat[lead:].split(sizes))
        dest = torch.full((sum(sizes) + 2,), 7.0, device="cuda", dtype=flat.dtype)
        out = None if in_place else list(dest[1:-1].split(sizes))
        groups = [k % 2 for k in range(len(sizes))]
        ref_norms, _ = _reference(grads, groups, 3, [1, 1, 1])
        limits = torch.tensor([0.5 * ref_norms[0], 2.0 * ref_norms[1] + 1, 1.0])   # one clipped, one not, one group empty
        ref_norms, ref_out = _reference(grads, groups, 3, limits)
        before = flat.clone()
        clip = pbt.GradientClip(grads, groups, out=out, n_groups=3)
        norms = clip.run(limits.float().cuda())
        _check(norms, grads if in_place else out, ref_norms, ref_out)
        assert norms[2].item() == 0.0
        if not in_place:
            assert torch.equal(flat, before)
            assert dest[0].item() == 7.0 and dest[-1].item() == 7.0     # nothing beyond the destinations
        else:
            assert torch.equal(flat[:lead], before[:lead])


@pytest.mark.gpu
def test_clip_a_number_for_every_group_and_runs_are_reproducible():
    import torch
    import paper_1711_09846_b200 as pbt
    gen = torch.Generator(device="cuda").manual_seed(3)
    grads = [torch.randn(n, generator=gen, device="cuda") for n in (70_001, 513, 40_000)]
    out = [torch.empty_like(g) for g in grads]
    clip = pbt.GradientClip(grads, out=out)
    first = clip.run(2.5)
    kept = [o.clone() for o in out]
    ref_norms, ref_out = _reference(grads, [0, 0, 0], 1, [2.5])
    _check(first, out, ref_norms, ref_out)
    for _ in range(3):
        assert torch.equal(clip.run(2.5), first)
        assert all(torch.equal(a, b) for a, b in zip(out, kept))
    assert abs(torch.cat(out).double().norm().item() - 2.5) < 2.5 * OUT_TOL["float32"]


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_clip_a_diverged_member_touches_nobody_else(bad):
    import torch
    import paper_1711_09846_b200 as pbt
    grads = [torch.ones(5000, device="cuda") for _ in range(3)]
    grads[1][4321] = bad
    out = [torch.empty_like(g) for g in grads]
    norms = pbt.GradientClip(grads, [0, 1, 2], out=out).run(1.0).cpu()
    for k in (0, 2):
        assert abs(norms[k].item() - math.sqrt(5000)) < math.sqrt(5000) * NORM_TOL
        assert torch.isfinite(out[k]).all()
    if math.isnan(bad):
        assert math.isnan(norms[1].item()) and torch.isnan(out[1]).all()
    else:
        assert math.isinf(norms[1].item())
        rest = torch.cat([out[1][:4321], out[1][4322:]])
        assert (rest == 0).all() and math.isnan(out[1][4321].item())


@pytest.mark.gpu
@pytest.mark.parametrize("count", [20_000, 8_000_000])
@pytest.mark.parametrize("value", [1e25, 1e-25, 0.0])
def test_clip_squares_beyond_the_range_of_fp32(value, count):
    import torch
    import paper_1711_09846_b200 as pbt
    g = torch.full((count,), value, device="cuda")
    out = torch.empty_like(g)
    clip = pbt.GradientClip([g], out=[out])
    norm = clip.run(value).item()
    want = float(g[0].double().item()) * math.sqrt(count)
    assert abs(norm - want) <= want * NORM_TOL
    if value:
        assert abs(out[7].item() - want / count) <= want / count * OUT_TOL["float32"] * 2


@pytest.mark.gpu
@pytest.mark.parametrize("groups, n_groups", [([0, 1, 2, 3], 6), ([3, 1, 0, 1], 6), ([5, 5, 5, 5], 6), ([2, 0, 2, 1], 3)])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip_many_megabytes_in_several_groups(groups, n_groups, in_place):
    """Groups larger than L2's part, small ones and empty ones, in every order."""
    import torch
    import paper_1711_09846_b200 as pbt
    gen = torch.Generator(device="cuda").manual_seed(n_groups)
    grads = [torch.randn(n, generator=gen, device="cuda") for n in (13_000_001, 4_000_003, 9_000_000, 17)]
    out = None if in_place else [torch.empty_like(g) for g in grads]
    limits = [0.5 + k for k in range(n_groups)]
    ref_norms, ref_out = _reference(grads, groups, n_groups, limits)
    norms = pbt.GradientClip(grads, groups, out=out, n_groups=n_groups).run(torch.tensor(limits, device="cuda"))
    _check(norms, grads if in_place else out, ref_norms, ref_out)


@pytest.mark.gpu
def test_clip_on_another_stream():
    import torch
    import paper_1711_09846_b200 as pbt
    side = torch.cuda.Stream()
    g = torch.randn(1_000_003, device="cuda")
    out = torch.empty_like(g)
    clip = pbt.GradientClip([g], out=[out])
    side.wait_stream(torch.cuda.current_stream())
    norms = clip.run(1.0, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    ref_norms, ref_out = _reference([g], [0], 1, [1.0])
    _check(norms, [out], ref_norms, ref_out)


@pytest.mark.gpu
def test_clip_refusals():
    import torch
    import paper_1711_09846_b200 as pbt
    a = torch.zeros(100, device="cuda")
    for grads, kw in (([], {}), ([a.half()], {}), ([a[::2]], {}), ([a.cpu()], {}), ([a], dict(groups=[0, 1])),
                      ([a], dict(out=[torch.zeros(99, device="cuda")])), ([a], dict(out=[a.bfloat16()]))):
        with pytest.raises(ValueError):
            pbt.GradientClip(grads, **kw)
    for grads, kw in (([a], dict(groups=[-1], n_groups=1)), ([a], dict(groups=[4], n_groups=2)),
                      ([a[:60], a[50:]], {}), ([a[:50]], dict(out=[a[20:70]]))):
        with pytest.raises(pbt.PbtError):
            pbt.GradientClip(grads, **kw)
    clip = pbt.GradientClip([a])
    with pytest.raises(ValueError):
        clip.run(torch.ones(2, device="cuda"))
    with pytest.raises(pbt.PbtError):
        clip.run(-1.0)
    with pytest.raises(pbt.PbtError):
        clip.run(math.nan)


def test_clip_arguments_are_checked_before_the_device_is_touched():
    import paper_1711_09846_b200 as pbt
    from paper_1711_09846_b200.binding import PbtClipTensor
    lib = pbt.load_library()
    n = C.c_size_t(0)
    t = (PbtClipTensor * 1)()
    t[0].src, t[0].dst, t[0].numel = 4096, 4096, 1000
    assert lib.pbt_clip_query_workspace(t, 1, 1, C.byref(n)) == 0 and n.value % 256 == 0 and n.value > 0
    assert lib.pbt_clip_query_workspace(t, 1, 1, None) == 1
    assert lib.pbt_clip_query_workspace(t, 1, 0, C.byref(n)) == 1
    assert lib.pbt_clip_query_workspace(None, 1, 1, C.byref(n)) == 1
    h = C.c_void_p(None)
    assert lib.pbt_clip_create(C.byref(h), t, 1, 1, None, 0, None) == 3 and not h.value
    for field, value, code in (("numel", -1, 1), ("src", None, 1), ("src", 4097, 1), ("dtype", 2, 2), ("group", 1, 1)):
        keep = getattr(t[0], field)
        setattr(t[0], field, value)
        assert lib.pbt_clip_query_workspace(t, 1, 1, C.byref(n)) == code, field
        assert lib.pbt_last_error(None)
        setattr(t[0], field, keep)
    assert lib.pbt_clip_run(None, 1.0, None, None, None) == 1
    assert lib.pbt_clip_destroy(None) == 0


@pytest.mark.gpu
def test_clip_norms_may_take_the_place_of_the_limits():
    import torch
    import paper_1711_09846_b200 as pbt
    grads = [torch.randn(n, device="cuda") for n in (70_001, 5, 40_000)]
    out = [torch.empty_like(g) for g in grads]
    limits = [2.5, 0.25, 1e6]
    both = torch.tensor(limits, device="cuda")
    clip = pbt.GradientClip(grads, [0, 1, 2], out=out)
    assert clip.lib.pbt_clip_run(clip._handle, 0.0, both.data_ptr(), both.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    ref_norms, ref_out = _reference(grads, [0, 1, 2], 3, limits)
    _check(both, out, ref_norms, ref_out)
