"""What a caller changes between two calls of the same sizes: the next call goes by it, or is refused."""
import pytest

from recording_library import install, on_device

CHANGES = [("rate", 0.25), ("seed", 99), ("step", 12), ("site", 3), ("first_member", 5)]


def _told(rule):
    return dict(rate=rule.rate_all, seed=rule.seed, step=rule.step, site=rule.site, first_member=rule.first_member)


@pytest.mark.parametrize("name, value", CHANGES)
@pytest.mark.parametrize("gated", [False, True])
def test_a_dropout_that_is_changed_is_what_the_next_call_is_told(monkeypatch, name, value, gated):
    import torch
    import paper_1711_09846_b200 as pbt
    lib = install(monkeypatch)
    x, dh = (on_device(torch.zeros(2, 3, n)) for n in (16, 8))
    unit = pbt.GatedUnit(on_device(torch.zeros(2, 16, 16)))
    drop = pbt.Dropout(0.5, 7, 11, 1, 2)

    def call():
        if gated:
            unit.forward(x, dropout=drop)
            unit.backward(dh, x, dropout=drop)
        else:
            pbt.dropout_forward(x, drop, residual=x)
            pbt.dropout_backward(x, drop)
        return [_told(r) for r in lib.rules[-2:]]
    before = dict(rate=0.5, seed=7, step=11, site=1, first_member=2)
    assert call() == [before, before]
    setattr(drop, name, value)
    assert getattr(drop, name) == value and call() == [{**before, name: value}] * 2
    drop.step += 1
    assert call() == [{**before, name: value, "step": (value if name == "step" else 11) + 1}] * 2


def test_a_dropout_takes_tensors_in_the_place_of_numbers_and_the_other_way_round(monkeypatch):
    import torch
    import paper_1711_09846_b200 as pbt
    lib = install(monkeypatch)
    x = on_device(torch.zeros(2, 3, 16))
    rate, step = on_device(torch.zeros(2)), on_device(torch.zeros(2, dtype=torch.int64))
    drop = pbt.Dropout(0.5, 7, 11)
    pbt.dropout_forward(x, drop)
    drop.rate, drop.step = rate, step
    drop.step += 1                                     # in place, and the same tensor again
    pbt.dropout_forward(x, drop)
    assert (lib.rules[-1].rate, lib.rules[-1].steps) == (rate.data_ptr(), step.data_ptr()) and step.tolist() == [1, 1]
    drop.rate = 0.25
    pbt.dropout_forward(x, drop)
    assert (lib.rules[-1].rate, lib.rules[-1].rate_all, lib.rules[-1].steps) == (None, 0.25, step.data_ptr())


def test_what_a_dropout_cannot_be_changed_to_leaves_it_as_it_was(monkeypatch):
    import torch
    import paper_1711_09846_b200 as pbt
    lib = install(monkeypatch)
    x = on_device(torch.zeros(2, 3, 16))
    drop = pbt.Dropout(0.5, 7, 11, 1, 2)
    pbt.dropout_forward(x, drop)
    three = on_device(torch.zeros(3))
    for name, bad in (("rate", 1.5), ("rate", float("nan")), ("rate", three.double()), ("seed", -1), ("step", -1), ("step", three), ("site", (1 << 30) + 1),
                      ("first_member", -1)):
        with pytest.raises(ValueError):
            setattr(drop, name, bad)
    pbt.dropout_forward(x, drop)
    assert _told(lib.rules[-1]) == _told(lib.rules[0])
    drop.rate = three                                  # one rate too many for these activations, in whatever order they meet
    with pytest.raises(ValueError):
        pbt.dropout_forward(x, drop)
    with pytest.raises(ValueError):
        drop.step = on_device(torch.zeros(2, dtype=torch.int64))
    with pytest.raises(AttributeError):
        drop.stage = 1


@pytest.mark.gpu
@pytest.mark.parametrize("name, value", CHANGES)
def test_the_masks_of_a_changed_dropout_are_those_of_a_new_one(name, value):
    import torch
    import paper_1711_09846_b200 as pbt
    args = dict(rate=0.5, seed=7, step=11, site=1, first_member=2)
    x = torch.ones(2, 40, 200, device="cuda")
    unit = pbt.GatedUnit(torch.randn(2, 64, 200, device="cuda"), "sigmoid")
    drop = pbt.Dropout(**args)

    def masks(d):
        return pbt.dropout_forward(x, d), unit.forward(x, dropout=d)
    first = masks(drop)
    setattr(drop, name, value)
    for was, got, want in zip(first, masks(drop), masks(pbt.Dropout(**{**args, name: value}))):
        assert torch.equal(got, want) and not torch.equal(got, was)


def test_a_dropout_follows_its_tensors_to_other_memory(monkeypatch):
    """A tensor whose storage is replaced (p.data = ..., which flattening optimizers and module moves do) is read where it lies now."""
    import torch
    import paper_1711_09846_b200 as pbt
    lib = install(monkeypatch)
    x = on_device(torch.zeros(2, 3, 16))
    unit = pbt.GatedUnit(on_device(torch.zeros(2, 16, 16)))
    rate, step = on_device(torch.zeros(2)), on_device(torch.zeros(2, dtype=torch.int64))
    drop = pbt.Dropout(rate, 7, step)

    def told():
        pbt.dropout_forward(x, drop)
        unit.forward(x, dropout=drop)
        assert _places(lib.rules[-1]) == _places(lib.rules[-2])
        return _places(lib.rules[-1])
    old = told()
    assert old == (rate.data_ptr(), step.data_ptr())
    other = on_device(torch.ones(2)), on_device(torch.ones(2, dtype=torch.int64))
    rate.data = other[0]
    assert told() == (other[0].data_ptr(), old[1])
    step.data = other[1]
    assert told() == (other[0].data_ptr(), other[1].data_ptr())
    for bad in (torch.zeros(3), torch.zeros(2, dtype=torch.float64), torch.zeros(4)[::2]):
        rate.data = on_device(bad)
        with pytest.raises(ValueError):
            pbt.dropout_forward(x, drop)
        with pytest.raises(ValueError):
            unit.forward(x, dropout=drop)
    rate.data = other[0][:1]                           # the same place, one rate too few
    with pytest.raises(ValueError):
        pbt.dropout_forward(x, drop)
    rate.data = other[0]
    assert told() == (other[0].data_ptr(), other[1].data_ptr())


def _places(rule):
    return rule.rate, rule.steps


def test_a_unit_follows_its_weight_to_other_memory(monkeypatch):
    """The same for a weight, in calls of sizes that were seen before; another geometry is refused."""
    import torch
    import paper_1711_09846_b200 as pbt
    lib = install(monkeypatch)
    x, dh = (on_device(torch.zeros(2, 3, n)) for n in (16, 8))
    w = on_device(torch.zeros(2, 16, 16))
    unit = pbt.GatedUnit(w)

    def told():
        _, kept = unit.forward(x, keep=True)
        unit.backward(dh, x, kept)
        places = {d.weight for _, d in lib.calls[-2:]}
        assert len(places) == 1 and all((d.weight_member, d.weight_row) == (256, 16) for _, d in lib.calls[-2:])
        return places.pop()
    assert told() == w.data_ptr()
    other = on_device(torch.ones(2, 16, 16))
    old, w.data = w.data_ptr(), other
    assert told() == other.data_ptr() != old
    assert unit.weight is w
    seen = len(lib.calls)
    for bad in (torch.zeros(2, 16, 18)[..., :16], torch.zeros(2, 16, 16).transpose(1, 2), torch.zeros(2, 18, 16), torch.zeros(1, 16, 16).expand(2, 16, 16),
                torch.zeros(2, 16, 16, dtype=torch.bfloat16)):
        w.data = on_device(bad)
        for call in (lambda: unit.forward(x), lambda: unit.backward(dh, x)):
            with pytest.raises(ValueError):
                call()
    assert len(lib.calls) == seen
    w.data = other
    assert told() == other.data_ptr()
    for name, value in (("weight", other), ("hidden", 4)):
        with pytest.raises(AttributeError):
            setattr(unit, name, value)
    assert unit.hidden == 8


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [3, 100, 400])
def test_results_of_tensors_that_were_moved(rows, dtype):
    """Weight, rates and steps in other memory (the weight's at another alignment, too), the old memory overwritten: the bits of new objects."""
    import torch
    import paper_1711_09846_b200 as pbt
    gen = torch.Generator().manual_seed(rows)
    x, w, dh = (torch.randn(*shape, generator=gen).to(getattr(torch, dtype)).cuda() for shape in ((2, rows, 72), (2, 80, 72), (2, rows, 40)))
    rate, step = torch.full((2,), 0.3, device="cuda"), torch.tensor([4, 5], device="cuda")
    unit, drop = pbt.GatedUnit(w), pbt.Dropout(rate, 7, step)

    def run(unit, drop):
        h, kept = unit.forward(x, dropout=drop, keep=True)
        return (h, *unit.backward(dh, x, kept, dropout=drop), pbt.dropout_forward(x, drop))
    run(unit, drop)
    for by in (0, 1, 8):
        olds = [t.data for t in (w, rate, step)]
        place = torch.empty(w.numel() + 8, dtype=w.dtype, device="cuda")[by:by + w.numel()].view(w.shape)
        w.data, rate.data, step.data = place.copy_(w).mul_(1 + by), torch.full((2,), 0.2 + by / 32, device="cuda"), step + 1 + by
        for old in olds:
            old.fill_(float("nan") if old.is_floating_point() else 1 << 20)
        for a, b in zip(run(unit, drop), run(pbt.GatedUnit(w), pbt.Dropout(rate, 7, step))):
            assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    unit.check()
