"""Gated units under another default type of torch: what a forward pass keeps is float32 all the same, as many bytes as the kernels write."""
import contextlib

import pytest

from recording_library import install, on_device


@contextlib.contextmanager
def _default(dtype):
    import torch
    before = torch.get_default_dtype()
    torch.set_default_dtype(dtype)
    try:
        yield
    finally:
        torch.set_default_dtype(before)


@pytest.mark.parametrize("default", ["bfloat16", "float16", "float64"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_what_is_kept_has_room_for_what_is_written(monkeypatch, default, dtype):
    import torch
    import paper_1711_09846_b200 as pbt
    lib = install(monkeypatch)
    with _default(getattr(torch, default)):
        x, w, dh = (on_device(torch.zeros(*shape, dtype=getattr(torch, dtype))) for shape in ((2, 3, 24), (2, 18, 24), (2, 3, 9)))
        unit = pbt.GatedUnit(w)
        h, kept = unit.forward(x, keep=True)
        assert kept.dtype is torch.float32 and kept.numel() * kept.element_size() == 2 * 3 * 2 * 16 * 4      # 9 hidden units, rounded up to 16
        dx, dweight = unit.backward(dh, x, kept)
    assert [name for name, _ in lib.calls] == ["forward", "backward"]
    assert all(t.dtype is x.dtype for t in (h, dx, dweight))


@pytest.mark.gpu
@pytest.mark.parametrize("default", ["bfloat16", "float64"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_results_do_not_depend_on_the_default_type(default, dtype):
    import torch
    import paper_1711_09846_b200 as pbt
    gen = torch.Generator().manual_seed(3)
    x, w, dh = (torch.randn(*shape, generator=gen).to(getattr(torch, dtype)).cuda() for shape in ((2, 70, 72), (2, 66, 72), (2, 70, 33)))

    def step():
        unit, drop = pbt.GatedUnit(w, "gelu"), pbt.Dropout(0.25, 3, 4)
        h, kept = unit.forward(x, dropout=drop, keep=True)
        assert kept.dtype is torch.float32
        return (h, kept[..., :33], *unit.backward(dh, x, kept, dropout=drop), pbt.dropout_forward(x, drop, residual=x))
    expected = step()
    with _default(getattr(torch, default)):
        for a, b in zip(step(), expected):
            assert a.dtype is b.dtype and torch.equal(a, b)
