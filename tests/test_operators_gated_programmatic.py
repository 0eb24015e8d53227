"""Gated units and dropout behind a population whose kernels are launched programmatically (the setting of the handle used last applies to the process):
the same bits as in plain stream order."""
import pytest

from test_operators_gated import _case


def _use(programmatic):
    import torch
    import paper_1711_09846_b200 as pbt
    from workloads import get_config, make_inputs
    cfg = get_config("c3_mini")
    pbt.Population(cfg, make_inputs(cfg), programmatic_launches=programmatic).step(1)
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 1, 1024, 512), (16, 5, 512, 512), (9, 21, 333, 129), (5, 301, 501, 515), (4, 256, 512, 512), (30, 90, 256, 136)], ids=str)
def test_passes_behind_a_programmatic_population(shape, dtype):
    import torch
    import paper_1711_09846_b200 as pbt
    c = _case(*shape, dtype, seed=sum(shape))
    unit, rule = pbt.GatedUnit(c["weight"]), c["dropout"]

    def steps(pause):
        x, out = c["x"].clone(), []
        for keep in (True, False, True):
            h = unit.forward(x, dropout=rule, keep=keep)
            pause()
            h, kept = h if keep else (h, None)
            d = pbt.dropout_backward(c["dh"], rule)
            pause()
            dx, dweight = unit.backward(d, x, kept, dropout=rule)
            pause()
            x = pbt.dropout_forward(dx, rule, residual=x)
            pause()
            out += [h, d, dx, dweight, x]
        return out
    _use(False)
    expected = steps(torch.cuda.synchronize)
    try:
        _use(True)
        for _ in range(5):
            for a, b in zip(steps(lambda: None), expected):
                assert torch.equal(a, b)
    finally:
        _use(False)
    unit.check()
