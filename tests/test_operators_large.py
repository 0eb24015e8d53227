"""Operands of more than 2^31 elements and 2^32 bytes: the last rows against the definition in 64 bits.

Tolerances: bf16 results carry their rounding (2^-9 relative to the element) and, for the adapters, that of S (2^-9 of the low-rank
part); 2^-7 of the largest element covers both.  The clipped values and norms are those of the small tests."""
import math

import pytest

ROWS, WIDTH = 1_100_000, 2048


def _close(got, want, tol=2.0 ** -7):
    assert (got.double().cpu() - want).abs().max() <= tol * want.abs().max()


@pytest.mark.gpu
def test_norms_beyond_32_bit_offsets():
    import torch
    import paper_1711_09846_b200 as pbt
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty((1, ROWS, WIDTH), device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    w = torch.rand((1, WIDTH), generator=gen, device="cuda") + 0.5
    out = pbt.block_norm_forward(x, next_weight=w, keep=True)
    last, w64 = x[0, -3:].double().cpu(), w.double().cpu()
    root = torch.rsqrt(last.square().mean(-1, keepdim=True) + 1e-6)
    _close(out.u[0, -3:], last * root * w64)
    g = pbt.block_norm_backward(None, out.u, x, next_weight=w, rstd_next=out.rstd_next)
    du = out.u[0, -3:].double().cpu() * w64
    _close(g.dx[0, -3:], root * (du - last * root * (du * last * root).mean(-1, keepdim=True)))


@pytest.mark.gpu
def test_clip_beyond_32_bit_offsets():
    import torch
    import paper_1711_09846_b200 as pbt
    n = 2_200_000_001
    g = torch.full((n,), 0.5, device="cuda")
    norm = pbt.GradientClip([g]).run(2.0).item()
    want = 0.5 * math.sqrt(n)
    assert abs(norm - want) <= 40 * 2.0 ** -24 * want
    for k in (0, 2 ** 30, 2 ** 31 + 1, n - 1):
        assert abs(g[k].item() - 1.0 / want) <= 44 * 2.0 ** -24 / want


@pytest.mark.gpu
@pytest.mark.parametrize("inputs, outputs", [(WIDTH, 64), (64, WIDTH)])
def test_adapters_beyond_32_bit_offsets(inputs, outputs):
    import torch
    import paper_1711_09846_b200 as pbt
    gen = torch.Generator(device="cuda").manual_seed(7)

    def normal(*shape, scale=1.0):
        return torch.empty(shape, device="cuda", dtype=torch.bfloat16).normal_(0.0, scale, generator=gen)

    x, w, a, b = normal(ROWS, inputs), normal(outputs, inputs, scale=inputs ** -0.5), normal(2, 4, inputs, scale=inputs ** -0.5), normal(2, outputs, 4)
    scale = torch.tensor([1.0, 0.5], device="cuda")
    offsets = torch.tensor([0, ROWS - 2, ROWS], dtype=torch.int32, device="cuda")
    layer = pbt.AdapterProjection(w, a, b, scale)
    y = layer.forward(x, offsets, torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    last = x[-2:].double().cpu()
    _close(y[-2:], last @ w.double().cpu().T + 0.5 * (last @ a[1].double().cpu().T) @ b[1].double().cpu().T)
    layer.check()
