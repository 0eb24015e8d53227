"""The operators of a feed-forward block together, as the example uses them."""
import json
import os
import subprocess
import sys

import pytest

from test_operators_dropout import scales

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import feed_forward_population
        return feed_forward_population
    finally:
        sys.path.pop(0)


def _reference(pop, x, target, seed):
    """Loss and gradients of the block in 64 bits, by autograd, with masks from the oracle's generator."""
    import torch
    m, rows, width = x.shape
    hidden = pop.unit.hidden
    p = {k: v.double().requires_grad_() for k, v in pop.params.items()}
    steps = pop.steps.cpu().numpy()

    def rms(v, w):
        return v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-6) * w[:, None]
    f = [torch.from_numpy(scales(m, rows, n, r.cpu().numpy(), seed, steps, site)).cuda()
         for site, (n, r) in enumerate(((hidden, pop.rate_hidden), (width, pop.rate_out)))]
    xd = x.double()
    g, u = (rms(xd, p["w_in"]) @ p["up"].transpose(1, 2)).chunk(2, -1)
    b = (torch.nn.functional.silu(g) * u * f[0]) @ p["down"].transpose(1, 2)
    out = rms(xd + b * f[1], p["w_out"])
    loss = (out - target.double()).square().mean(dim=(1, 2))
    return loss.detach(), dict(zip(p, torch.autograd.grad(loss.sum(), list(p.values()))))


# fp32: products of at most 1024 terms, each good to 1024 eps of its terms' magnitudes (6e-5), five of them one after the other: 5e-4 of a gradient's norm.
# bf16: every intermediate (u0, h, b, y, u, du, dy, db, dh, dg and du, dx) is rounded, 2^-8 at most and in either direction: a dozen of them add up to
# 4 x 2^-8 of the norm in quadrature; twice that.
@pytest.mark.parametrize("dtype, bound", [("float32", 5e-4), ("bfloat16", 2.0 ** -5)])
@pytest.mark.parametrize("members, rows, width, hidden", [(3, 40, 96, 136), (4, 200, 256, 384), (2, 5, 64, 100)])
def test_a_training_step_has_the_blocks_gradients(members, rows, width, hidden, dtype, bound):
    import torch
    ex = _example()
    dt = getattr(torch, dtype)
    pop = ex.FeedForwardPopulation(members, width, hidden, dt, seed=7)
    pop.steps += torch.arange(members, device="cuda") * 3
    x = torch.randn(members, rows, width, generator=pop.gen, device="cuda").to(dt)
    target = torch.randn(members, rows, width, generator=pop.gen, device="cuda").to(dt)
    loss = pop.loss_and_gradients(x, target)
    want_loss, want = _reference(pop, x, target, 7)
    assert ((loss.double() - want_loss).abs() <= bound * want_loss).all()
    for k, w in want.items():
        off = (pop.grads[k].double() - w).flatten(1).norm(dim=1) / w.flatten(1).norm(dim=1)
        assert (off <= bound).all(), (k, off)
    pop.unit.check()
    before = {k: v.clone() for k, v in pop.masters.items()}
    grads = {k: v.float().clone() for k, v in pop.grads.items()}      # (the step clips them in place)
    _, norms = pop.step(x, target)
    total = sum(g.double().flatten(1).square().sum(1) for g in grads.values()).sqrt()
    assert ((norms.double() - total).abs() <= 1e-5 * total).all()
    for k in before:
        scale = (pop.limit / norms).clamp_max(1.0) * pop.lr
        moved = scale.view(-1, *[1] * (before[k].dim() - 1)) * grads[k]
        assert torch.allclose(before[k] - pop.masters[k], moved, rtol=2.0 ** -7 if dtype == "bfloat16" else 1e-4, atol=1e-6), k


def test_a_step_is_repeated_bit_for_bit_and_a_shard_draws_like_the_whole():
    import torch
    import paper_1711_09846_b200 as pbt
    ex = _example()

    def run(k, steps=3):
        pop = ex.FeedForwardPopulation(4, 64, 96, torch.bfloat16, seed=3)
        gen = torch.Generator(device="cuda").manual_seed(5)
        losses = []
        for _ in range(steps):
            x, t = (torch.randn(4, 33, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
            losses.append(pop.step(x, t)[0])
        return torch.stack(losses), pop, x
    a, pop, x = run(0)
    b, _, _ = run(1)
    assert torch.equal(a, b)
    whole, kept = pop.unit.forward(x, dropout=pop.drop_hidden, keep=True)
    part = pbt.GatedUnit(pop.params["up"][2:]).forward(x[2:], dropout=pbt.Dropout(pop.rate_hidden[2:], 3, pop.steps[2:], first_member=2))
    assert torch.equal(whole[2:], part)


def test_a_captured_step_draws_anew_at_every_replay():
    import torch
    ex = _example()
    pop = ex.FeedForwardPopulation(3, 64, 96, torch.bfloat16, seed=3)
    x = torch.randn(3, 50, 64, generator=pop.gen, device="cuda").bfloat16()
    target = torch.zeros_like(x)
    pop.loss_and_gradients(x, target)
    start = {k: v.clone() for k, v in pop.masters.items()}

    def restart():
        for k, v in start.items():
            pop.masters[k].copy_(v)
            if pop.params[k] is not pop.masters[k]:
                pop.params[k].copy_(v)
        pop.steps.zero_()
    restart()
    want = [pop.step(x, target)[0].clone() for _ in range(3)]
    restart()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss, _ = pop.step(x, target)
    got = []
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        got.append(loss.clone())
    for w, g in zip(want, got):
        assert torch.equal(w, g)
    assert pop.steps.tolist() == [3, 3, 3]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_the_example_runs(dtype):
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "feed_forward_population.py"), "--members", "6", "--steps", "21", "--rows", "48",
                        "--width", "72", "--hidden", "88", "--dtype", dtype], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    out = json.loads(r.stdout)
    assert out["members"] == 6 and 0 <= out["best_member"] < 6 and out["first_loss"] > 0 and out["best_loss"] > 0
