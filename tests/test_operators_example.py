"""The example that runs adapters, block norms and clipping together (examples/adapter_population.py).

One step's gradients in fp32 against autograd of the formulas in 64 bits.  Each operator's fp32 error is below 1e-5 of its result's
largest element (sums of at most a few hundred fp32 terms); five of them in a row, and cancellation between the two terms of a norm's
gradient, leave 1e-4 of the largest element of each gradient."""
import importlib.util
import json
import os

import pytest


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "adapter_population.py")
    spec = importlib.util.spec_from_file_location("adapter_population", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _formulas(pop, p, x, target):
    import torch
    rms = lambda t: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)
    w, scale = pop.weight.double().cpu(), pop.adapter_scale.double().cpu()[:, None, None]
    u0 = rms(x) * p["w_in"][:, None]
    b = u0 @ w.T + scale * (u0 @ p["A"].transpose(1, 2)) @ p["B"].transpose(1, 2)
    y = x + pop.residual.double().cpu()[:, None, None] * torch.sigmoid(p["gate"])[:, None] * rms(b) * p["w_post"][:, None]
    u = rms(y) * p["w_out"][:, None]
    return u, (u - target).square().mean(dim=(1, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("members, rows, width, rank", [(3, 5, 33, 3), (4, 64, 128, 8), (1, 1, 16, 1)])
def test_a_step_of_the_example_has_the_formulas_gradients(members, rows, width, rank):
    import torch
    example = _example()
    pop = example.AdapterPopulation(members, rows, width, rank, torch.float32, seed=members)
    for k in ("B", "gate", "w_in", "w_post", "w_out"):              # away from the symmetric start
        pop.params[k].add_(torch.randn(pop.params[k].shape, generator=pop.gen, device="cuda") * 0.2)
    x = torch.randn(pop.shape, generator=pop.gen, device="cuda")
    target = torch.randn(pop.shape, generator=pop.gen, device="cuda")
    loss = pop.loss_and_gradients(x, target)
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in pop.params.items()}
    _, want = _formulas(pop, p, x.double().cpu(), target.double().cpu())
    want.sum().backward()
    assert torch.allclose(loss.double().cpu(), want.detach(), rtol=1e-5)
    for k, g in pop.grads.items():
        ref = p[k].grad
        assert (g.double().cpu() - ref).abs().max() <= 1e-4 * ref.abs().max() + 1e-9, k
    norms = pop.clip.run(pop.limit).double().cpu()
    ref = torch.stack([sum(p[k].grad[m].square().sum() for k in p).sqrt() for m in range(members)])
    assert torch.allclose(norms, ref, rtol=1e-4)
    after = torch.stack([sum(g[m].double().cpu().square().sum() for g in pop.grads.values()).sqrt() for m in range(members)])
    assert (after <= torch.minimum(ref, pop.limit.double().cpu()) * (1 + 1e-4)).all()
    pop.layer.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_population_learns_and_serves_every_member_as_it_trained(dtype):
    import torch
    example = _example()
    pop, first, last = example.train(members=10, rows=64, width=128, rank=4, steps=60, dtype=getattr(torch, dtype), seed=1)
    assert torch.isfinite(last).any() and last.min() < 0.7 * first.min()
    # single tokens of many requests give what the members' own batches give
    x = torch.randn((10, 3, 128), generator=pop.gen, device="cuda").to(pop.weight.dtype)
    offsets = torch.arange(11, dtype=torch.int32, device="cuda") * 3
    whole = pop.forward(x, offsets, pop.adapter_ids)[0].u.view(30, 128)
    served = pop.serve(x.view(30, 128), torch.arange(10, device="cuda", dtype=torch.int32).repeat_interleave(3))
    # bf16: S, b, y and u are rounded (2^-9 each) at places that differ with the kernels; fp32: sums in another order
    tol = 1e-5 if dtype == "float32" else 4 * 2.0 ** -8
    ok = torch.isfinite(whole)
    assert (served.float() - whole.float())[ok].abs().max() <= tol * whole.float()[ok].abs().max()
    pop.layer.check()


@pytest.mark.gpu
def test_the_example_runs_as_a_command(capsys):
    _example().main(["--members", "5", "--rows", "16", "--width", "64", "--rank", "4", "--steps", "12", "--requests", "7"])
    line = json.loads(capsys.readouterr().out)
    assert line["members"] == 5 and line["best_loss"] > 0
