"""A population that fine-tunes low-rank adapters on one frozen residual block, and serves them.

Every member has its own adapter (A, B), norm weights and gate beside the shared projection W:

    u0 = rms(x) w_in,   b = u0 W^T + scale (u0 A^T) B^T,   y = x + residual sigmoid(gate) rms(b) w_post,   u = rms(y) w_out

and learns to reproduce a hidden adapter from the mean squared error of u.  Gradients are clipped per member to the
member's own limit; learning rate and limit are the hyperparameters that the population searches: at every ready point
the worst fifth copies weights and hyperparameters of the best fifth and perturbs the latter.  At the end single
tokens of many requests go through the block at once, each with the adapter of the member it asks for.

    python examples/adapter_population.py [--members 16] [--rows 128] [--width 512] [--rank 8] [--steps 100] [--dtype bfloat16]
"""
from __future__ import annotations

import argparse
import json
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1711_09846_b200 as pbt


class AdapterPopulation:
    def __init__(self, members: int, rows: int, width: int, rank: int, dtype=torch.bfloat16, seed: int = 0):
        self.shape = (members, rows, width)
        self.gen = gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale=1.0):
            return torch.randn(shape, generator=gen, device="cuda") * scale

        self.weight = normal(width, width, scale=width ** -0.5).to(dtype)
        # what the kernels read, and the fp32 masters that the updates go to
        self.masters = {"A": normal(members, rank, width, scale=width ** -0.5), "B": torch.zeros(members, width, rank, device="cuda"),
                        "gate": torch.zeros(members, width, device="cuda"), "w_in": torch.ones(members, width, device="cuda"),
                        "w_post": torch.ones(members, width, device="cuda"), "w_out": torch.ones(members, width, device="cuda")}
        self.params = {k: v.to(dtype) if k in ("A", "B", "gate") else v for k, v in self.masters.items()}
        self.adapter_scale = torch.full((members,), 2.0, device="cuda")      # alpha / rank
        self.residual = torch.ones(members, device="cuda")
        self.lr = torch.logspace(-0.5, 1.5, members, device="cuda")
        self.limit = torch.full((members,), 0.1, device="cuda")
        self.layer = pbt.AdapterProjection(self.weight, self.params["A"], self.params["B"], self.adapter_scale)
        self.row_offsets = torch.arange(members + 1, dtype=torch.int32, device="cuda") * rows
        self.adapter_ids = torch.arange(members, dtype=torch.int32, device="cuda")
        # the gradients' places, and one clip group per member over its slices of them
        self.grads = {k: torch.zeros_like(v if k not in ("A", "B") else self.masters[k]) for k, v in self.params.items()}
        slices = [(g[m], m) for g in self.grads.values() for m in range(members)]
        self.clip = pbt.GradientClip([g for g, _ in slices], [m for _, m in slices])

    def forward(self, x, row_offsets, adapter_ids, params=None, residual=None, keep=False):
        """The block on x [members, rows, width] (or [1, tokens, width] with one segment per token)."""
        p = params or self.params
        residual = self.residual if residual is None else residual
        first = pbt.block_norm_forward(x, next_weight=p["w_in"], keep=keep)
        u0 = first.u.view(-1, x.shape[2])
        b, kept = self.layer.forward(u0, row_offsets, adapter_ids, keep=True) if keep else (self.layer.forward(u0, row_offsets, adapter_ids), None)
        b = b.view(x.shape)
        out = pbt.block_norm_forward(x, b, post_weight=p["w_post"], gate=p["gate"], scale=residual, next_weight=p["w_out"], keep=keep)
        return out, (first, u0, b, kept)

    def loss_and_gradients(self, x, target):
        """Loss of every member; leaves the gradients in self.grads."""
        p = self.params
        out, (first, u0, b, kept) = self.forward(x, self.row_offsets, self.adapter_ids, keep=True)
        error = out.u.float() - target.float()
        loss = error.square().mean(dim=(1, 2))
        du = (error * (2.0 / error[0].numel())).to(out.u.dtype)
        g = pbt.block_norm_backward(None, du, out.y, b, post_weight=p["w_post"], gate=p["gate"], scale=self.residual, next_weight=p["w_out"],
                                    rstd_block=out.rstd_block, rstd_next=out.rstd_next)
        du0, d_a, d_b = self.layer.backward(g.dblock.view(u0.shape), u0, kept, self.row_offsets, self.adapter_ids)
        g_in = pbt.block_norm_backward(None, du0.view(x.shape), x, next_weight=p["w_in"], rstd_next=first.rstd_next)
        new = {"A": d_a, "B": d_b, "gate": g.dgate, "w_in": g_in.dnext_weight, "w_post": g.dpost_weight, "w_out": g.dnext_weight}
        for k, v in new.items():
            self.grads[k].copy_(v)
        return loss

    def step(self, x, target):
        """One training step of all members: loss and gradient norm of each (both before the update)."""
        loss = self.loss_and_gradients(x, target)
        norms = self.clip.run(self.limit)
        for k, master in self.masters.items():
            lr = self.lr.view(-1, *[1] * (master.dim() - 1))
            master.sub_(lr * self.grads[k])
            if self.params[k] is not master:
                self.params[k].copy_(master)
        return loss, norms

    def exploit_explore(self, fitness):
        """Truncation selection: the worst fifth takes over weights and hyperparameters of a member of the best fifth."""
        n = max(1, fitness.numel() // 5)
        order = torch.nan_to_num(fitness, nan=-float("inf")).argsort(descending=True)
        best, worst = order[:n], order[-n:]
        source = best[torch.randint(n, (n,), generator=self.gen, device="cuda")]
        for t in (*self.masters.values(), self.lr, self.limit):
            t[worst] = t[source]
        for k, master in self.masters.items():
            if self.params[k] is not master:
                self.params[k].copy_(master)
        for t in (self.lr, self.limit):
            factor = torch.where(torch.rand(n, generator=self.gen, device="cuda") < 0.5, 0.8, 1.2)
            t[worst] = t[worst] * factor

    def serve(self, tokens, members):
        """u of single tokens [requests, width], request i through member members[i]'s block, all in one pass."""
        n = tokens.shape[0]
        offsets = torch.arange(n + 1, dtype=torch.int32, device="cuda")
        index = members.long()
        params = {k: self.params[k][index] for k in ("w_in", "w_post", "w_out", "gate")}
        # a token is a "member" of one row with its own norm weights, and a segment of one row with its own adapter
        return self.forward(tokens.view(n, 1, -1), offsets, members.int(), params, self.residual[index])[0].u.view(n, -1)


def hidden_target(pop: AdapterPopulation, x, strength: float = 1.0):
    """u of x [members, rows, width] behind a hidden adapter that no member has."""
    _, _, width = pop.shape
    rank = pop.params["A"].shape[1]
    gen = torch.Generator(device="cuda").manual_seed(1234)
    a = torch.randn((1, rank, width), generator=gen, device="cuda").mul_(width ** -0.5).to(pop.weight.dtype)
    b = torch.randn((1, width, rank), generator=gen, device="cuda").mul_(strength * rank ** -0.5).to(pop.weight.dtype)
    flat = x.reshape(1, -1, width)
    one = torch.ones((1, width), device="cuda")
    teacher = pbt.AdapterProjection(pop.weight, a, b, torch.ones(1, device="cuda"))
    rows = flat.shape[1]
    u0 = pbt.block_norm_forward(flat, next_weight=one).u.view(rows, width)
    out = teacher.forward(u0, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    return pbt.block_norm_forward(flat, out.view(flat.shape), post_weight=one, gate=torch.zeros((1, width), device="cuda", dtype=x.dtype),
                                  next_weight=one).u.view(x.shape)


def train(members=16, rows=128, width=512, rank=8, steps=100, ready_every=10, dtype=torch.bfloat16, seed=0):
    pop = AdapterPopulation(members, rows, width, rank, dtype, seed)
    first = loss = None
    for step in range(steps):
        x = torch.randn((members, rows, width), generator=pop.gen, device="cuda").to(dtype)
        loss, _ = pop.step(x, hidden_target(pop, x))
        first = loss if first is None else first
        if (step + 1) % ready_every == 0:
            pop.exploit_explore(-loss)
    return pop, first, loss


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("members", 16), ("rows", 128), ("width", 512), ("rank", 8), ("steps", 100), ("requests", 32)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=["bfloat16", "float32"], default="bfloat16")
    args = ap.parse_args(argv)
    pop, first, last = train(args.members, args.rows, args.width, args.rank, args.steps, dtype=getattr(torch, args.dtype))
    pop.layer.check()
    tokens = torch.randn((args.requests, args.width), generator=pop.gen, device="cuda").to(pop.weight.dtype)
    members = torch.randint(args.members, (args.requests,), generator=pop.gen, device="cuda", dtype=torch.int32)
    served = pop.serve(tokens, members)
    error = (served.float() - hidden_target(pop, tokens.view(1, *tokens.shape)).view(served.shape).float()).square().mean()
    print(json.dumps({"members": args.members, "steps": args.steps, "first_loss": round(first.min().item(), 5), "best_loss": round(last.min().item(), 5),
                      "best_member": int(last.argmin()), "best_lr": round(pop.lr[last.argmin()].item(), 4), "served_error": round(error.item(), 5)}))


if __name__ == "__main__":
    main()
