"""A population of residual feed-forward blocks with gated units and dropout.

Every member has its own block

    u0 = rms(x) w_in,   h = drop_hidden(silu(u0 Wg^T) * (u0 Wu^T)),   y = x + drop_out(h Wd^T),   u = rms(y) w_out

and learns a hidden teacher block from the mean squared error of u, from noisy targets.  Gradients are clipped per member to the member's own limit; learning
rate, limit and the two dropout rates are the hyperparameters that the population searches: at every ready point the worst fifth copies weights and
hyperparameters of the best fifth (by the loss without dropout on held-out rows) and perturbs the latter.  A member's masks follow from (seed, member, its
own step): a run can be repeated, and a member that was copied goes on with its own draws.

    python examples/feed_forward_population.py [--members 10] [--rows 128] [--width 256] [--hidden 512] [--steps 60] [--dtype bfloat16]
"""
from __future__ import annotations

import argparse
import json
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1711_09846_b200 as pbt


class FeedForwardPopulation:
    def __init__(self, members: int, width: int, hidden: int, dtype=torch.bfloat16, seed: int = 0, activation: str = "silu"):
        self.gen = gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale=1.0):
            return torch.randn(shape, generator=gen, device="cuda") * scale

        # what the kernels read, and the fp32 masters that the updates go to
        self.masters = {"up": normal(members, 2 * hidden, width, scale=width ** -0.5), "down": normal(members, width, hidden, scale=hidden ** -0.5),
                        "w_in": torch.ones(members, width, device="cuda"), "w_out": torch.ones(members, width, device="cuda")}
        self.params = {k: v.to(dtype) if k in ("up", "down") else v for k, v in self.masters.items()}
        self.unit = pbt.GatedUnit(self.params["up"], activation)
        self.lr = torch.logspace(-1.5, 0.5, members, device="cuda")
        self.limit = torch.full((members,), 0.5, device="cuda")
        self.rate_hidden = torch.empty(members, device="cuda").uniform_(0.0, 0.4, generator=gen)
        self.rate_out = torch.empty(members, device="cuda").uniform_(0.0, 0.4, generator=gen)
        self.steps = torch.zeros(members, dtype=torch.int64, device="cuda")      # every member's own
        self.drop_hidden = pbt.Dropout(self.rate_hidden, seed, self.steps, site=0)
        self.drop_out = pbt.Dropout(self.rate_out, seed, self.steps, site=1)
        # the gradients' places, and one clip group per member over its slices of them
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        slices = [(g[m], m) for g in self.grads.values() for m in range(members)]
        self.clip = pbt.GradientClip([g for g, _ in slices], [m for _, m in slices])
        self.status = torch.zeros(8, dtype=torch.int32, device="cuda")

    def product(self, a, b, out, **layout):
        """A member-batched product on the current stream (see grouped_gemm)."""
        pbt.grouped_gemm(a, b, out, status=self.status, stream=torch.cuda.current_stream(), **layout)
        return out

    def forward(self, x, train: bool = False):
        """The blocks on x [members, rows, width]; with `train`, dropped, and with what the backward pass takes."""
        p = self.params
        first = pbt.block_norm_forward(x, next_weight=p["w_in"], keep=train)
        h, kept = self.unit.forward(first.u, dropout=self.drop_hidden, keep=True) if train else (self.unit.forward(first.u), None)
        b = self.product(h, p["down"], torch.empty_like(x))
        y = pbt.dropout_forward(b, self.drop_out, residual=x) if train else x + b
        out = pbt.block_norm_forward(y, next_weight=p["w_out"], keep=train)
        return out.u, (first, h, kept, y, out)

    def loss_and_gradients(self, x, target):
        """Loss of every member; leaves the gradients in self.grads."""
        p, g = self.params, self.grads
        u, (first, h, kept, y, out) = self.forward(x, train=True)
        error = u.float() - target.float()
        loss = error.square().mean(dim=(1, 2))
        du = (error * (2.0 / error[0].numel())).to(u.dtype)
        last = pbt.block_norm_backward(None, du, y, next_weight=p["w_out"], rstd_next=out.rstd_next)
        db = pbt.dropout_backward(last.dx, self.drop_out)
        dh = self.product(db, p["down"], torch.empty_like(h), b_mn=True)
        self.product(db, h, g["down"], a_mn=True, b_mn=True)
        du0, d_up = self.unit.backward(dh, first.u, kept, dropout=self.drop_hidden)
        g_in = pbt.block_norm_backward(None, du0, x, next_weight=p["w_in"], rstd_next=first.rstd_next)
        for k, v in (("up", d_up), ("w_in", g_in.dnext_weight), ("w_out", last.dnext_weight)):
            g[k].copy_(v)
        return loss

    def step(self, x, target):
        """One training step of all members: loss and gradient norm of each (both before the update)."""
        loss = self.loss_and_gradients(x, target)
        norms = self.clip.run(self.limit)
        for k, master in self.masters.items():
            master.sub_(self.lr.view(-1, *[1] * (master.dim() - 1)) * self.grads[k])
            if self.params[k] is not master:
                self.params[k].copy_(master)
        self.steps += 1
        return loss, norms

    def evaluate(self, x, target):
        """Loss of every member without dropout."""
        return (self.forward(x)[0].float() - target.float()).square().mean(dim=(1, 2))

    def exploit_explore(self, fitness):
        """Truncation selection: the worst fifth takes over weights and hyperparameters of a member of the best fifth, and perturbs the latter."""
        n = max(1, fitness.numel() // 5)
        order = torch.nan_to_num(fitness, nan=-float("inf")).argsort(descending=True)
        best, worst = order[:n], order[-n:]
        source = best[torch.randint(n, (n,), generator=self.gen, device="cuda")]
        searched = (self.lr, self.limit, self.rate_hidden, self.rate_out)
        for t in (*self.masters.values(), *searched):
            t[worst] = t[source]
        for k, master in self.masters.items():
            if self.params[k] is not master:
                self.params[k].copy_(master)
        for t in searched:
            t[worst] *= torch.where(torch.rand(n, generator=self.gen, device="cuda") < 0.5, 0.8, 1.2)
        for t in (self.rate_hidden, self.rate_out):
            t.clamp_(0.0, 0.9)


def train(members=10, rows=128, width=256, hidden=512, steps=60, ready_every=10, dtype=torch.bfloat16, seed=0, noise=0.3):
    pop = FeedForwardPopulation(members, width, hidden, dtype, seed)
    teacher = FeedForwardPopulation(1, width, hidden, dtype, seed=1234)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)

    def batch(n):
        x = torch.randn((1, n, width), generator=gen, device="cuda").to(dtype)
        return x, teacher.forward(x)[0]

    def everyone(t):
        return t.expand(members, -1, -1).contiguous()
    held_x, held_u = (everyone(t) for t in batch(rows))
    pool_x, pool_u = batch(4 * rows)                       # a small pool of noisy targets: what dropout is for
    pool_u = pool_u + noise * torch.randn(pool_u.shape, generator=gen, device="cuda").to(dtype)
    first = pop.evaluate(held_x, held_u)
    for step in range(steps):
        at = step % 4 * rows
        pop.step(everyone(pool_x[:, at:at + rows]), everyone(pool_u[:, at:at + rows]))
        if (step + 1) % ready_every == 0:
            pop.exploit_explore(-pop.evaluate(held_x, held_u))
    return pop, first, pop.evaluate(held_x, held_u)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("members", 10), ("rows", 128), ("width", 256), ("hidden", 512), ("steps", 60)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=["bfloat16", "float32"], default="bfloat16")
    args = ap.parse_args(argv)
    pop, first, last = train(args.members, args.rows, args.width, args.hidden, args.steps, dtype=getattr(torch, args.dtype))
    pop.unit.check()
    best = int(last.argmin())
    print(json.dumps({"members": args.members, "steps": args.steps, "first_loss": round(first.min().item(), 5), "best_loss": round(last.min().item(), 5),
                      "best_member": best, "best_lr": round(pop.lr[best].item(), 4), "best_rate_hidden": round(pop.rate_hidden[best].item(), 3),
                      "best_rate_out": round(pop.rate_out[best].item(), 3)}))


if __name__ == "__main__":
    main()
