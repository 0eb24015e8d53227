"""Measured cases of the adapter, block-norm and gradient-clipping operators.

A population that fine-tunes low-rank adapters on one shared projection takes, per residual block and step, a norm
before the block, the projection with every member's (or request's) own adapter, a norm after the block with its gate
and residual scale, their gradients, and the clipping of each member's gradient to its own global norm.  Each case is
one pass through one of the three operators:

  adapters   y_i = x_i W^T + b + c_a (x_i A_a^T) B_a^T for the rows i of each request, a the request's adapter
  norm       n = rms(block) w_post,  y = x + c sigmoid(gate) n,  u = rms(y) w_next,  per member
  clip       g <- g min(1, limit / ||g||) over all tensors of a member, ||g|| returned

With `own` false the passes are elementary torch operations in 32 bits, rounded once at the end; with `own` true they
are the calls a user makes of this package.
"""
import random

import torch

own = False

EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # --- adapters ---------------------------------------------------------------------------------------------
        # eight requests generate one token each through a layer of the 784-1024-1024-10 classifiers: latency
        dict(name="adapters one token x 8", op="adapters", dtype="bf16", mode="forward", layout="single", segments=8,
             rows=8, inputs=1024, outputs=1024, rank=8, adapters=6, pick=1),
        # a full serving batch of single tokens on a 2048-wide layer, a few of them without an adapter
        dict(name="adapters one token x 64", op="adapters", dtype="bf16", mode="forward", layout="single", segments=64,
             rows=64, inputs=2048, outputs=2048, rank=16, adapters=24, pick=2),
        # prompts of unequal length, adapters shared between requests, the ragged 784-wide input of the classifiers
        dict(name="adapters ragged prompts", op="adapters", dtype="bf16", mode="forward", layout="ragged", segments=23,
             rows=3001, inputs=784, outputs=1024, rank=8, adapters=9, pick=3),
        # one training step of 80 members with 512 rows each on a 2048 x 2048 layer: the large population's shape
        dict(name="adapters train 80 x 512", op="adapters", dtype="bf16", mode="train", layout="equal", segments=80,
             rows=40960, inputs=2048, outputs=2048, rank=16, adapters=80, pick=4),
        # the fp32 population: 16 members with 128 rows each on its 256 x 512 layer
        dict(name="adapters train fp32 16 x 128", op="adapters", dtype="fp32", mode="train", layout="equal", segments=16,
             rows=2048, inputs=256, outputs=512, rank=4, adapters=16, pick=5),
        # --- norms with gate and residual scale ---------------------------------------------------------------------
        # the smallest useful call: one short batch of one member, as when serving
        dict(name="norm forward 1 x 32 x 1024", op="norm", dtype="bf16", mode="forward", gate="vector", members=1,
             rows=32, width=1024),
        # the large population's activations, a gate per element
        dict(name="norm forward 80 x 512 x 2048", op="norm", dtype="bf16", mode="forward", gate="full", members=80,
             rows=512, width=2048),
        dict(name="norm backward 80 x 512 x 2048", op="norm", dtype="bf16", mode="backward", gate="full", members=80,
             rows=512, width=2048),
        # odd sizes in fp32, one gate vector per member whose gradient sums over the member's rows
        dict(name="norm backward fp32 6 x 333 x 1001", op="norm", dtype="fp32", mode="backward", gate="vector",
             members=6, rows=333, width=1001),
        # --- gradient clipping ----------------------------------------------------------------------------------------
        # 16 regressors 256-512-512-1, six tensors each, a threshold per member
        dict(name="clip 16 regressors", op="clip", dtype="fp32", shapes="256-512-512-1", members=16),
        # odd bf16 tensors packed end to end, so that most of them start off any vector boundary, in two groups
        dict(name="clip 60 odd bf16 tensors", op="clip", dtype="bf16", shapes="odd", members=2, tensors=60, pick=6),
        # all gradients of the large population: 80 members of 14,687,232 parameters
        dict(name="clip 80 large members", op="clip", dtype="fp32", shapes="2048-2048-2048-2048-1024", members=80),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["adapters", "adapters", "norm", "clip"])
    if op == "adapters":
        layout = rng.choice(["single", "ragged", "equal"])
        # the fp32 population's layers are at most 512 wide and its batches a few thousand rows
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        mode = "forward" if layout == "single" else rng.choice(["forward", "train"])
        widest = 2048 if dtype == "bf16" else 512
        inputs, outputs = (_spread(rng, 64, widest) for _ in range(2))
        if rng.random() < 0.75:                       # most layers are a multiple of eight wide, some are not
            inputs, outputs = (8 * ((n + 7) // 8) for n in (inputs, outputs))
        segments = _spread(rng, 1, 80)
        if layout == "single":
            rows = segments
        elif layout == "equal":
            rows = segments * _spread(rng, 2, 512 if dtype == "bf16" else 128)
        else:
            rows = segments * _spread(rng, 2, 256 if dtype == "bf16" else 64) + rng.randrange(7)
        return dict(op=op, dtype=dtype, mode=mode, layout=layout, segments=segments, rows=rows, inputs=inputs,
                    outputs=outputs, rank=rng.choice([4, 8, 16, 32, 64]), adapters=rng.randint(1, 80),
                    pick=rng.randrange(1 << 20))
    if op == "norm":
        return dict(op=op, dtype=rng.choice(["bf16", "fp32"]), mode=rng.choice(["forward", "backward"]),
                    gate=rng.choice(["none", "vector", "full"]), members=_spread(rng, 1, 80), rows=_spread(rng, 1, 256),
                    width=_spread(rng, 64, 4096))
    if rng.random() < 0.5:
        widths = [str(_spread(rng, 2, 2048)) for _ in range(rng.randint(3, 5))]
        return dict(op=op, dtype=rng.choice(["bf16", "fp32"]), shapes="-".join(widths), members=_spread(rng, 1, 60))
    return dict(op=op, dtype=rng.choice(["bf16", "fp32"]), shapes="odd", members=rng.randint(1, 8),
                tensors=_spread(rng, 8, 60), pick=rng.randrange(1 << 20))


# --- what a user's program has in hand --------------------------------------------------------------------------------


def _segments(case):
    """[(first row, end row, adapter)] of the requests; adapter -1: none.  Zero-length requests occur when ragged."""
    rng = random.Random(case["pick"])
    n, rows, adapters = case["segments"], case["rows"], case["adapters"]
    if case["layout"] == "ragged":
        cuts = sorted(rng.randrange(rows + 1) for _ in range(n - 1))
    else:
        cuts = [rows // n * k for k in range(1, n)]
    at = [0] + cuts + [rows]
    if case["layout"] == "equal" and adapters >= n:
        ids = list(range(n))                                    # a population: every member has its own
    else:
        ids = [rng.randrange(adapters) if rng.random() < 0.9 else -1 for _ in range(n)]
    return list(zip(at[:-1], at[1:], ids))


def _sizes(case):
    """Elements of the gradient tensors of one member, or of all tensors when they are odd ones."""
    if case["shapes"] == "odd":
        rng = random.Random(case["pick"])
        return [_spread(rng, 1, 400_000) for _ in range(case["tensors"])]
    w = [int(n) for n in case["shapes"].split("-")]
    return [n for a, b in zip(w, w[1:]) for n in (a * b, b)]


def _normal(gen, *shape, dtype=torch.float32, scale=1.0):
    out = torch.empty(shape, device="cuda", dtype=dtype)
    return out.normal_(0.0, scale, generator=gen)


def _uniform(gen, lo, hi, *shape):
    return torch.empty(shape, device="cuda").uniform_(lo, hi, generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"adapters": _prepare_adapters, "norm": _prepare_norm, "clip": _prepare_clip}[case["op"]](case, gen)


def _prepare_adapters(case, gen):
    dt, segs = DTYPES[case["dtype"]], _segments(case)
    t, k, n, r, a = (case[key] for key in ("rows", "inputs", "outputs", "rank", "adapters"))
    s = dict(case=case, segments=segs,
             row_offsets=torch.tensor([b for b, _, _ in segs] + [t], dtype=torch.int32, device="cuda"),
             adapter_ids=torch.tensor([i for _, _, i in segs], dtype=torch.int32, device="cuda"),
             x=_normal(gen, t, k, dtype=dt), weight=_normal(gen, n, k, dtype=dt, scale=k ** -0.5),
             bias=_normal(gen, n, scale=0.1), A=_normal(gen, a, r, k, dtype=dt, scale=k ** -0.5),
             B=_normal(gen, a, n, r, dtype=dt, scale=0.5 * r ** -0.5), scale=_uniform(gen, 0.5, 2.0, a))
    if case["mode"] == "train":
        s["dy"] = _normal(gen, t, n, dtype=dt, scale=1e-2)
    if own:
        from paper_1711_09846_b200 import AdapterProjection
        s["layer"] = AdapterProjection(s["weight"], s["A"], s["B"], s["scale"], bias=s["bias"])
    return s


def _prepare_norm(case, gen):
    dt = DTYPES[case["dtype"]]
    m, rows, d = case["members"], case["rows"], case["width"]
    s = dict(case=case, x=_normal(gen, m, rows, d, dtype=dt), block=_normal(gen, m, rows, d, dtype=dt, scale=0.7),
             post_weight=_uniform(gen, 0.5, 1.5, m, d), next_weight=_uniform(gen, 0.5, 1.5, m, d),
             scale=_uniform(gen, 0.2, 1.0, m), gate=None)
    if case["gate"] != "none":
        s["gate"] = _normal(gen, *((m, rows, d) if case["gate"] == "full" else (m, d)), dtype=dt)
    if case["mode"] == "backward":   # y and the two reciprocal roots are what the forward pass left
        s["dy"], s["du"] = (_normal(gen, m, rows, d, dtype=dt, scale=1e-2) for _ in range(2))
        s["y"] = s.pop("x")
        s["rstd_block"], s["rstd_next"] = ((s[key].float().square().mean(-1) + EPS).rsqrt() for key in ("block", "y"))
    return s


def _prepare_clip(case, gen):
    dt, m, sizes = DTYPES[case["dtype"]], case["members"], _sizes(case)
    if case["shapes"] == "odd":
        groups = [k % m for k in range(len(sizes))]
        flat = _normal(gen, sum(sizes), dtype=dt, scale=1e-2)
        grads = list(flat.split(sizes))
    else:
        groups = [k for k in range(m) for _ in sizes]
        flat = _normal(gen, m, sum(sizes), dtype=dt, scale=1e-2)
        grads = [g for row in flat for g in row.split(sizes)]
    count = [sum(g.numel() for g, k in zip(grads, groups) if k == j) for j in range(m)]
    # thresholds on both sides of the norms, so that some members are clipped and some are not
    limit = 1e-2 * torch.tensor(count, device="cuda", dtype=torch.float32).sqrt() * _uniform(gen, 0.3, 1.5, m)
    s = dict(case=case, flat=flat, grads=grads, groups=groups, limit=limit)
    if own:
        from paper_1711_09846_b200 import GradientClip
        s["out"] = torch.zeros_like(flat)
        out = list(s["out"].split(sizes)) if flat.dim() == 1 else [g for row in s["out"] for g in row.split(sizes)]
        s["clip"] = GradientClip(grads, groups, out=out)
    return s


# --- one pass ----------------------------------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    if case["op"] == "adapters":
        return (_adapters_own if own else _adapters_plain)(state)
    if case["op"] == "norm":
        return (_norm_own if own else _norm_plain)(state)
    return (_clip_own if own else _clip_plain)(state)


def _adapters_own(s):
    layer, where = s["layer"], (s["row_offsets"], s["adapter_ids"])
    if s["case"]["mode"] == "forward":
        return {"y": layer.forward(s["x"], *where)}
    y, kept = layer.forward(s["x"], *where, keep=True)
    dx, d_a, d_b = layer.backward(s["dy"], s["x"], kept, *where)
    return {"y": y, "dx": dx, "dA": d_a, "dB": d_b}


def _per_segment(s, x, w):
    """Rows of x times the transposed matrix w[a] of their request's adapter, zero for the requests without one."""
    segs = s["segments"]
    if s["case"]["layout"] != "ragged":               # equal requests: one batched product
        ids = s["adapter_ids"].long()
        per = x.view(len(segs), -1, x.shape[1]) @ w[ids.clamp_min(0)].transpose(1, 2)
        return (per * (ids >= 0).view(-1, 1, 1)).view(x.shape[0], -1)
    return torch.cat([x[a:b] @ w[i].T if i >= 0 else x.new_zeros(b - a, w.shape[1]) for a, b, i in segs])


def _adapter_gradient(s, left, right):
    """sum of left_i^T right_i over the rows i of each adapter."""
    segs, n = s["segments"], s["case"]["adapters"]
    out = left.new_zeros(n + 1, left.shape[1], right.shape[1])      # the last one collects the requests without adapter
    if s["case"]["layout"] != "ragged":
        per = left.view(len(segs), -1, left.shape[1]).transpose(1, 2) @ right.view(len(segs), -1, right.shape[1])
    else:
        per = torch.stack([left[a:b].T @ right[a:b] for a, b, _ in segs])
    return out.index_add_(0, s["adapter_ids"].long() % (n + 1), per)[:n]


def _adapters_plain(s):
    case, dt = s["case"], DTYPES[s["case"]["dtype"]]
    x, w, a, b = (s[key].float() for key in ("x", "weight", "A", "B"))
    scaled = b * s["scale"].view(-1, 1, 1)
    kept = _per_segment(s, x, a)
    y = (x @ w.T + s["bias"] + _per_segment(s, kept, scaled)).to(dt)
    if case["mode"] == "forward":
        return {"y": y}
    dy = s["dy"].float()
    ds = _per_segment(s, dy, scaled.transpose(1, 2))
    dx = (dy @ w + _per_segment(s, ds, a.transpose(1, 2))).to(dt)
    return {"y": y, "dx": dx, "dA": _adapter_gradient(s, ds, x),
            "dB": _adapter_gradient(s, dy, kept) * s["scale"].view(-1, 1, 1)}


def _norm_own(s):
    from paper_1711_09846_b200 import block_norm_backward, block_norm_forward
    shared = dict(post_weight=s["post_weight"], gate=s["gate"], scale=s["scale"], next_weight=s["next_weight"])
    if s["case"]["mode"] == "forward":
        out = block_norm_forward(s["x"], s["block"], eps=EPS, **shared)
        return {"y": out.y, "u": out.u}
    g = block_norm_backward(s["dy"], s["du"], s["y"], s["block"], rstd_block=s["rstd_block"], rstd_next=s["rstd_next"],
                            **shared)
    return {"dx": g.dx, "dblock": g.dblock, "dgate": g.dgate, "dpost": g.dpost_weight, "dnext": g.dnext_weight,
            "dscale": g.dscale}


def _opened(s):
    """sigmoid of the gate, broadcast over rows when there is one per member; 1 without a gate."""
    if s["gate"] is None:
        return 1.0
    g = torch.sigmoid(s["gate"].float())
    return g if g.dim() == 3 else g[:, None]


def _norm_plain(s):
    dt = DTYPES[s["case"]["dtype"]]
    c, w_post, w_next = s["scale"].view(-1, 1, 1), s["post_weight"][:, None], s["next_weight"][:, None]
    block, g = s["block"].float(), _opened(s)
    if s["case"]["mode"] == "forward":
        normed = block * (block.square().mean(-1, keepdim=True) + EPS).rsqrt() * w_post
        y = s["x"].float() + c * g * normed
        u = y * (y.square().mean(-1, keepdim=True) + EPS).rsqrt() * w_next
        return {"y": y.to(dt), "u": u.to(dt)}
    dy, du, y = (s[key].float() for key in ("dy", "du", "y"))
    r_block, r_next = s["rstd_block"][..., None], s["rstd_next"][..., None]
    y_hat, b_hat = y * r_next, block * r_block
    d_hat = du * w_next
    dx = dy + r_next * (d_hat - y_hat * (d_hat * y_hat).mean(-1, keepdim=True))
    dn = c * g * dx
    e_hat = dn * w_post
    dblock = r_block * (e_hat - b_hat * (e_hat * b_hat).mean(-1, keepdim=True))
    opened = dx * b_hat * w_post * g
    dgate = None
    if s["gate"] is not None:
        dgate = c * opened * (1.0 - g)
        dgate = (dgate if s["gate"].dim() == 3 else dgate.sum(1)).to(dt)
    return {"dx": dx.to(dt), "dblock": dblock.to(dt), "dgate": dgate, "dpost": (dn * b_hat).sum(1),
            "dnext": (du * y_hat).sum(1), "dscale": opened.sum((1, 2))}


def _clip_own(s):
    return {"norms": s["clip"].run(s["limit"]), "clipped": s["out"]}


def _clip_plain(s):
    dt = DTYPES[s["case"]["dtype"]]
    if s["flat"].dim() == 2:                          # the members' gradients are the rows of one slab
        g = s["flat"].float()
        norms = g.square().sum(1).sqrt()
        return {"norms": norms, "clipped": (g * (s["limit"] / norms).clamp_max(1.0)[:, None]).to(dt)}
    grads = [g.float() for g in s["grads"]]
    squares = torch.stack([g.square().sum() for g in grads])
    groups = torch.tensor(s["groups"], device="cuda")
    norms = squares.new_zeros(s["case"]["members"]).index_add_(0, groups, squares).sqrt()
    coef = (s["limit"] / norms).clamp_max(1.0)[groups].unbind()
    return {"norms": norms, "clipped": torch.cat([g * c for g, c in zip(grads, coef)]).to(dt)}


# --- what a pass cannot do without ---------------------------------------------------------------------------------------


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "adapters":
        t, k, n, r = (case[key] for key in ("rows", "inputs", "outputs", "rank"))
        segs = _segments(case)
        used = len({i for a, b, i in segs if i >= 0 and b > a})
        low = sum(b - a for a, b, i in segs if i >= 0) * r * (k + n)
        once = size * (t * k + k * n + used * r * (k + n) + t * n) + 4 * n
        if case["mode"] == "forward":
            return {"bytes": once, "flops": 2 * (t * k * n + low)}
        # a step reads x, dy and the weights and writes y, dx and the two gradients of every adapter
        return {"bytes": once + size * t * (n + k) + 4 * case["adapters"] * r * (k + n),
                "flops": 2 * (2 * t * k * n + 3 * low)}
    if case["op"] == "norm":
        cells, row = case["members"] * case["rows"] * case["width"], case["members"] * case["width"]
        gate = {"none": 0, "vector": row, "full": cells}[case["gate"]]
        if case["mode"] == "forward":
            return {"bytes": size * (4 * cells + gate) + 8 * row, "flops": 15 * cells}
        return {"bytes": size * (6 * cells + 2 * gate) + 16 * row, "flops": 35 * cells}
    total = sum(_sizes(case)) * (1 if case["shapes"] == "odd" else case["members"])
    return {"bytes": 2 * size * total, "flops": 3 * total}


# --- the definitions in 64 bits --------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    out = {"adapters": _adapters_exact, "norm": _norm_exact, "clip": _clip_exact}[case["op"]](s)
    torch.cuda.synchronize()
    return out


def _adapters_exact(s):
    x, w, a, b, c = (s[key].double() for key in ("x", "weight", "A", "B", "scale"))
    y = torch.einsum("tk,nk->tn", x, w) + s["bias"].double()
    train = s["case"]["mode"] == "train"
    if train:
        dy = s["dy"].double()
        dx, d_a, d_b = torch.einsum("tn,nk->tk", dy, w), torch.zeros_like(a), torch.zeros_like(b)
    for lo, hi, i in s["segments"]:
        if i < 0 or hi == lo:
            continue
        merged = c[i] * b[i] @ a[i]                    # the adapter as one matrix [outputs, inputs]
        y[lo:hi] += torch.einsum("tk,nk->tn", x[lo:hi], merged)
        if train:
            dx[lo:hi] += torch.einsum("tn,nk->tk", dy[lo:hi], merged)
            d_merged = torch.einsum("tn,tk->nk", dy[lo:hi], x[lo:hi])
            d_a[i] += c[i] * torch.einsum("nr,nk->rk", b[i], d_merged)
            d_b[i] += c[i] * torch.einsum("nk,rk->nr", d_merged, a[i])
    return {"y": y, "dx": dx, "dA": d_a, "dB": d_b} if train else {"y": y}


def _norm_exact(s):
    case = s["case"]
    out = []
    for m in range(case["members"]):                  # a member at a time, its two maps differentiated by hand
        f = {key: s[key][m].double() for key in ("block", "post_weight", "next_weight", "scale")}
        z = None if s["gate"] is None else s["gate"][m].double()
        g = torch.ones((), device="cuda", dtype=torch.float64) if z is None else 1 / (1 + torch.exp(-z))
        d = case["width"]
        if case["mode"] == "forward":
            v = f["block"] / torch.sqrt((f["block"] ** 2).sum(1, keepdim=True) / d + EPS)
            y = s["x"][m].double() + f["scale"] * g * f["post_weight"] * v
            out.append((y, f["next_weight"] * y / torch.sqrt((y ** 2).sum(1, keepdim=True) / d + EPS)))
            continue
        y, dy, du = (s[key][m].double() for key in ("y", "dy", "du"))
        ry, rb = s["rstd_next"][m].double()[:, None], s["rstd_block"][m].double()[:, None]
        h = f["next_weight"] * du
        dx = dy + ry * h - y * ry ** 3 * (h * y).sum(1, keepdim=True) / d
        k = f["scale"] * g * f["post_weight"] * dx
        dblock = rb * k - f["block"] * rb ** 3 * (k * f["block"]).sum(1, keepdim=True) / d
        base = dx * f["block"] * rb
        dz = None
        if z is not None:
            dz = f["scale"] * f["post_weight"] * base * g * (1 - g)
            dz = dz if z.dim() == 2 else dz.sum(0)
        out.append((dx, dblock, dz, (f["scale"] * g * base).sum(0), (du * y * ry).sum(0),
                    (g * f["post_weight"] * base).sum()))
    names = ("y", "u") if case["mode"] == "forward" else ("dx", "dblock", "dgate", "dpost", "dnext", "dscale")
    return {name: None if out[0][k] is None else torch.stack([o[k] for o in out]) for k, name in enumerate(names)}


def _clip_exact(s):
    total = torch.zeros(s["case"]["members"], dtype=torch.float64, device="cuda")
    for g, k in zip(s["grads"], s["groups"]):
        total[k] += (g.double() ** 2).sum()
    norms, limit = total.sqrt(), s["limit"].double()
    done = torch.empty_like(s["flat"], dtype=torch.float64)
    rest = done.view(-1)
    for g, k in zip(s["grads"], s["groups"]):
        n = g.numel()
        rest[:n] = g.double() * torch.where(norms[k] > limit[k], limit[k] / norms[k], torch.ones_like(norms[k]))
        rest = rest[n:]
    return {"norms": norms, "clipped": done}
