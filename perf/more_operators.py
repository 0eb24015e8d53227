"""Measured cases of the gated unit and of dropout.

A population that trains residual feed-forward blocks takes, per block and step, a gated unit with a weight of every
member's own, whose hidden units are dropped at the member's rate, and drops the block's output before it is added to
the residual stream.  Each case is one pass through one of the two operators:

  gated      h = keep / (1 - p) * act(x Wg^T) * (x Wu^T), and the gradients of x and W = [Wg; Wu]
  dropout    y = residual + keep / (1 - p) * x, and the gradient of x

keep comes from a counter-based generator (Philox4x32-10), 16 bits an element, one block of it for eight neighbouring
columns: counter (member, the member's step, 5 + site, row * ceil(width / 8) + column // 8), key = seed.  An element
is dropped where its bits are below t = round(65536 rate); 1 - p = (65536 - t) / 65536.

With `own` false the passes are elementary torch operations in 32 bits, rounded once at the end; with `own` true they
are the calls a user makes of this package.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
ACTIVATIONS = ["silu", "gelu", "relu", "sigmoid"]


def listed():
    return [
        # --- gated unit ----------------------------------------------------------------------------------------------
        # one token of one member when serving: latency
        dict(name="gated one token", op="gated", dtype="bf16", mode="forward", members=1, rows=1, width=1024, hidden=2048,
             activation="silu", drop=False),
        # a full batch of single tokens of one member: the weight is read once
        dict(name="gated one token x 32", op="gated", dtype="bf16", mode="forward", members=1, rows=32, width=2048, hidden=4096,
             activation="silu", drop=False),
        # a few tokens for each of 16 members of their own weights, 1024 wide as in the classifiers
        dict(name="gated 16 members x 5 tokens", op="gated", dtype="bf16", mode="forward", members=16, rows=5, width=1024,
             hidden=1024, activation="gelu", drop=False),
        # evaluation of three classifiers on a ragged number of rows, 784 inputs
        dict(name="gated forward 3 x 777", op="gated", dtype="bf16", mode="forward", members=3, rows=777, width=784,
             hidden=1000, activation="gelu", drop=False),
        # a training step of the large population's shape: 80 members, 512 rows each, 2048 wide
        dict(name="gated train 80 x 512", op="gated", dtype="bf16", mode="train", members=80, rows=512, width=2048,
             hidden=2048, activation="silu", drop=True),
        # odd sizes: no row is a multiple of 16 bytes
        dict(name="gated train odd 5 x 301", op="gated", dtype="bf16", mode="train", members=5, rows=301, width=1001,
             hidden=515, activation="relu", drop=True),
        # the fp32 population: 16 members with 128 rows each, 256 -> 512
        dict(name="gated train fp32 16 x 128", op="gated", dtype="fp32", mode="train", members=16, rows=128, width=256,
             hidden=512, activation="silu", drop=True),
        # --- dropout ---------------------------------------------------------------------------------------------------
        # one short batch of one member: latency
        dict(name="dropout 1 x 32 x 1024", op="dropout", dtype="bf16", mode="forward", members=1, rows=32, width=1024, residual=True),
        # the large population's activations, dropped and added to the residual stream
        dict(name="dropout 80 x 512 x 2048", op="dropout", dtype="bf16", mode="forward", members=80, rows=512, width=2048, residual=True),
        # and the way back
        dict(name="dropout backward 80 x 512 x 2048", op="dropout", dtype="bf16", mode="backward", members=80, rows=512, width=2048,
             residual=False),
        # 24 members with 1024 rows of 512, fp32
        dict(name="dropout fp32 24 x 1024 x 512", op="dropout", dtype="fp32", mode="forward", members=24, rows=1024, width=512,
             residual=True),
        # odd rows
        dict(name="dropout odd 7 x 333 x 1001", op="dropout", dtype="bf16", mode="forward", members=7, rows=333, width=1001, residual=True),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    if rng.random() < 0.65:
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        mode = rng.choice(["forward", "train"])
        widest = 2048 if dtype == "bf16" else 512         # the fp32 population's layers are at most 512 wide
        width, hidden = (_spread(rng, 64, widest) for _ in range(2))
        if rng.random() < 0.75:                           # most layers are a multiple of eight wide, some are not
            width, hidden = (8 * ((n + 7) // 8) for n in (width, hidden))
        members = _spread(rng, 1, 80)
        rows = _spread(rng, 1, 512 if dtype == "bf16" else 128)
        return dict(op="gated", dtype=dtype, mode=mode, members=members, rows=rows, width=width, hidden=hidden,
                    activation=rng.choice(ACTIVATIONS), drop=mode == "train" and rng.random() < 0.75)
    mode = rng.choice(["forward", "backward"])
    return dict(op="dropout", dtype=rng.choice(["bf16", "fp32"]), mode=mode, members=_spread(rng, 1, 80), rows=_spread(rng, 1, 512),
                width=_spread(rng, 64, 2048), residual=mode == "forward" and rng.random() < 0.75)


# --- what a user's program has in hand --------------------------------------------------------------------------------


def _normal(gen, *shape, dtype=torch.float32, scale=1.0):
    out = torch.empty(shape, device="cuda", dtype=dtype)
    return out.normal_(0.0, scale, generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    m, rows, width = case["members"], case["rows"], case["width"]
    # rates of every member, its own step count, and which dropout of the network it is
    s = dict(case=case, seed=(0x9E3779B97F4A7C15 * (seed + 1)) & 0xFFFFFFFFFFFFFFFF, site=seed % 3,
             rate=torch.empty(m, device="cuda").uniform_(0.02, 0.5, generator=gen),
             step=torch.randint(0, 100_000, (m,), device="cuda", generator=gen))
    if case["op"] == "gated":
        s["x"] = _normal(gen, m, rows, width, dtype=dt)
        s["weight"] = _normal(gen, m, 2 * case["hidden"], width, dtype=dt, scale=width ** -0.5)
        if case["mode"] == "train":
            s["dh"] = _normal(gen, m, rows, case["hidden"], dtype=dt, scale=1e-2)
    elif case["mode"] == "forward":
        s["x"] = _normal(gen, m, rows, width, dtype=dt)
        s["residual"] = _normal(gen, m, rows, width, dtype=dt) if case["residual"] else None
    else:
        s["dy"] = _normal(gen, m, rows, width, dtype=dt, scale=1e-2)
    if own:
        from paper_1711_09846_b200 import Dropout, GatedUnit
        s["dropout"] = Dropout(s["rate"], s["seed"], s["step"], site=s["site"])
        if case["op"] == "gated":
            s["layer"] = GatedUnit(s["weight"], case["activation"])
            if not case["drop"]:
                s["dropout"] = None
    return s


# --- one pass ----------------------------------------------------------------------------------------------------------


def run(state):
    if state["case"]["op"] == "gated":
        return (_gated_own if own else _gated_plain)(state)
    return (_dropout_own if own else _dropout_plain)(state)


def _gated_own(s):
    layer, drop = s["layer"], s["dropout"]
    if s["case"]["mode"] == "forward":
        return {"h": layer.forward(s["x"], dropout=drop)}
    h, kept = layer.forward(s["x"], dropout=drop, keep=True)
    dx, d_weight = layer.backward(s["dh"], s["x"], kept, dropout=drop)
    return {"h": h, "dx": dx, "dweight": d_weight}


def _dropout_own(s):
    from paper_1711_09846_b200 import dropout_backward, dropout_forward
    if s["case"]["mode"] == "forward":
        return {"y": dropout_forward(s["x"], s["dropout"], residual=s["residual"])}
    return {"dx": dropout_backward(s["dy"], s["dropout"])}


def _high_low(a, b):
    """High and low 32 bits of the product of two 32-bit numbers in int64 (its wrapped bits are the product's)."""
    p = a * b
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _kept_scale(s, rows, width):
    """keep / (1 - p) of every element, float32 [members, rows, width]."""
    groups = (width + 7) // 8
    c0 = torch.arange(s["case"]["members"], device="cuda").view(-1, 1)
    c1, c2 = s["step"].view(-1, 1), torch.full_like(c0, 5 + s["site"])
    c3 = torch.arange(rows * groups, device="cuda").view(1, -1)
    k0, k1 = s["seed"] & 0xFFFFFFFF, s["seed"] >> 32
    for _ in range(10):
        h0, l0 = _high_low(c0, 0xD2511F53)
        h1, l1 = _high_low(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], -1)                             # two elements a word, the lower bits first
    bits = torch.stack([words & 0xFFFF, words >> 16], -1).view(-1, rows, 8 * groups)[..., :width]
    limit = (s["rate"] * 65536).round()
    return (bits >= limit.view(-1, 1, 1)) * (65536 / (65536 - limit)).view(-1, 1, 1)


def _activation(kind, g):
    """act(g) and its derivative."""
    if kind == "relu":
        return g.clamp_min(0), (g > 0).float()
    if kind == "gelu":
        cdf = 0.5 * torch.erfc(g * -math.sqrt(0.5))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    opened, closed = torch.sigmoid(g), torch.sigmoid(-g)
    if kind == "sigmoid":
        return opened, opened * closed
    return g * opened, opened * (1 + g * closed)


def _gated_plain(s):
    case, dt = s["case"], DTYPES[s["case"]["dtype"]]
    x, w = s["x"].float(), s["weight"].float()
    g, u = (x @ w.transpose(1, 2)).chunk(2, -1)
    a, slope = _activation(case["activation"], g)
    scale = _kept_scale(s, case["rows"], case["hidden"]) if case["drop"] else 1.0
    h = (a * u * scale).to(dt)
    if case["mode"] == "forward":
        return {"h": h}
    dh = s["dh"].float() * scale
    dz = torch.cat([dh * u * slope, dh * a], -1)
    return {"h": h, "dx": (dz @ w).to(dt), "dweight": (dz.transpose(1, 2) @ x).to(dt)}


def _dropout_plain(s):
    dt = DTYPES[s["case"]["dtype"]]
    scale = _kept_scale(s, s["case"]["rows"], s["case"]["width"])
    if s["case"]["mode"] == "backward":
        return {"dx": (s["dy"].float() * scale).to(dt)}
    y = s["x"].float() * scale
    return {"y": (y if s["residual"] is None else y + s["residual"].float()).to(dt)}


# --- what a pass cannot do without ---------------------------------------------------------------------------------------


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    m, t, width = case["members"], case["members"] * case["rows"], case["width"]
    if case["op"] == "dropout":
        cells = t * width
        return {"bytes": size * cells * (3 if case["residual"] else 2), "flops": 3 * cells}
    hidden = case["hidden"]
    weights = m * 2 * hidden * width
    if case["mode"] == "forward":
        return {"bytes": size * (t * width + weights + t * hidden), "flops": 4 * t * width * hidden}
    # a step reads x, dh and the weights and writes h, dx and the weights' gradients
    return {"bytes": size * (2 * t * width + 2 * weights + 2 * t * hidden), "flops": 12 * t * width * hidden}


# --- the definitions in 64 bits --------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        scale = _scale_exact(s, case["rows"], case["width"])
        if case["mode"] == "backward":
            out = {"dx": s["dy"].double() * scale}
        else:
            out = {"y": s["x"].double() * scale + (0 if s["residual"] is None else s["residual"].double())}
    else:
        out = _gated_exact(s)
    torch.cuda.synchronize()
    return out


def _times(constant, v):
    """The 64-bit product of a 32-bit constant and 32-bit numbers, as its high and low half, from 16-bit pieces."""
    a1, a0, b1, b0 = constant >> 16, constant & 0xFFFF, v >> 16, v & 0xFFFF
    middle = a1 * b0 + (a0 * b0 >> 16)
    other = a0 * b1 + (middle & 0xFFFF)
    return a1 * b1 + (middle >> 16) + (other >> 16), (other & 0xFFFF) << 16 | (a0 * b0 & 0xFFFF)


def _scale_exact(s, rows, width):
    per_row = -(-width // 8)
    out = torch.zeros((s["case"]["members"], rows, per_row * 8), dtype=torch.float64, device="cuda")
    limits = [round(r * 65536) for r in s["rate"].double().tolist()]
    for m, (limit, step) in enumerate(zip(limits, s["step"].tolist())):
        block = torch.arange(rows * per_row, device="cuda").view(rows, per_row)
        x = [torch.full_like(block, m), torch.full_like(block, step), torch.full_like(block, 5 + s["site"]), block]
        for r in range(10):
            key = [(s["seed"] + r * 0x9E3779B9) % 2 ** 32, ((s["seed"] >> 32) + r * 0xBB67AE85) % 2 ** 32]
            (top0, low0), (top2, low2) = _times(0xD2511F53, x[0]), _times(0xCD9E8D57, x[2])
            x = [top2 ^ x[1] ^ key[0], low2, top0 ^ x[3] ^ key[1], low0]
        for j in range(8):
            draw16 = x[j // 2] >> 16 if j % 2 else x[j // 2] % 65536
            out[m, :, j::8] = torch.where(draw16 < limit, 0.0, 65536 / (65536 - limit) if limit < 65536 else 0.0)
    return out[:, :, :width]


def _gated_exact(s):
    case, n = s["case"], s["case"]["hidden"]
    scale = _scale_exact(s, case["rows"], n) if case["drop"] else None
    act = {"silu": lambda g: g / (1 + torch.exp(-g)), "sigmoid": lambda g: 1 / (1 + torch.exp(-g)),
           "gelu": lambda g: g * (1 + torch.erf(g / 2 ** 0.5)) / 2, "relu": lambda g: torch.where(g > 0, g, 0.0)}[case["activation"]]
    train = case["mode"] == "train"
    out = []
    for m in range(case["members"]):                  # a member at a time, the definition differentiated by torch
        x, w = (s[key][m].double().requires_grad_(train) for key in ("x", "weight"))
        h = act(x @ w[:n].T) * (x @ w[n:].T)
        if scale is not None:
            h = h * scale[m]
        out.append((h.detach(), *(torch.autograd.grad(h, (x, w), s["dh"][m].double()) if train else ())))
    return dict(zip(("h", "dx", "dweight"), (torch.stack(part) for part in zip(*out))))
