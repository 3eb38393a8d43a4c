"""Operators of fine-tuning that are measured: low-rank adapters of many requests beside a shared projection, and the
orthogonalised update of stacks of matrices (experts, adapter factors).

A case names an operation and its sizes.  Operations:

  adapt        y = x W + scale[a] (x A_a^T) B_a for the adapter a = ids[t] of every token t (none: x W alone); one forward,
               a prompt's tokens or one token of every request
  adapt_train  the same forward and its backward: dx, dA, dB for a given dy (W is frozen)
  orthogonal   Newton-Schulz steps X <- (a I + b G + c G^2) X, G = X X^T, from X = g / (|g| + eps), for n matrices
  update       momentum, orthogonalised update and weight decay of E experts' fp32 weights, and the rounded copies that the
               experts' replica slots train with

Layouts are the framework's: W [d_in, d_out], A [n, rank, d_in], B [n, rank, d_out], all row-major; weights of a slot
[rows, cols].  Sizes are those of this repository's configurations (widths 128, 2048, 4096; experts 128 x 256, 2048 x 1408,
4096 x 14336) or generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
WEIGHT_STD = 0.02
COEF = (3.4445, -4.7750, 2.0315)  # the quintic that takes singular values of (0, 1] near 1 in five steps
EPS = 1e-7
MU, LR, DECAY = 0.95, 2e-3, 0.1


def _adapter(name, op, dtype, T, d_in, d_out, rank, n, requests, bare=0.0):
    """requests: how many contiguous requests the batch holds (T: every token is one of its own); bare: share without adapter."""
    out = dict(op=op, dtype=dtype, T=T, d_in=d_in, d_out=d_out, rank=rank, n=n, requests=requests, bare=bare)
    return dict(out, name=name) if name else out


def _matrices(name, op, dtype, n, rows, cols, slots=0):
    out = dict(op=op, dtype=dtype, n=n, rows=rows, cols=cols, slots=slots)
    return dict(out, name=name) if name else out


def listed():
    return [
        # the smallest call: one request's next token through one projection
        _adapter("adapt_token", "adapt", "bf16", 1, 4096, 4096, 16, 8, 1),
        # a decoding batch: every token has its own request, 64 adapters are resident, some requests use none
        _adapter("adapt_decode", "adapt", "bf16", 64, 4096, 4096, 16, 64, 64, 0.1),
        # prompts of sixteen requests through one projection
        _adapter("adapt_prompts", "adapt", "bf16", 8192, 4096, 4096, 16, 16, 16),
        # full precision at sizes that no power of two divides: a ragged batch of nine requests
        _adapter("adapt_odd_f32", "adapt", "f32", 1021, 500, 1301, 12, 9, 9, 0.2),
        # training the adapters of four tenants at once beside a wide projection
        _adapter("adapt_train_wide", "adapt_train", "bf16", 8192, 2048, 8192, 32, 4, 8),
        # ... of thirty-two, with a larger rank and short sequences
        _adapter("adapt_train_many", "adapt_train", "bf16", 16384, 2048, 2048, 64, 32, 128, 0.05),
        # gradient checks and ablations: the fp32 test layer's width
        _adapter("adapt_train_f32", "adapt_train", "f32", 256, 128, 256, 8, 3, 6),
        # gradients of a stack of adapter factors
        _matrices("orthogonal_factors", "orthogonal", "bf16", 32, 16, 4096),
        # the fp32 test layer's first matrices
        _matrices("orthogonal_f32", "orthogonal", "f32", 8, 128, 256),
        # two of the large experts' matrices (the most arithmetic)
        _matrices("orthogonal_large", "orthogonal", "bf16", 2, 4096, 14336),
        # an optimizer step of fine-grained experts: 64 second matrices, replicated over 128 slots
        _matrices("update_finegrained", "update", "bf16", 64, 1408, 2048, 128),
        # full precision, sizes that no power of two divides, taller than wide
        _matrices("update_odd_f32", "update", "f32", 5, 777, 333, 7),
    ]


def _log_int(rng, lo, hi, step=1):
    """An integer multiple of `step` in [lo, hi], uniform over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def draw(rng):
    """A case of the same ranges: every operation, both types, sizes over their logarithm."""
    while True:
        op = rng.choices(["adapt", "adapt_train", "orthogonal", "update"], [4, 3, 3, 2])[0]
        dtype = "bf16" if rng.random() < 0.8 else "f32"
        if op in ("adapt", "adapt_train"):
            # widths: mostly multiples of 64, sometimes only of 8 (fp32: of anything)
            step = rng.choices([64, 8], [7, 3])[0] if dtype == "bf16" else rng.choices([64, 8, 1], [4, 3, 3])[0]
            hi = 8192 if dtype == "bf16" else 2048
            d_in, d_out = _log_int(rng, 128, hi, step), _log_int(rng, 128, hi, step)
            T = _log_int(rng, 1 if op == "adapt" else 64, 16384)
            rank = rng.choice([8, 16, 32, 64, 128]) if dtype == "bf16" else rng.randint(1, 64)
            n = _log_int(rng, 1, 128)
            requests = T if T <= 256 and rng.random() < 0.6 else min(T, _log_int(rng, 1, 256))
            case = _adapter(None, op, dtype, T, d_in, d_out, rank, n, requests, round(rng.choice([0.0, 0.0, rng.uniform(0, 0.5)]), 2))
            if n * rank > 4096:
                continue
        else:
            rows, cols = _log_int(rng, 8, 4096), _log_int(rng, 64, 8192)
            if rng.random() < 0.7:
                rows, cols = max(8, rows // 64 * 64 if rows >= 64 else rows // 8 * 8), max(64, cols // 64 * 64)
            if rng.random() < 0.4:
                rows, cols = cols, rows
            n = _log_int(rng, 1, 64)
            if n * rows * cols > 2e8:
                continue
            case = _matrices(None, op, dtype, n, rows, cols, n + rng.randint(0, n) if op == "update" else 0)
        if work(case)["flops"] <= (5e12 if dtype == "bf16" else 4e11):
            return case


def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("adapt", "adapt_train"):
        T, d_in, d_out, rank = (case[k] for k in ("T", "d_in", "d_out", "rank"))
        with_adapter = T * (1 - case["bare"])
        used = min(case["n"], case["requests"])  # adapters that can have tokens
        tensors = T * (d_in + d_out) + d_in * d_out + used * rank * (d_in + d_out)
        base, low = 2 * T * d_in * d_out, 2 * with_adapter * rank * (d_in + d_out)
        if case["op"] == "adapt":
            return {"bytes": b * tensors + 4 * T, "flops": base + low}
        grads = T * (d_in + d_out) + case["n"] * rank * (d_in + d_out)
        return {"bytes": b * (tensors + grads) + 4 * T, "flops": 2 * base + 3 * low}
    n, rows, cols = case["n"], case["rows"], case["cols"]
    small, large = min(rows, cols), max(rows, cols)
    # the Gram matrix and its square are symmetric: half of their products; then one full product a step
    flops = 5 * n * (3 * small * small * large + small * small * small)
    size = n * rows * cols
    if case["op"] == "orthogonal":
        return {"bytes": 2 * b * size, "flops": flops}
    return {"bytes": b * size + 16 * size + b * case["slots"] * rows * cols, "flops": flops}


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1_000_003 * int(seed) + 17)
    dt = _dtype(case)

    def normal(*shape, std=1.0, dtype=dt):
        out = torch.empty(shape, dtype=dtype, device=DEV)
        for part in out.split(max(1, 2 ** 26 // max(1, math.prod(shape[1:])))):  # no fp32 copy of the whole
            part.copy_(torch.randn(part.shape, generator=gen, device=DEV, dtype=torch.float32) * std)
        return out

    if case["op"] in ("adapt", "adapt_train"):
        T, d_in, d_out, rank, n = (case[k] for k in ("T", "d_in", "d_out", "rank", "n"))
        rng = np.random.default_rng([int(seed), 5])
        q = case["requests"]
        cuts = np.sort(rng.choice(np.arange(1, T), q - 1, replace=False)) if q > 1 else np.zeros(0, np.int64)
        lengths = np.diff(np.concatenate([[0], cuts, [T]]))
        adapter = rng.integers(0, n, q)
        adapter[rng.random(q) < case["bare"]] = -1
        ids = np.repeat(adapter, lengths).astype(np.int32)
        state = {
            "case": dict(case), "ids": torch.from_numpy(ids).to(DEV), "x": normal(T, d_in),
            "w": normal(d_in, d_out, std=WEIGHT_STD), "a": normal(n, rank, d_in, std=1 / math.sqrt(d_in)),
            "b": normal(n, rank, d_out, std=0.1),
            "scale": torch.rand(n, generator=gen, device=DEV) + 0.5,
        }
        if case["op"] == "adapt_train":
            state["dy"] = normal(T, d_out)
        return state

    n, rows, cols = case["n"], case["rows"], case["cols"]
    # gradients: a part of low rank, as batches of few directions leave it, and noise of every direction
    k = min(32, rows, cols)
    g = torch.empty((n, rows, cols), dtype=dt, device=DEV)
    for i in range(n):
        left, right = (torch.randn(s, generator=gen, device=DEV) for s in ((rows, k), (k, cols)))
        noise = torch.randn((rows, cols), generator=gen, device=DEV)
        g[i] = (1e-3 * (left @ right / math.sqrt(k) * 0.5 + noise)).to(dt)
    state = {"case": dict(case), "g": g}
    if case["op"] == "update":
        rng = np.random.default_rng([int(seed), 6])
        plan = np.concatenate([np.arange(n), rng.integers(0, n, case["slots"] - n)])  # every expert has a slot
        state["slot_expert"] = torch.from_numpy(rng.permutation(plan).astype(np.int32)).to(DEV)
        state["momentum"] = normal(n, rows, cols, std=3e-3, dtype=torch.float32)
        state["master"] = normal(n, rows, cols, std=WEIGHT_STD, dtype=torch.float32)
    return state


# ---------------------------------------------------------------- plain forms


def _plain_adapters(s):
    case, n = s["case"], s["case"]["n"]
    x, w, a, b = (s[k].float() for k in ("x", "w", "a", "b"))
    rank = a.shape[1]
    # all adapters' first factors side by side; a token keeps the columns of its own
    gate = (s["ids"][:, None] == torch.arange(n, device=x.device)[None]).float() * s["scale"][None]
    gate = gate[:, :, None].expand(-1, -1, rank).reshape(-1, n * rank)
    af, bf = a.reshape(n * rank, -1), b.reshape(n * rank, -1)
    h = (x @ af.t()) * gate
    y = (x @ w + h @ bf).to(s["x"].dtype)
    if case["op"] == "adapt":
        return y
    dy = s["dy"].float()
    dh = (dy @ bf.t()) * gate
    dx = dy @ w.t() + dh @ af
    dt = s["x"].dtype
    return {"y": y, "dx": dx.to(dt), "da": (dh.t() @ x).reshape(a.shape).to(dt), "db": (h.t() @ dy).reshape(b.shape).to(dt)}


def _plain_orthogonal(u):
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / (x.double().square().sum((1, 2), keepdim=True).sqrt() + EPS).float()
    a, b, c = COEF
    for _ in range(5):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _plain_update(s):
    g = s["g"].float()
    m = MU * s["momentum"] + g
    o = _plain_orthogonal(g + MU * m)
    scale = math.sqrt(max(1.0, g.shape[1] / g.shape[2]))
    master = (1 - LR * DECAY) * s["master"] - LR * scale * o
    return {"momentum": m, "master": master, "slots": master.to(s["g"].dtype)[s["slot_expert"].long()]}


# ---------------------------------------------------------------- the framework's calls


def _own_adapters(s):
    case = s["case"]
    layer = s.get("layer")
    if layer is None:  # the buffers of a projection, made once
        import paper_2407_04656_amd as lz
        shape = lz.AdapterShape(case["T"], case["d_in"], case["d_out"], case["rank"], case["n"],
                                lz.LZ_F32 if case["dtype"] == "f32" else lz.LZ_BF16)
        layer = s["layer"] = lz.AdapterProjection(shape, DEV)
        layer.set_weights(s["w"], s["a"], s["b"], s["scale"])
        if case["op"] == "adapt_train":
            layer.enable_training()
    layer.plan(s["ids"])
    y = layer.forward(s["x"])
    if case["op"] == "adapt":
        return y
    dx, da, db = layer.backward(s["dy"])
    return {"y": y, "dx": dx, "da": da, "db": db}


def _own_orthogonal(s):
    case = s["case"]
    update = s.get("update")
    if update is None:
        import paper_2407_04656_amd as lz
        shape = lz.OrthogonalShape(case["n"], case["rows"], case["cols"], lz.LZ_F32 if case["dtype"] == "f32" else lz.LZ_BF16)
        update = s["update"] = lz.OrthogonalUpdate(shape, DEV, coef=[COEF] * 5, eps=EPS)
    if case["op"] == "orthogonal":
        return update.orthogonalize(s["g"])
    scale = math.sqrt(max(1.0, case["rows"] / case["cols"]))
    m, master, slots = update.step(s["g"], s["momentum"], s["master"], s["slot_expert"], mu=MU, lr=LR, weight_decay=DECAY,
                                   scale=scale, nesterov=True)
    return {"momentum": m, "master": master, "slots": slots}


def run(state):
    adapters = state["case"]["op"] in ("adapt", "adapt_train")
    if own:
        return _own_adapters(state) if adapters else _own_orthogonal(state)
    if adapters:
        return _plain_adapters(state)
    if state["case"]["op"] == "orthogonal":
        return _plain_orthogonal(state["g"].float()).to(state["g"].dtype)
    return _plain_update(state)


# ---------------------------------------------------------------- the definitions in 64 bits


def _exact_adapters(s):
    case = s["case"]
    x, w, a, b, scale = (s[k].double() for k in ("x", "w", "a", "b", "scale"))
    y = x @ w
    train = case["op"] == "adapt_train"
    if train:
        dy = s["dy"].double()
        dx, da, db = dy @ w.t(), torch.zeros_like(a), torch.zeros_like(b)
    for i in range(case["n"]):
        rows = torch.nonzero(s["ids"] == i)[:, 0]
        if not rows.numel():
            continue
        xi = x[rows]
        y[rows] += scale[i] * ((xi @ a[i].t()) @ b[i])
        if train:
            dyi = dy[rows]
            dhi = scale[i] * (dyi @ b[i].t())
            dx[rows] += dhi @ a[i]
            da[i] = dhi.t() @ xi
            db[i] = scale[i] * (xi @ a[i].t()).t() @ dyi
    return {"y": y, "dx": dx, "da": da, "db": db} if train else y


def _exact_orthogonal(u):
    """Odd polynomials of the singular values by way of the small side's products alone: u -> Q u with Q a polynomial of u u^T."""
    out = torch.empty_like(u)
    for i in range(u.shape[0]):
        m = u[i] if u.shape[1] <= u.shape[2] else u[i].t()
        m = m / (torch.linalg.matrix_norm(m) + EPS)
        for a, b, c in [COEF] * 5:
            s = m @ m.t()
            inner = c * s
            inner.diagonal().add_(b)
            outer = s @ inner
            outer.diagonal().add_(a)
            m = outer @ m
        out[i] = m if u.shape[1] <= u.shape[2] else m.t()
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("adapt", "adapt_train"):
        return _exact_adapters(s)
    if case["op"] == "orthogonal":
        return _exact_orthogonal(s["g"].double())
    g, rows, cols = s["g"].double(), case["rows"], case["cols"]
    m = MU * s["momentum"].double() + g
    o = _exact_orthogonal(g + MU * m)
    master = s["master"].double() * (1 - LR * DECAY) - LR * math.sqrt(max(1.0, rows / cols)) * o
    return {"momentum": m, "master": master, "slots": master[s["slot_expert"].long()]}
