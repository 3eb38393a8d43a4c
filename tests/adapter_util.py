"""Low-rank adapters beside a projection in 64 bits, and how far a result may be off: half a rounding step per stored tensor,
and fp32 sums of K terms off by K half steps of fp32, both counted on the magnitudes that are summed."""
import numpy as np
import torch

import paper_2407_04656_amd as lz

DEV = "cuda:0"


def tokens(rng, T, n, requests, bare):
    """Adapters of contiguous requests (requests = T: of every token), some of them -1."""
    cuts = np.sort(rng.choice(np.arange(1, T), requests - 1, replace=False)) if requests > 1 else np.zeros(0, np.int64)
    lengths = np.diff(np.concatenate([[0], cuts, [T]]))
    ids = rng.integers(0, n, requests)
    ids[rng.random(requests) < bare] = -1
    return np.repeat(ids, lengths).astype(np.int32)


def inputs(T, d_in, d_out, rank, n, dtype, ids, seed=0):
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == lz.LZ_F32 else torch.bfloat16

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen) * std).to(dt)

    return {"ids": torch.from_numpy(np.asarray(ids, dtype=np.int32)), "x": normal(T, d_in), "w": normal(d_in, d_out, std=0.05),
            "a": normal(n, rank, d_in, std=d_in ** -0.5), "b": normal(n, rank, d_out, std=0.2),
            "scale": torch.rand(n, generator=gen) + 0.5, "dy": normal(T, d_out)}


def reference(s, dtype):
    """{name: (value, bound)} in 64 bits."""
    u = 2.0 ** -24 if dtype == lz.LZ_F32 else 2.0 ** -8
    f = 2.0 ** -24
    x, w, a, b, scale, dy = (s[k].double() for k in ("x", "w", "a", "b", "scale", "dy"))
    ids = s["ids"].long()
    T, d_in = x.shape
    d_out, rank, n = w.shape[1], a.shape[1], a.shape[0]
    h, eh = torch.zeros(T, rank, dtype=torch.float64), torch.zeros(T, rank, dtype=torch.float64)
    dh, edh = h.clone(), h.clone()
    y, ey = x @ w, d_in * f * (x.abs() @ w.abs())
    dx, edx = dy @ w.t(), d_out * f * (dy.abs() @ w.abs().t())
    da, eda, db, edb = (torch.zeros_like(t) for t in (a, a, b, b))
    for i in range(n):
        r = torch.nonzero(ids == i)[:, 0]
        if not r.numel():
            continue
        h[r] = scale[i] * (x[r] @ a[i].t())
        eh[r] = u * h[r].abs() + (d_in + 1) * f * scale[i] * (x[r].abs() @ a[i].abs().t())
        dh[r] = scale[i] * (dy[r] @ b[i].t())
        edh[r] = u * dh[r].abs() + (d_out + 1) * f * scale[i] * (dy[r].abs() @ b[i].abs().t())
        y[r] += h[r] @ b[i]
        ey[r] += eh[r] @ b[i].abs() + (rank + 1) * f * (h[r].abs() @ b[i].abs())
        dx[r] += dh[r] @ a[i]
        edx[r] += edh[r] @ a[i].abs() + (rank + 1) * f * (dh[r].abs() @ a[i].abs())
        m = r.numel()
        da[i] = dh[r].t() @ x[r]
        eda[i] = edh[r].t() @ x[r].abs() + m * f * (dh[r].abs().t() @ x[r].abs())
        db[i] = h[r].t() @ dy[r]
        edb[i] = eh[r].t() @ dy[r].abs() + m * f * (h[r].abs().t() @ dy[r].abs())
    out = {"y": (y, ey), "dx": (dx, edx), "da": (da, eda), "db": (db, edb)}
    # rounded once when stored; 1.01: the product terms of the above
    return {k: (v, 1.01 * (e + u * v.abs()) + 1e-30) for k, (v, e) in out.items()}


def check(name, got, value, bound):
    got = got.detach().double().cpu()
    assert torch.isfinite(got).all(), name
    over = ((got - value).abs() / bound).max().item() if got.numel() else 0.0
    assert over <= 1.0, f"{name}: {over:.3g} of the bound"


def projection(s, T, d_in, d_out, rank, n, dtype, training=True):
    p = lz.AdapterProjection(lz.AdapterShape(T, d_in, d_out, rank, n, dtype), DEV)
    p.set_weights(*(s[k].to(DEV) for k in ("w", "a", "b", "scale")))
    if training:
        p.enable_training()
    return p
