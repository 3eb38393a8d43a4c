"""Fine-tuning of many tenants' low-rank adapters beside one frozen projection, with orthogonalised updates of their factors, then
serving: the same adapters, a token of every request at a time.  And the same update of a layer's experts, whose replica slots get the
new weights.  Synthetic data, on one GPU.

Every tenant has a target projection W + S_a with S_a of low rank, and learns it from its own tokens.  A step is one forward and backward
of the batch (all tenants at once) and one update of either stack of factors, [n, rank, d_in] and [n, rank, d_out]: momentum, Newton-Schulz
steps, weight decay on fp32 weights, and the rounded copies that the next forward reads, written in place.

    python -m paper_2407_04656_amd.adapter_finetune
"""
from __future__ import annotations

import argparse
import math

from . import binding as lz
from .finetune import AdapterProjection, AdapterShape, OrthogonalShape, OrthogonalUpdate


def train(T=4096, d_in=1024, d_out=1024, rank=16, n=8, steps=60, lr=0.2, dtype=lz.LZ_BF16, seed=0, dev="cuda:0"):
    """Returns the mean squared error before and after, per token and column, and the serving check's largest difference."""
    import torch
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = torch.float32 if dtype == lz.LZ_F32 else torch.bfloat16

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=dev) * std).to(dt)

    w = normal(d_in, d_out, std=0.02)
    low = rank // 2 if rank > 1 else 1  # of the targets
    left, right = normal(n, d_in, low, std=d_in ** -0.5), normal(n, low, d_out, std=0.3)
    scale = torch.ones(n, device=dev)
    # factors: fp32 weights and the rounded copies in use; the second starts at zero
    a, b = normal(n, rank, d_in, std=d_in ** -0.5), torch.zeros((n, rank, d_out), dtype=dt, device=dev)
    factors = []
    for weights in (a, b):
        rows, cols = weights.shape[1:]
        update = OrthogonalUpdate(OrthogonalShape(n, rows, cols, dtype), dev)
        factors.append((update, torch.zeros(weights.shape, device=dev), weights.float(), weights))
    own = torch.arange(n, dtype=torch.int32, device=dev)  # a factor's copy is its own

    layer = AdapterProjection(AdapterShape(T, d_in, d_out, rank, n, dtype), dev)
    layer.set_weights(w, a, b, scale)
    layer.enable_training()
    # sixteen requests of a tenant each, a few without an adapter
    ids = (torch.arange(T, device=dev) * 16 // T % (n + 1)).to(torch.int32) - 1
    layer.plan(ids)

    def batch():
        x = normal(T, d_in)
        target = x.float() @ w.float()
        for i in range(n):
            mine = torch.nonzero(ids == i)[:, 0]
            target[mine] += (x[mine].float() @ left[i].float()) @ right[i].float()
        return x, target

    errors = []
    for step in range(steps):
        x, target = batch()
        off = layer.forward(x).float() - target
        errors.append((off * off).mean())
        layer.backward((off / T).to(dt))
        rate = lr * (1 - step / steps)
        for (update, momentum, master, weights), grad in zip(factors, (layer.da, layer.db)):
            rows, cols = weights.shape[1:]
            update.step(grad, momentum, master, own, lr=rate, scale=math.sqrt(max(1.0, cols / rows)) / 4, momentum_out=momentum,
                        master_out=master, slot_weights=weights)
    x, target = batch()
    after = (layer.forward(x).float() - target).square().mean()

    # serving: one token of every request, whatever adapter it has, against the same rows of the batch
    some = torch.arange(0, T, max(1, T // 64), device=dev)[:64]
    served = AdapterProjection(AdapterShape(len(some), d_in, d_out, rank, n, dtype), dev)
    served.set_weights(w, a, b, scale)
    served.plan(ids[some].contiguous())
    differ = (served.forward(x[some].contiguous()).float() - layer.y[some].float()).abs().max()
    return {"before": float(errors[0]), "after": float(after), "served_differ": float(differ), "largest": float(layer.y.abs().max())}


def update_experts(E=8, slots=12, d=256, ffn=384, dtype=lz.LZ_BF16, seed=1, dev="cuda:0"):
    """One orthogonalised step of the experts' second matrices from the replicas' gradients: sums over the replicas, the update, the new
    weights in every slot.  Returns the slots' weights and the experts' (fp32)."""
    import torch
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = torch.float32 if dtype == lz.LZ_F32 else torch.bfloat16
    slot_expert = torch.arange(slots, dtype=torch.int32, device=dev) % E
    dw2_slot = (torch.randn((slots, ffn, d), generator=gen, device=dev) * 1e-3).to(dt)
    dw2 = torch.empty((E, ffn, d), dtype=dt, device=dev)
    lz.lz_reduce_replica_grads_dtype(dw2_slot, slot_expert, slots, E, ffn * d, dtype, dw2)
    master = torch.randn((E, ffn, d), generator=gen, device=dev) * 0.02
    update = OrthogonalUpdate(OrthogonalShape(E, ffn, d, dtype), dev)
    _, master, w2 = update.step(dw2, torch.zeros_like(master), master, slot_expert, lr=2e-3, weight_decay=0.1,
                                scale=math.sqrt(max(1.0, ffn / d)))
    return w2, master, slot_expert


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--steps", type=int, default=60)
    args = p.parse_args()
    r = train(steps=args.steps)
    print(f"adapters: mean squared error {r['before']:.4f} -> {r['after']:.4f}; served tokens differ by {r['served_differ']:.2e} "
          f"of {r['largest']:.2f}")
    w2, master, slot_expert = update_experts()
    print(f"experts: {w2.shape[0]} slots hold the new weights of {master.shape[0]} experts")


if __name__ == "__main__":
    main()
