"""Orthogonalised updates against the steps in 64 bits.  How far a result may be off is counted by an emulation that rounds to the
documented 16-bit parts at every stored factor and is exact otherwise: its own distance from the steps in 64 bits, twice, plus half
a rounding step of the result and the fp32 sums."""
import math

import numpy as np
import pytest
import torch

import paper_2407_04656_amd as lz

DEV = "cuda:0"
pytestmark = pytest.mark.gpu

F32, BF16 = lz.LZ_F32, lz.LZ_BF16
NS5 = lz.NEWTON_SCHULZ_5
CUBIC = ((1.5, -0.5, 0.0),) * 4
EPS = 1e-7


def exact(u, coef, eps=EPS):
    m = u.double()
    tall = m.shape[1] > m.shape[2]
    m = m.transpose(1, 2) if tall else m
    m = m / (m.square().sum((1, 2), keepdim=True).sqrt() + eps)
    for a, b, c in coef:
        s = m @ m.transpose(1, 2)
        m = a * m + (b * s + c * (s @ s)) @ m
    return m.transpose(1, 2) if tall else m


def parts(v, planes):
    """What `planes` fp16 numbers at 2^14 times the size hold of v."""
    hi = (v * 16384).half().double()
    lo = (v * 16384 - hi).half().double() if planes == 2 else 0.0
    return (hi + lo) / 16384


def emulated(u, coef, planes, eps=EPS):
    m = u.double()
    tall = m.shape[1] > m.shape[2]
    m = m.transpose(1, 2) if tall else m
    m = parts(m / (m.square().sum((1, 2), keepdim=True).sqrt() + eps), planes)
    for a, b, c in coef:
        g = parts(m @ m.transpose(1, 2), planes)
        m = parts(a * m + parts(b * g + c * (g @ g), planes) @ m, planes)
    return m.transpose(1, 2) if tall else m


def matrices(n, rows, cols, dtype, seed, kind="noise"):
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn((n, rows, cols), generator=gen)
    if kind == "few":  # a few directions and little else
        k = min(4, rows, cols)
        g = 0.02 * g + torch.randn((n, rows, k), generator=gen) @ torch.randn((n, k, cols), generator=gen)
    return (1e-3 * g).to(torch.float32 if dtype == F32 else torch.bfloat16)


def distance(got, want):
    """Of every matrix, 2-norm of the difference over that of the result."""
    got, want = got.detach().double().cpu(), want
    assert torch.isfinite(got).all()
    return ((got - want).square().sum((1, 2)) / want.square().sum((1, 2))).sqrt()


def allowed(u, coef, planes, dtype):
    e = exact(u, coef)
    # fp32 sums of K terms in 15 products, each off by at most K / 32 roundings in a row; a result's rounding is half a step
    sums = 15 * max(u.shape[1:]) / 32 * 2.0 ** -24
    rounding = 2.0 ** -24 if dtype == F32 else 2.0 ** -8
    return e, 2 * distance(emulated(u, coef, planes), e) + sums * 4 + rounding


# n, rows, cols
SIZES = [(1, 1, 1), (3, 1, 7), (2, 5, 1), (4, 8, 64), (2, 64, 8), (1, 63, 65), (2, 65, 63), (3, 100, 130), (2, 130, 100), (1, 128, 1000),
         (2, 16, 4096), (1, 4096, 16), (8, 128, 256), (2, 200, 777), (1, 777, 333), (1, 320, 320), (70, 33, 40), (1, 520, 1300),
         (64, 100, 1100), (1, 200, 3000), (2, 1700, 448)]


@pytest.mark.parametrize("kind", ["noise", "few"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize(size, dtype, kind):
    print(f"orthogonalize: {size} dtype={dtype} {kind}", flush=True)
    g = matrices(*size, dtype, 3, kind)
    e, bound = allowed(g, NS5, 2 if dtype == F32 else 1, dtype)
    u = lz.OrthogonalUpdate(lz.OrthogonalShape(*size, dtype), DEV, eps=EPS)
    d = distance(u.orthogonalize(g.to(DEV)), e)
    assert (d <= bound).all(), (d / bound).max()


# as many tiles as the wide kernel takes, whole ones and of 64, 128 and 192 rows; several bands of them
# and a few tiles more than the chip has places
WIDE = [(90, 300, 330), (70, 290, 500), (40, 300, 500), (36, 330, 440), (34, 380, 400), (7, 1090, 1150), (11, 1300, 770)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", WIDE, ids=lambda s: "x".join(map(str, s)))
def test_many_tiles(size, dtype):
    test_orthogonalize(size, dtype, "noise")


# thin ones of so many columns that their workgroups are more than sixteen
LONG = [(1, 24, 9001), (1, 20001, 20), (3, 64, 5000), (1, 100, 6007), (40, 16, 3000)]


@pytest.mark.parametrize("kind", ["noise", "few"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", LONG, ids=lambda s: "x".join(map(str, s)))
def test_long_thin_matrices(size, dtype, kind):
    test_orthogonalize(size, dtype, kind)


@pytest.mark.parametrize("coef", [CUBIC, ((2.0, -1.5, 0.5),) * 3, ((1.0, 0.0, 0.0),), ((0.0, 0.0, 1.0),), ((1.0, -2.0, 0.25),),
                                  ((3.4445, -4.7750, 2.0315),) * 3 + ((1.875, -1.25, 0.375),) * 2], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_other_coefficients(coef, dtype):
    size = (2, 96, 300)
    g = matrices(*size, dtype, 4)
    e, bound = allowed(g, coef, 2 if dtype == F32 else 1, dtype)
    u = lz.OrthogonalUpdate(lz.OrthogonalShape(*size, dtype), DEV, coef=coef, eps=EPS)
    d = distance(u.orthogonalize(g.to(DEV)), e)
    assert (d <= bound).all(), (d / bound).max()


@pytest.mark.parametrize("factor", [1e-30, 1e-12, 1e12, 1e30])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_size_of_the_input_does_not_matter(factor, dtype):
    size = (2, 72, 90)
    g = (matrices(*size, dtype, 6).double() * factor).to(torch.float32 if dtype == F32 else torch.bfloat16)
    e = exact(g, NS5, 0.0)
    u = lz.OrthogonalUpdate(lz.OrthogonalShape(*size, dtype), DEV, eps=0.0)
    _, bound = allowed((g.double() / factor).to(g.dtype), NS5, 2 if dtype == F32 else 1, dtype)
    assert (distance(u.orthogonalize(g.to(DEV)), e) <= 1.1 * bound).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_zeros_and_what_is_not_finite_stay_in_their_matrix(dtype):
    g = matrices(4, 40, 70, dtype, 7)
    g[0] = 0
    g[2, 3, 5] = float("nan")
    g[3, 1, 1] = float("inf")
    out = lz.OrthogonalUpdate(lz.OrthogonalShape(4, 40, 70, dtype), DEV).orthogonalize(g.to(DEV)).cpu()
    e, bound = allowed(g[1:2], NS5, 2 if dtype == F32 else 1, dtype)
    assert not out[0].any()
    assert (distance(out[1:2], e) <= bound).all()
    assert torch.isnan(out[2]).all() and torch.isnan(out[3]).any()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 100, 70), (2, 16, 300), (1, 7, 5), (2, 200, 330)], ids=lambda s: "x".join(map(str, s)))
def test_in_place_and_unaligned(size, dtype):
    g = matrices(*size, dtype, 8).to(DEV)
    u = lz.OrthogonalUpdate(lz.OrthogonalShape(*size, dtype), DEV)
    want = u.orthogonalize(g).clone()
    room = torch.empty(g.numel() + 1, dtype=g.dtype, device=DEV)
    view = room[1:].view(g.shape)
    view.copy_(g)
    assert u.orthogonalize(view, out=view) is view
    assert torch.equal(view, want)


@pytest.mark.parametrize("size,dtype", [((32, 1344, 256), BF16), ((50, 256, 192), BF16), ((61, 1024, 256), F32), ((8, 768, 1664), F32),
                                        ((40, 24, 600), F32), ((9, 100, 900), BF16)])
def test_same_bits_every_time(size, dtype):
    gen = torch.Generator(device=DEV).manual_seed(2)
    g = torch.randn(size, generator=gen, device=DEV).to(torch.float32 if dtype == F32 else torch.bfloat16)
    u = lz.OrthogonalUpdate(lz.OrthogonalShape(*size, dtype), DEV)
    want = u.orthogonalize(g).clone()
    differ = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(300):
        differ += (u.orthogonalize(g) != want).sum()
    assert int(differ.item()) == 0


STEPS = [((3, 100, 70), 5), ((2, 16, 300), 2), ((4, 64, 64), 9), ((1, 9, 1), 0), ((5, 130, 260), 70), ((2, 300, 130), 3)]


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size,slots", STEPS, ids=lambda v: str(v).replace(" ", ""))
def test_step(size, slots, dtype, nesterov):
    print(f"step: {size} slots={slots} dtype={dtype} nesterov={nesterov}", flush=True)
    n, rows, cols = size
    gen = torch.Generator().manual_seed(5)
    g = matrices(*size, dtype, 9)
    momentum, master = torch.randn(size, generator=gen) * 3e-3, torch.randn(size, generator=gen) * 0.02
    expert = torch.randint(0, n, (slots,), generator=gen, dtype=torch.int32)
    if slots > 2:
        expert[0], expert[2] = n, -1  # nobody's: left as they are
    mu, lr, decay = 0.95, 2e-2, 0.1
    scale = math.sqrt(max(1.0, rows / cols))
    u = lz.OrthogonalUpdate(lz.OrthogonalShape(*size, dtype), DEV, eps=EPS)
    dev = [t.to(DEV) for t in (g, momentum, master, expert)]
    copies = torch.full((slots, rows, cols), 7.0, dtype=g.dtype, device=DEV)
    kw = dict(mu=mu, lr=lr, weight_decay=decay, scale=scale, nesterov=nesterov)
    m1, w1, s1 = u.step(*dev, slot_weights=copies, **kw) if slots else u.step(*dev[:3], **kw)
    f = 2.0 ** -24
    m64 = mu * momentum.double() + g.double()
    # mu is an fp32 number (half a step), and the sum is rounded (twice if not fused)
    assert ((m1.double().cpu() - m64).abs() <= 3 * f * (m64.abs() + mu * momentum.double().abs())).all()
    m = m1.double().cpu()
    v = g.double() + mu * m if nesterov else m
    e, bound = allowed(v, NS5, 2, F32)
    w64 = (1 - lr * decay) * master.double() - lr * scale * e
    off = (w1.double().cpu() - w64).square().sum((1, 2)).sqrt()
    most = lr * scale * bound * e.square().sum((1, 2)).sqrt() + 4 * f * (master.double().square().sum((1, 2)).sqrt() + w64.square().sum((1, 2)).sqrt())
    assert (off <= most).all(), (off / most).max()
    if not slots:
        assert s1 is None
    for s in range(slots):
        want = w1[int(expert[s])].to(g.dtype) if 0 <= int(expert[s]) < n else torch.full_like(copies[s], 7.0)
        assert torch.equal(s1[s], want), s
    # in place
    args = (dev[0], dev[1], dev[2]) + ((dev[3],) if slots else ())
    more = dict(slot_weights=copies) if slots else {}
    m2, w2, _ = u.step(*args, momentum_out=dev[1], master_out=dev[2], **more, **kw)
    assert m2 is dev[1] and torch.equal(m2, m1) and torch.equal(w2, w1)


@pytest.mark.parametrize("size,dtype", [((2, 100, 300), BF16), ((1, 320, 200), F32), ((8, 16, 512), BF16)])
def test_captured_step(size, dtype):
    g = matrices(*size, dtype, 10).to(DEV)
    momentum, master = torch.zeros(size, device=DEV), torch.ones(size, device=DEV)
    expert = torch.arange(size[0], dtype=torch.int32, device=DEV)
    u = lz.OrthogonalUpdate(lz.OrthogonalShape(*size, dtype), DEV)
    eager = [t.clone() for t in u.step(g, momentum, master, expert)]
    update = u.orthogonalize(g).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        u.step(g, momentum, master, expert)
        u.orthogonalize(g)
    for _ in range(3):
        for t in (u.momentum, u.master, u.slot_weights, u.out):
            t.zero_()
        u.orthogonalize(momentum if dtype == F32 else momentum.bfloat16())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*eager, update), (u.momentum, u.master, u.slot_weights, u.out)):
            assert torch.equal(a, b)


def test_on_another_stream():
    g = matrices(2, 140, 300, BF16, 12).to(DEV)
    u = lz.OrthogonalUpdate(lz.OrthogonalShape(2, 140, 300, BF16), DEV)
    want = u.orthogonalize(g).clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = u.orthogonalize(g)
    stream.synchronize()
    assert torch.equal(got, want)
