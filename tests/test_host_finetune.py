"""What the fine-tuning calls refuse, before any device is asked for."""
import numpy as np
import pytest
import torch

import paper_2407_04656_amd as lz
from paper_2407_04656_amd.binding import LZ_EINVAL, LZ_ESHAPE, LZ_EWORKSPACE

NS5 = lz.NEWTON_SCHULZ_5


def _code(call, *args, **kw):
    with pytest.raises(lz.LzError) as e:
        call(*args, **kw)
    return e.value.code


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(d_in=0), dict(d_out=0), dict(rank=0), dict(rank=1025), dict(n=0), dict(n=4097), dict(dtype=2), dict(T=1 << 30, d_in=1 << 20)])
def test_adapter_shapes(bad):
    shape = lz.AdapterShape(**{**dict(T=4, d_in=8, d_out=8, rank=8, n=2, dtype=lz.LZ_BF16), **bad})
    assert lz.lz_adapter_workspace_bytes(shape) == 0
    assert _code(lz.lz_adapter_plan, None, shape, None, None, 0, stream=0) == LZ_ESHAPE
    assert _code(lz.lz_adapter_forward, *[None] * 5, shape, None, None, None, 0, stream=0) == LZ_ESHAPE
    assert _code(lz.lz_adapter_backward, *[None] * 7, shape, None, None, None, None, 0, stream=0) == LZ_ESHAPE
    if shape.T <= 4:
        assert _code(lz.AdapterProjection, shape, "cpu") == LZ_ESHAPE


def test_adapter_workspace_and_pointers():
    shape = lz.AdapterShape(4, 8, 16, 8, 2, lz.LZ_BF16)
    size = lz.lz_adapter_workspace_bytes(shape)
    room = np.zeros(size + 512, np.uint8)
    at = -room.ctypes.data % 256
    ws = room[at:at + size]
    for given, n in ((None, size), (room[at + 1:at + 1 + size], size), (ws, size - 1)):
        assert _code(lz.lz_adapter_plan, None, shape, None, given, n, stream=0) == LZ_EWORKSPACE
        assert _code(lz.lz_adapter_forward, *[None] * 5, shape, None, None, given, n, stream=0) == LZ_EWORKSPACE
        assert _code(lz.lz_adapter_backward, *[None] * 7, shape, None, None, None, given, n, stream=0) == LZ_EWORKSPACE
    assert _code(lz.lz_adapter_plan, None, shape, None, ws, size, stream=0) == LZ_EINVAL
    some = np.zeros(1024, np.uint8)
    for missing in range(7):
        args = [None if i == missing else some for i in range(7)]
        assert _code(lz.lz_adapter_forward, *args[:5], shape, *args[5:], ws, size, stream=0) == LZ_EINVAL
    for missing in range(10):
        args = [None if i == missing else some for i in range(10)]
        assert _code(lz.lz_adapter_backward, *args[:7], shape, *args[7:], ws, size, stream=0) == LZ_EINVAL


def test_adapter_tensors():
    shape = lz.AdapterShape(4, 8, 16, 8, 2, lz.LZ_BF16)
    p = lz.AdapterProjection(shape, "cpu")
    bf = torch.bfloat16
    w, a, b, scale = torch.zeros(8, 16, dtype=bf), torch.zeros(2, 8, 8, dtype=bf), torch.zeros(2, 8, 16, dtype=bf), torch.ones(2)
    assert _code(p.forward, torch.zeros(4, 8, dtype=bf)) == LZ_EINVAL  # no weights, no plan
    assert _code(p.backward, torch.zeros(4, 16, dtype=bf)) == LZ_EINVAL
    assert _code(p.set_weights, w.float(), a, b, scale) == LZ_EINVAL
    assert _code(p.set_weights, w.t(), a, b, scale) == LZ_ESHAPE
    assert _code(p.set_weights, torch.zeros(16, 8, dtype=bf).t(), a, b, scale) == LZ_ESHAPE  # strided
    assert _code(p.set_weights, w, a[:1], b, scale) == LZ_ESHAPE
    assert _code(p.set_weights, w, a, b, scale.double()) == LZ_EINVAL
    assert _code(p.plan, torch.zeros(4, dtype=torch.int64)) == LZ_EINVAL
    assert _code(p.plan, torch.zeros(5, dtype=torch.int32)) == LZ_ESHAPE


@pytest.mark.parametrize("bad", [dict(n=0), dict(n=65536), dict(rows=0), dict(cols=-3), dict(dtype=3), dict(rows=1 << 15, cols=1 << 15),
                                 dict(rows=1, cols=1 << 29)])
def test_orthogonal_shapes(bad):
    shape = lz.OrthogonalShape(**{**dict(n=2, rows=8, cols=16, dtype=lz.LZ_F32), **bad})
    assert lz.lz_orthogonal_workspace_bytes(shape) == 0
    assert _code(lz.lz_orthogonalize, None, shape, NS5, 1e-7, None, None, 0, stream=0) == LZ_ESHAPE
    assert _code(lz.OrthogonalUpdate, shape, "cpu") == LZ_ESHAPE


@pytest.mark.parametrize("coef", [
    [(np.nan, 0, 0)], [(np.inf, 0, 0)], [(5.0, 0, 0)], [(3.4445, 4.775, 2.0315)], [(3.4445, -4.775, 2.0315)] * 17, [(2.0, -1.5, 4.0)] * 3])
def test_orthogonal_coefficients(coef):
    shape = lz.OrthogonalShape(1, 8, 16, lz.LZ_F32)
    size = lz.lz_orthogonal_workspace_bytes(shape)
    room = np.zeros(size + 512, np.uint8)
    ws = room[-room.ctypes.data % 256:][:size]
    some = np.zeros(1024, np.uint8)
    assert _code(lz.lz_orthogonalize, some, shape, coef, 1e-7, some, ws, size, stream=0) == LZ_EINVAL


def test_orthogonal_arguments():
    shape = lz.OrthogonalShape(2, 8, 16, lz.LZ_F32)
    size = lz.lz_orthogonal_workspace_bytes(shape)
    room = np.zeros(size + 512, np.uint8)
    at = -room.ctypes.data % 256
    ws = room[at:at + size]
    some = np.zeros(1024, np.uint8)
    for given, n in ((None, size), (room[at + 1:at + 1 + size], size), (ws, size - 1)):
        assert _code(lz.lz_orthogonalize, some, shape, NS5, 1e-7, some, given, n, stream=0) == LZ_EWORKSPACE
    for eps in (-1e-3, np.nan, np.inf):
        assert _code(lz.lz_orthogonalize, some, shape, NS5, eps, some, ws, size, stream=0) == LZ_EINVAL
    assert _code(lz.lz_orthogonalize, None, shape, NS5, 1e-7, some, ws, size, stream=0) == LZ_EINVAL
    assert _code(lz.lz_orthogonalize, some, shape, NS5, 1e-7, None, ws, size, stream=0) == LZ_EINVAL
    assert _code(lz.lz_orthogonalize, some, shape, [(1.0, 2.0)], 1e-7, some, ws, size, stream=0) == LZ_EINVAL
    options = dict(coef=NS5, eps=1e-7, mu=0.9, lr=1e-2, weight_decay=0.0, scale=1.0, nesterov=True, stream=0)
    expert = torch.zeros(3, dtype=torch.int32)
    for missing in range(6):
        args = [None if i == missing else some for i in range(6)]
        assert _code(lz.lz_orthogonal_step, *args[:3], expert, shape, *args[3:], ws, size, **options) == LZ_EINVAL
    u = lz.OrthogonalUpdate(shape, "cpu")
    f = torch.zeros(2, 8, 16)
    assert _code(u.orthogonalize, f.bfloat16()) == LZ_EINVAL
    assert _code(u.orthogonalize, f.transpose(1, 2)) == LZ_ESHAPE
    assert _code(u.orthogonalize, f[:1]) == LZ_ESHAPE
    assert _code(u.step, f, f.double(), f) == LZ_EINVAL
    assert _code(u.step, f, f, f, expert.long()) == LZ_EINVAL
    assert _code(u.step, f, f, f, None, slot_weights=f) == LZ_EINVAL
