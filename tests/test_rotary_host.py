"""What the rotation checks before it touches a device: status codes, workspace sizes, tensors of another device."""
import ctypes as C
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

from test_language_devices import BF16, F32, I64, Elsewhere, Library

PTR = 1 << 20        # an aligned address that no call here gets to use


@pytest.fixture(scope="module")
def omni():
    return B.Omni(1, 1, 1, 1)


def rotary(pairs=4, frequency=None, axis=None, **kw):
    a = dict(batch=2, length=5, heads=4, kv_heads=2, dim=64, pairs=pairs, axes=2, interleaved=0, dtype=B.BF16, weight_dtype=B.F32,
             position_type=B.I64, eps=1e-6, frequency=(C.c_double * 8)(*(frequency or [1.0] * 8)), axis=(C.c_int32 * 8)(*(axis or [0] * 8)),
             positions=PTR, position_axis=0, position_batch=5, position_row=1, q_weight=PTR, k_weight=PTR, lengths=None)
    a.update(kw)
    return B.omni_rotary(*a.values())


ROWS, KEYS = B.omni_attn_view(PTR, 5 * 256, 256, 64), B.omni_attn_view(PTR, 5 * 128, 128, 64)


def forward(ctx, r, change=None):
    v = [ROWS, KEYS, ROWS, KEYS]
    for i, view in (change or {}).items():
        v[i] = view
    return B.lib().omni_rotary_forward(ctx, None if r is None else C.byref(r), *(None if x is None else C.byref(x) for x in v), None)


def backward(ctx, r, change=None, dq_weight=PTR, dk_weight=PTR, dtype=B.F32, workspace=PTR, size=1 << 30):
    v = [ROWS, KEYS] * 3
    for i, view in (change or {}).items():
        v[i] = view
    return B.lib().omni_rotary_backward(ctx, None if r is None else C.byref(r), *(None if x is None else C.byref(x) for x in v), dq_weight,
                                        dk_weight, dtype, workspace, size, None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), B.ERR_BAD_CONFIG), (dict(length=-1), B.ERR_BAD_CONFIG), (dict(heads=0), B.ERR_BAD_CONFIG),
    (dict(kv_heads=0), B.ERR_BAD_CONFIG), (dict(dim=63), B.ERR_BAD_CONFIG), (dict(dim=0), B.ERR_BAD_CONFIG), (dict(dim=6), B.ERR_BAD_CONFIG),
    (dict(pairs=0), B.ERR_BAD_CONFIG), (dict(pairs=33), B.ERR_BAD_CONFIG), (dict(axes=0), B.ERR_BAD_CONFIG), (dict(axes=5), B.ERR_BAD_CONFIG),
    (dict(dtype=2), B.ERR_BAD_CONFIG), (dict(weight_dtype=-1), B.ERR_BAD_CONFIG), (dict(position_type=2), B.ERR_BAD_CONFIG),
    (dict(eps=-1e-9), B.ERR_BAD_CONFIG), (dict(eps=math.inf), B.ERR_BAD_CONFIG), (dict(eps=math.nan), B.ERR_BAD_CONFIG),
    (dict(frequency=[1.0, math.inf, 1, 1, 1, 1, 1, 1]), B.ERR_BAD_CONFIG), (dict(axis=[0, 2, 0, 0, 0, 0, 0, 0]), B.ERR_BAD_CONFIG),
    (dict(axis=[0, -1, 0, 0, 0, 0, 0, 0]), B.ERR_BAD_CONFIG), (dict(dim=258), B.ERR_TOO_LARGE), (dict(heads=65536), B.ERR_TOO_LARGE),
    (dict(batch=1 << 16, length=1 << 15), B.ERR_TOO_LARGE), (dict(q_weight=None), B.ERR_NULL), (dict(k_weight=None), B.ERR_NULL),
    (dict(positions=None), B.ERR_NULL), (dict(positions=PTR + 4), B.ERR_ALIGN), (dict(lengths=PTR + 2), B.ERR_ALIGN),
    (dict(q_weight=PTR + 2), B.ERR_ALIGN),
])
def test_refuses_sizes(omni, change, status):
    size = C.c_uint64()
    assert forward(omni._h, rotary(**change)) == status
    assert backward(omni._h, rotary(**change)) == status
    assert B.lib().omni_rotary_workspace(C.byref(rotary(**change)), C.byref(size)) == status


@pytest.mark.parametrize("view,status,results_only", [
    (None, B.ERR_NULL, False), (B.omni_attn_view(None, 1280, 256, 64), B.ERR_NULL, False),
    (B.omni_attn_view(PTR + 1, 1280, 256, 64), B.ERR_ALIGN, False), (B.omni_attn_view(PTR, 1 << 40, 256, 64), B.ERR_TOO_LARGE, False),
    (B.omni_attn_view(PTR, 1280, 256, 63), B.ERR_BAD_CONFIG, True), (B.omni_attn_view(PTR, 1280, 0, 64), B.ERR_BAD_CONFIG, True),
])
def test_refuses_operands(omni, view, status, results_only):
    for i in (2, 3) if results_only else range(4):
        assert forward(omni._h, rotary(), {i: view}) == status
    for i in (4, 5) if results_only else range(6):
        assert backward(omni._h, rotary(), {i: view}) == status
    assert forward(None, rotary()) == backward(None, rotary()) == forward(omni._h, None) == backward(omni._h, None) == B.ERR_NULL


def test_backward_workspace_and_weights(omni):
    size = C.c_uint64()
    assert B.lib().omni_rotary_workspace(C.byref(rotary()), None) == B.ERR_NULL
    assert B.lib().omni_rotary_workspace(C.byref(rotary(q_weight=None, k_weight=None)), C.byref(size)) == B.OK and size.value == 0
    assert B.lib().omni_rotary_workspace(C.byref(rotary()), C.byref(size)) == B.OK and size.value >= 2 * 64 * 4
    assert backward(omni._h, rotary(), size=size.value - 1) == B.ERR_TOO_LARGE
    assert backward(omni._h, rotary(), workspace=None) == backward(omni._h, rotary(), dq_weight=None) == B.ERR_NULL
    assert backward(omni._h, rotary(), dk_weight=None) == B.ERR_NULL and backward(omni._h, rotary(), dtype=2) == B.ERR_BAD_CONFIG
    assert backward(omni._h, rotary(), workspace=PTR + 8) == backward(omni._h, rotary(), dk_weight=PTR + 2) == B.ERR_ALIGN


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(L, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(L, "_like", lambda t: Elsewhere(t.shape, t.dtype))
    monkeypatch.setattr(Elsewhere, "stride", lambda t, i=None: t._like.stride() if i is None else t._like.stride(i))
    r = L.Rotary(B.Omni(1, 1, 1, 1), 2, 1, 8, [1.0])
    r._lib = Library()
    q, k, at, w = Elsewhere((1, 3, 2, 8), BF16), Elsewhere((1, 3, 1, 8), BF16), Elsewhere((1, 3), I64), Elsewhere((8,), F32)
    for call in (lambda: r.forward(q, k, at, w, w), lambda: r.backward(q, k, at, q, k, w, w)):
        monkeypatch.setattr(L, "_device", lambda: 0)
        with pytest.raises(ValueError, match="cuda:1"):
            call()
        monkeypatch.setattr(L, "_device", lambda: 1)
        with pytest.raises(AssertionError, match="omni_"):
            call()
    t = torch.zeros(1, 3, 2, 8)
    with pytest.raises(ValueError):
        r.forward(t, t[:, :, :1], torch.zeros(1, 3, dtype=torch.int64))
