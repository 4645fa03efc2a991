"""What the AdamW step checks before it touches a device: status codes, the record of the tensors, tensors of another device."""
import ctypes as C
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

PTR = 1 << 20        # an aligned address that no call here gets to use


@pytest.fixture(scope="module")
def omni():
    return B.Omni(1, 1, 1, 1)


def tensor(at=PTR, grads=(1 << 28, 1 << 28), **kw):
    d = dict(param=at, param_lp=at + (1 << 16), grads=(C.c_void_p * 2)(*grads) if grads else None, m=at + (2 << 16), v=at + (3 << 16),
             tops=at + (4 << 16), n=5000, weight_decay=0.1)
    d.update(kw)
    return B.omni_adamw_tensor(*d.values())


def plan(*tensors, K=2, dtype=B.BF16, bits=8, size=1 << 20):
    array = (B.omni_adamw_tensor * max(1, len(tensors)))(*tensors)
    need = C.c_uint64()
    rc = B.lib().omni_adamw_plan_bytes(array, len(tensors), K, dtype, bits, C.byref(need))
    record = C.create_string_buffer(size + 8)
    at = (C.addressof(record) + 7) // 8 * 8
    return rc, B.lib().omni_adamw_plan(array, len(tensors), K, dtype, bits, at, size if rc == B.OK else 1 << 20), record, at, need.value


def step(ctx, record, dev=PTR, b=(1, 2), lr=0.1, beta1=0.9, beta2=0.9, eps=1e-8, t=1, clock=None):
    return B.lib().omni_adamw_step(ctx, record, dev, (C.c_int32 * 2)(*b) if b else None, lr, beta1, beta2, eps, t, clock, None)


@pytest.mark.parametrize("change,status", [
    (dict(param=None), B.ERR_NULL), (dict(grads=None), B.ERR_NULL), (dict(grads=(1 << 28, 0)), B.ERR_NULL), (dict(m=None), B.ERR_NULL),
    (dict(v=None), B.ERR_NULL), (dict(tops=None), B.ERR_NULL), (dict(param=PTR + 2), B.ERR_ALIGN), (dict(param_lp=PTR + 1), B.ERR_ALIGN),
    (dict(grads=(1 << 28, (1 << 28) + 1)), B.ERR_ALIGN), (dict(tops=PTR + (4 << 16) + 2), B.ERR_ALIGN), (dict(weight_decay=math.nan), B.ERR_BAD_CONFIG),
    (dict(n=1 << 42), B.ERR_TOO_LARGE), (dict(n=(1 << 42) - 1), B.ERR_TOO_LARGE),
])
def test_refuses_tensors(change, status):
    for tensors in ((tensor(**change),), (tensor(1 << 25), tensor(**change))):
        first, second, *_ = plan(*tensors)
        assert first == second == status
    assert plan(tensor(), K=0)[0] == plan(tensor(), K=33)[0] == B.ERR_BAD_K
    assert plan(tensor(), dtype=2)[0] == plan(tensor(), bits=16)[0] == B.ERR_BAD_CONFIG
    assert plan(tensor(m=PTR + (2 << 16) + 2), bits=32)[0] == B.ERR_ALIGN
    assert plan(tensor(tops=None), bits=32)[0] == B.OK


@pytest.mark.parametrize("change", [dict(m=PTR), dict(v=PTR + 4 * 4999), dict(param_lp=PTR + (2 << 16) + 4998), dict(tops=PTR + (1 << 16))])
def test_refuses_results_that_overlap(change):
    assert plan(tensor(**change))[:2] == (B.OK, B.ERR_BAD_CONFIG)
    assert plan(tensor(), tensor())[1] == B.ERR_BAD_CONFIG
    assert plan(tensor(), tensor(1 << 25))[1] == B.OK
    assert plan(tensor(n=0), tensor(n=0), tensor())[1] == B.OK               # nothing is written there


@pytest.mark.parametrize("at,status", [
    (PTR, B.ERR_BAD_CONFIG), (PTR + 4 * 5000 - 2, B.ERR_BAD_CONFIG), (PTR - 2 * 5000 + 2, B.ERR_BAD_CONFIG), (PTR - 2 * 5000, B.OK),
    (PTR + (2 << 16) + 4000, B.ERR_BAD_CONFIG), (PTR + 4 * 5000, B.OK),
])
def test_refuses_gradients_that_a_step_writes(at, status):
    elsewhere = 1 << 24
    assert plan(tensor(grads=(elsewhere, at)))[1] == status
    assert plan(tensor(1 << 25, grads=(at, elsewhere)), tensor(grads=(elsewhere, elsewhere)))[1] == status


def test_record(omni):
    rc, rc2, keep, record, need = plan(tensor(), tensor(1 << 25, n=0), tensor(1 << 26, n=2049))
    assert rc == rc2 == B.OK and need >= 64 * 4 + 6 * 8 + 5 * 4
    array = (B.omni_adamw_tensor * 1)(tensor())
    one = C.c_uint64()
    assert B.lib().omni_adamw_plan_bytes(array, 1, 2, B.BF16, 8, C.byref(one)) == B.OK
    assert B.lib().omni_adamw_plan(array, 1, 2, B.BF16, 8, record, one.value - 1) == B.ERR_TOO_LARGE
    assert B.lib().omni_adamw_plan(array, 1, 2, B.BF16, 8, None, one.value) == B.ERR_NULL
    assert B.lib().omni_adamw_plan(array, 1, 2, B.BF16, 8, record + 4, one.value) == B.ERR_ALIGN
    assert B.lib().omni_adamw_plan_bytes(array, 1, 2, B.BF16, 8, None) == B.ERR_NULL
    assert B.lib().omni_adamw_plan_bytes(array, -1, 2, B.BF16, 8, C.byref(one)) == B.ERR_BAD_CONFIG
    assert B.lib().omni_adamw_plan_bytes(None, 1, 2, B.BF16, 8, C.byref(one)) == B.ERR_NULL


@pytest.mark.parametrize("change,status", [
    (dict(lr=math.nan), B.ERR_BAD_CONFIG), (dict(beta1=1.0), B.ERR_BAD_CONFIG), (dict(beta2=-0.1), B.ERR_BAD_CONFIG),
    (dict(eps=math.inf), B.ERR_BAD_CONFIG), (dict(eps=-1.0), B.ERR_BAD_CONFIG), (dict(t=0), B.ERR_BAD_CONFIG), (dict(b=(1, 0)), B.ERR_BAD_BATCH),
    (dict(b=None), B.ERR_NULL), (dict(dev=None), B.ERR_NULL), (dict(dev=PTR + 8), B.ERR_ALIGN), (dict(clock=PTR + 4), B.ERR_ALIGN),
])
def test_refuses_steps(omni, change, status):
    _, _, keep, record, _ = plan(tensor())
    assert step(omni._h, record, **change) == status
    assert step(None, record) == step(omni._h, None) == B.ERR_NULL
    junk = C.create_string_buffer(256)
    assert step(omni._h, (C.addressof(junk) + 7) // 8 * 8) == B.ERR_BAD_CONFIG


def test_moments_refuse(omni):
    tables = [(C.c_void_p * 1)(p) for p in (PTR, None, PTR + 2)]
    _, _, keep, record, _ = plan(tensor())
    call = lambda m, v, r=record: B.lib().omni_adamw_moments(omni._h, r, PTR, m, v, None)  # noqa: E731
    assert call(tables[0], tables[1]) == call(None, tables[0]) == B.ERR_NULL and call(tables[2], tables[0]) == B.ERR_ALIGN
    _, _, keep32, record32, _ = plan(tensor(), bits=32)
    assert call(tables[0], tables[0], record32) == B.ERR_BAD_CONFIG


def test_tensors_of_another_device_are_refused(omni, monkeypatch):
    monkeypatch.setattr(L, "_device", lambda: 0)
    p, g = torch.zeros(4), torch.zeros(4)
    with pytest.raises(ValueError, match="cpu"):
        L.AdamW(omni, [p], [[g]])
    op = object.__new__(L.AdamW)
    op._at, op.K, op.bits, op._record_dev = 1, 1, 8, p
    for call in (lambda: op.step(1e-3), lambda: op.moments()):
        with pytest.raises(ValueError):
            call()
