"""What the policy loss checks before it touches a device: status codes, tensors of another device."""
import ctypes as C
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

from test_language_devices import F32, I64, Elsewhere, Library

PTR = 1 << 20        # an aligned address that no call here gets to use


@pytest.fixture(scope="module")
def omni():
    return B.Omni(1, 1, 1, 1)


def policy(**kw):
    d = dict(logits=PTR, rows=3, row_stride=50, vocab=50, dtype=B.F32, tokens=PTR, old=PTR, advantage=PTR, reference=PTR,
             index_type=B.I64, clip_low=0.2, clip_high=0.2, kl=0.1, temperature=1.0)
    d.update(kw)
    return C.byref(B.omni_policy(*d.values()))


@pytest.mark.parametrize("change,status,valued_only", [
    (dict(dtype=3), B.ERR_BAD_CONFIG, False), (dict(index_type=2), B.ERR_BAD_CONFIG, False), (dict(vocab=0), B.ERR_BAD_CONFIG, False),
    (dict(temperature=0.0), B.ERR_BAD_CONFIG, False), (dict(temperature=math.nan), B.ERR_BAD_CONFIG, False),
    (dict(row_stride=49), B.ERR_BAD_CONFIG, False), (dict(rows=1 << 31), B.ERR_TOO_LARGE, False), (dict(logits=None), B.ERR_NULL, False),
    (dict(tokens=None), B.ERR_NULL, False), (dict(logits=PTR + 2), B.ERR_ALIGN, False), (dict(tokens=PTR + 4), B.ERR_ALIGN, False),
    (dict(clip_low=-0.1), B.ERR_BAD_CONFIG, True), (dict(clip_high=math.inf), B.ERR_BAD_CONFIG, True), (dict(kl=math.nan), B.ERR_BAD_CONFIG, True),
    (dict(old=None), B.ERR_NULL, True), (dict(advantage=None), B.ERR_NULL, True), (dict(reference=None), B.ERR_NULL, True),
    (dict(old=PTR + 2), B.ERR_ALIGN, True), (dict(reference=PTR + 1), B.ERR_ALIGN, True),
])
def test_refuses(omni, change, status, valued_only):
    lib = B.lib()
    assert lib.omni_policy_forward(omni._h, policy(**change), PTR, PTR, PTR, None) == status
    assert lib.omni_policy_backward(omni._h, policy(**change), PTR, PTR, PTR, 50, None) == status
    assert lib.omni_policy_step(omni._h, policy(**change), PTR, PTR, PTR, PTR, PTR, 50, None) == status
    if not valued_only:
        assert lib.omni_policy_logprob(omni._h, policy(**change), PTR, PTR, None) == status


def test_refuses_outputs(omni):
    lib = B.lib()
    assert lib.omni_policy_logprob(omni._h, policy(), None, PTR, None) == lib.omni_policy_logprob(omni._h, policy(), PTR, None, None) == B.ERR_NULL
    assert lib.omni_policy_logprob(None, policy(), PTR, PTR, None) == lib.omni_policy_logprob(omni._h, None, PTR, PTR, None) == B.ERR_NULL
    assert lib.omni_policy_forward(omni._h, policy(), None, PTR, PTR, None) == B.ERR_NULL
    assert lib.omni_policy_backward(omni._h, policy(), None, PTR, PTR, 50, None) == B.ERR_NULL
    assert lib.omni_policy_backward(omni._h, policy(), PTR, PTR, PTR, 49, None) == B.ERR_BAD_CONFIG
    assert lib.omni_policy_step(omni._h, policy(), None, PTR, PTR, PTR, PTR, 50, None) == B.ERR_NULL
    assert lib.omni_policy_step(omni._h, policy(), PTR, PTR, PTR + 2, PTR, PTR, 50, None) == B.ERR_ALIGN


def test_tensors_of_another_device_are_refused(omni, monkeypatch):
    monkeypatch.setattr(L, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(L, "_like", lambda t: Elsewhere(t.shape, t.dtype))
    monkeypatch.setattr(Elsewhere, "unbind", lambda t, dim: [Elsewhere(t.shape[1:], t.dtype) for _ in range(t.shape[0])], raising=False)
    p = L.Policy(omni, kl=0.1)
    p._lib = Library()
    z, t, r = Elsewhere((4, 50), F32), Elsewhere((4,), I64), Elsewhere((4,), F32)
    for call in (lambda: p.logprob(z, t), lambda: p.forward(z, t, r, r, r), lambda: p.backward(z, t, r, r, r, r, r),
                 lambda: p.step(z, t, r, r, r, r)):
        monkeypatch.setattr(L, "_device", lambda: 0)
        with pytest.raises(ValueError, match="cuda:1"):
            call()
        monkeypatch.setattr(L, "_device", lambda: 1)
        with pytest.raises(AssertionError, match="omni_"):
            call()
    with pytest.raises(ValueError):
        p.logprob(torch.zeros(4, 50), torch.zeros(4, dtype=torch.int64))
