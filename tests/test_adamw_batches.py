"""Batch sizes that the library takes as 32 bits are refused, not cut, and where its limit on elements lies: without a GPU."""
import ctypes as C

import pytest

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L


class Library:
    """Notes what a step passes on."""

    def __init__(self):
        self.batches = []

    def omni_adamw_step(self, ctx, record, dev, batches, *rest):
        self.batches.append(list(batches))
        return B.OK


@pytest.fixture
def op(monkeypatch):
    monkeypatch.setattr(L, "_device", lambda: 0)
    monkeypatch.setattr(L, "_raw_stream", lambda d: 0)
    op = object.__new__(L.AdamW)
    op._at, op.K, op.bits, op.steps, op.betas, op.eps, op.ctx, op._lib = 0, 2, 32, 0, (0.9, 0.9), 1e-8, B.Omni(1, 1, 1, 1), Library()
    op._record = op._record_dev = type("Record", (), {"data_ptr": staticmethod(lambda: 1 << 20)})
    op._batches = C.c_int32 * 2
    return op


@pytest.mark.parametrize("batches", [(1, 1 << 31), ((1 << 32) + 5, 1), (1, -(1 << 31) - 1), (1 << 40, 1 << 40)])
def test_sizes_past_32_bits(op, batches):
    with pytest.raises(ValueError):
        op.step(1e-3, batches)
    assert op.steps == 0 and op._lib.batches == []


def test_sizes_of_32_bits(op):
    for batches in ((1, 2), ((1 << 31) - 1, 7), [3, 4]):
        op.step(1e-3, batches)
    assert op.steps == 3 and op._lib.batches == [[1, 2], [(1 << 31) - 1, 7], [3, 4]]


def test_pieces_of_all_tensors():
    """Fewer than 2^31 of 1024 elements."""
    at, need, grads = 1 << 20, C.c_uint64(), (C.c_void_p * 1)(1 << 20)
    for sizes, status in (([(1 << 41) - 1024], B.OK), ([(1 << 41) - 1023], B.ERR_TOO_LARGE), ([1 << 40, (1 << 40) - 1024], B.OK),
                          ([1 << 40, (1 << 40) - 1024, 1], B.ERR_TOO_LARGE)):
        tensors = (B.omni_adamw_tensor * len(sizes))(*(B.omni_adamw_tensor(at, None, grads, at, at, at, n, 0.0) for n in sizes))
        assert B.lib().omni_adamw_plan_bytes(tensors, len(sizes), 1, B.F32, 8, C.byref(need)) == status
