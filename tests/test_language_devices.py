"""Which GPU a call of the language-model operators runs on: tensors that are together, but not on the current device, are
refused before the library is reached.  Stand-ins for tensors of a second GPU, so no GPU is needed."""
import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

BF16, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


class Elsewhere:
    """A contiguous tensor on cuda:1, as far as the operators look at one."""

    is_cuda, device = True, torch.device("cuda", 1)

    def __init__(self, shape, dtype):
        self.shape, self.dtype = torch.Size(shape), dtype
        self._like = torch.empty(shape, dtype=dtype, device="meta")

    def get_device(self):
        return 1

    def is_contiguous(self):
        return True

    def stride(self):
        return self._like.stride()

    def dim(self):
        return self._like.dim()

    def numel(self):
        return self._like.numel()

    def data_ptr(self):
        return 1 << 20

    def new_empty(self, shape, dtype=None):
        return Elsewhere((shape,) if isinstance(shape, int) else shape, dtype or self.dtype)


class Library:
    """What must not be reached."""

    def __getattr__(self, name):
        raise AssertionError(f"{name} was called with tensors of another device")


@pytest.fixture
def operator(monkeypatch):
    monkeypatch.setattr(L, "_device", lambda: 0)
    monkeypatch.setattr(L, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(L, "_like", lambda t: Elsewhere(t.shape, t.dtype))
    omni = B.Omni(1, 1, 1, 1)

    def make(cls, *args, **kw):
        op = cls(omni, *args, **kw)
        op._lib = Library()
        return op

    return make


def calls(make):
    e, a, d = make(L.Embedding, 10, 8), make(L.Attention, 2, 1, 8), make(L.Distillation)
    t, w, g = Elsewhere((4,), I64), Elsewhere((10, 8), F32), Elsewhere((4, 8), F32)
    q, k, lse = Elsewhere((1, 3, 2, 8), BF16), Elsewhere((1, 5, 1, 8), BF16), Elsewhere((1, 2, 3), F32)
    z, top, index, rows = Elsewhere((4, 50), F32), Elsewhere((4, 3), F32), Elsewhere((4, 3), I32), Elsewhere((4,), F32)
    return {
        "lookup": lambda: e.forward(t, w), "embedding gradient": lambda: e.backward(t, g),
        "attention": lambda: a.forward(q, k, k), "attention gradient": lambda: a.backward(q, k, k, q, lse, q),
        "loss": lambda: d.forward(z, top, index), "loss gradient": lambda: d.backward(z, top, index, rows, rows),
        "loss and gradient": lambda: d.step(z, top, index, rows),
    }


@pytest.mark.parametrize("name", ["lookup", "embedding gradient", "attention", "attention gradient", "loss", "loss gradient",
                                  "loss and gradient"])
def test_tensors_of_another_device_are_refused(operator, name):
    with pytest.raises(ValueError, match="cuda:1"):
        calls(operator)[name]()


@pytest.mark.parametrize("name", ["lookup", "embedding gradient", "attention", "attention gradient", "loss", "loss gradient",
                                  "loss and gradient"])
def test_tensors_of_the_current_device_reach_the_library(operator, monkeypatch, name):
    monkeypatch.setattr(L, "_device", lambda: 1)
    with pytest.raises(AssertionError, match="omni_"):
        calls(operator)[name]()
