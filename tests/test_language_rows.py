"""What the operators make of strides and shapes before they look at a device; no GPU is needed."""
import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L


def test_the_stride_of_a_single_row_does_not_matter():
    """Two matrices of one row with the same number of columns have the same layout, whatever they were cut from."""
    assert L._rows(torch.empty(1, 100)[:, :5], "x") == L._rows(torch.empty(1, 5), "x") == 5
    assert L._rows(torch.empty(3, 100)[:1, :5], "x") == 5
    assert L._rows(torch.empty(0, 100)[:, :5], "x") == 5
    assert L._rows(torch.empty(3, 100)[:, :5], "x") == 100

@pytest.mark.parametrize("grad", [torch.zeros(8, 3, 2).permute(2, 1, 0), torch.zeros(2, 3, 7), torch.zeros(47), torch.zeros(7, 8)])
def test_gradients_that_are_no_matrix_of_rows_are_refused_as_such(grad):
    e = L.Embedding(B.Omni(1, 1, 1, 1), 10, 8)
    with pytest.raises(ValueError, match="6 rows of 8"):
        e.backward(torch.zeros(2, 3, dtype=torch.int64), grad)


class Sized:
    """A tensor of a size that nobody has, as far as the checks look at it."""

    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, *shape, dtype=torch.float32):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def stride(self):
        s, at = [], 1
        for n in reversed(self.shape):
            s.insert(0, at)
            at *= n
        return tuple(s)

    def get_device(self):
        return 0

    def data_ptr(self):
        return 1 << 20


def test_sizes_that_the_library_does_not_count_in_are_refused(monkeypatch):
    """The C ABI takes them as 32 bits; 2^32 + 10 would be 10 there."""
    monkeypatch.setattr(L, "_device", lambda: 0)
    omni, big = B.Omni(1, 1, 1, 1), 2 ** 32 + 10
    for make in (lambda: L.Embedding(omni, big, 8), lambda: L.Embedding(omni, 10, big), lambda: L.Attention(omni, big, big, 8),
                 lambda: L.Attention(omni, 2, 2, big)):
        with pytest.raises(ValueError, match="2\\*\\*31"):
            make()
    d, a = L.Distillation(omni), L.Attention(omni, 2, 2, 8)
    with pytest.raises(ValueError, match="2\\*\\*31"):
        d._describe(Sized(1, big), Sized(1, 4), Sized(1, 4, dtype=torch.int64))
    with pytest.raises(ValueError, match="2\\*\\*31"):
        d._describe(Sized(1, 50), Sized(1, big), Sized(1, big, dtype=torch.int64))
    q, long = Sized(1, 5, 2, 8, dtype=torch.bfloat16), Sized(1, big, 2, 8, dtype=torch.bfloat16)
    for x, y in ((q, long), (long, q), (Sized(big, 5, 2, 8), Sized(big, 5, 2, 8))):
        with pytest.raises(ValueError, match="2\\*\\*31"):
            a._describe(x, y, None, None)
    a._describe(q, q, None, None)
    d._describe(Sized(1, 2 ** 31 - 1), Sized(1, 4), Sized(1, 4, dtype=torch.int64))
