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
