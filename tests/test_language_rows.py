"""What the operators make of strides and shapes before they look at a device; no GPU is needed."""
import torch

from paper_2503_17469_b200 import language as L


def test_the_stride_of_a_single_row_does_not_matter():
    """Two matrices of one row with the same number of columns have the same layout, whatever they were cut from."""
    assert L._rows(torch.empty(1, 100)[:, :5], "x") == L._rows(torch.empty(1, 5), "x") == 5
    assert L._rows(torch.empty(3, 100)[:1, :5], "x") == 5
    assert L._rows(torch.empty(0, 100)[:, :5], "x") == 5
    assert L._rows(torch.empty(3, 100)[:, :5], "x") == 100
