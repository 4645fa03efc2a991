"""The gradient of a padded batch with as many rows as a call may have, 2^31 - 1: bundles of rows are counted without passing 31 bits."""
import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu
N = (1 << 31) - 1


def test_as_many_rows_as_a_call_may_have():
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 20 GB on the device")
    ctx = B.Omni(1, 1, 1, 1)
    r = L.Rotary(ctx, 1, 1, 2, [1.0], interleaved=True)
    x, g = (torch.tensor([v], device="cuda").bfloat16().view(1, 1, 1, 2) for v in ([0.5, -1.25], [0.75, 2.0]))
    at, w = torch.full((1, 1), 3, device="cuda"), torch.tensor([1.5, -0.5], device="cuda")
    one = r.backward(x, x, at, g, g, w, w)
    many = [t.expand(1, N, 1, 2) for t in (x, x, g, g)]
    out = tuple(torch.zeros(1, N, 1, 2, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for length in (N, N - 5):
        lengths = torch.tensor([length], device="cuda", dtype=torch.int32)
        got = r.backward(*many[:2], at.expand(1, N), *many[2:], w, w, lengths=lengths, grads=out)
        for y, first in zip(got, one[:2]):
            same = y.view(torch.int32).view(-1) == first.view(torch.int32).view(-1)
            assert int(same.sum()) == length and bool(same[:length].all()) and not bool(y[:, length:].any())
        for dw, first in zip(got[2:], one[2:]):
            # equal terms: a chain of at most 2^16 of them in each of at least 2^15 threads, and a tree
            want = first.double() * length
            assert bool(((dw.double() - want).abs() <= want.abs() * (2 ** 16 + 64) * 2.0 ** -24).all())
