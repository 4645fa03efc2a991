"""Queries inside their sequence that see no key (causal, more queries than keys) take part in no gradient, whatever they and
their output's gradient hold.  Bits are compared: a row that does not take part changes nothing."""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

from test_gpu_attention import tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_len,kv_len,q_lengths,kv_lengths", [
    (200, 130, None, None), (300, 44, None, None), (256, 128, None, None), (3000, 11, None, None),
    (333, 333, [333, 300, 129], [200, 300, 1]),
])
def test_queries_without_keys_may_hold_anything(dim, q_len, kv_len, q_lengths, kv_lengths):
    ctx = B.Omni(1, 1, 1, 1)
    batch = len(q_lengths) if q_lengths else 2
    q, k, v, do = tensors(batch, q_len, kv_len, 4, 2, dim, 90)
    ql, kl = (None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_lengths, kv_lengths))
    a = L.Attention(ctx, 4, 2, dim)
    out, lse = a.forward(q, k, v, ql, kl)
    want = a.backward(q, k, v, out, lse, do, ql, kl)
    for b in range(batch):
        n, m = (q_lengths[b], kv_lengths[b]) if q_lengths else (q_len, kv_len)
        q[b, :n - m] = math.nan
        do[b, :n - m] = math.inf
    out2, lse2 = a.forward(q, k, v, ql, kl)
    got = a.backward(q, k, v, out2, lse2, do, ql, kl)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    ctx.stats()


@pytest.mark.parametrize("dim", [16, 64, 80, 128])
@pytest.mark.parametrize("batch,q_len,kv_len", [(3, 200, 200), (2, 3000, 70)])
def test_what_stands_behind_the_lengths_stays_zero_beside_a_nan(dim, batch, q_len, kv_len):
    """A NaN in the output's gradient belongs to the keys that its query sees, not to the padding behind them."""
    ctx = B.Omni(1, 1, 1, 1)
    q, k, v, do = tensors(batch, q_len, kv_len, 4, 2, dim, 95)
    n = torch.tensor([60, 9, 33][:batch], dtype=torch.int32, device="cuda")
    a = L.Attention(ctx, 4, 2, dim, causal=False)
    out, lse = a.forward(q, k, v, n, n)
    want = a.backward(q, k, v, out, lse, do, n, n)
    do[0, 3] = math.nan
    got = a.backward(q, k, v, out, lse, do, n, n)
    for x, y in zip(want, got):
        assert torch.equal(x[1:], y[1:]) and not bool(y[0, 60:].any())
        assert bool(y[0, :60].isnan().any())
    ctx.stats()
