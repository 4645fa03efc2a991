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
