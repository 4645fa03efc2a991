"""The backward pass begins while its own first kernel, the row sums, still runs.  A call without a pair of a query and a key
needs nothing of that kernel, but may not be over before it: what follows it in a graph takes over the scratch memory and the
output's gradient.  What is asked for is exact."""
import gc

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv_len,keys", [(0, None), (256, 0)])
def test_a_call_without_pairs_ends_after_its_row_sums(kv_len, keys):
    ctx = B.Omni(1, 1, 1, 1)
    batch, q_len, heads, dim = 8, 4096, 16, 64
    a = L.Attention(ctx, heads, 4, dim)
    q, do = (torch.randn(batch, q_len, heads, dim, device="cuda").bfloat16() for _ in range(2))
    k = torch.randn(batch, kv_len, 4, dim, device="cuda").bfloat16()
    lengths = None if keys is None else torch.full((batch,), keys, dtype=torch.int32, device="cuda")
    out, lse = a.forward(q, k, k, None, lengths)
    a.backward(q, k, k, out, lse, do, None, lengths)
    torch.cuda.synchronize()
    gc.collect()
    scratch = 2 * batch * heads * q_len * 4
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        grads = a.backward(q, k, k, out, lse, do, None, lengths)
        after = torch.full((scratch,), 7, dtype=torch.uint8, device="cuda")      # the allocator's next block of that size
    for _ in range(20):
        g.replay()
        torch.cuda.synchronize()
        assert bool((after == 7).all()) and not any(bool(x.any()) for x in grads)
    ctx.stats()
