"""The losses over as many tokens as a call may have, 2^31 - 1, with a gradient that lies to 16-byte boundaries otherwise than the logits: the
element-by-element walk ends there instead of passing 31 bits.

Equal logits: a probability is 1 / V, the sum over the row V times 1 (e = (V / 512 / 4 + 16) 2^-24 for partial sums that are all whole numbers
below 2^24, and so exact; their tree 2^-20), then the stored type's 2^-8."""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu
V = (1 << 31) - 1


@pytest.mark.parametrize("loss", ["policy", "distillation", "distillation without a target"])
def test_as_many_tokens_as_a_call_may_have(loss):
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 20 GB on the device")
    ctx = B.Omni(1, 1, 1, 1)
    z = torch.zeros(1, V, device="cuda", dtype=torch.bfloat16)
    store = torch.full((V + 600,), 5.0, device="cuda", dtype=torch.bfloat16)
    grad, one, last = store[1:V + 1].view(1, V), torch.ones(1, device="cuda"), torch.full((1,), V - 1, device="cuda")
    if loss == "policy":
        old = torch.full((1,), -math.log(V), device="cuda")
        _, logp, lse, _ = L.Policy(ctx, 0.5).step(z, last, old, one, one, grad=grad)
        assert abs(float(logp) + math.log(V)) < 1e-4
    else:
        index = last[:, None] if loss == "distillation" else -torch.ones(1, 1, device="cuda", dtype=torch.int64)
        _, lse, _ = L.Distillation(ctx).step(z, torch.zeros(1, 1, device="cuda"), index, one, grad=grad)
    torch.cuda.synchronize()
    assert abs(float(lse) - math.log(V)) < 1e-4
    p = 0.0 if loss.endswith("target") else 1.0 / V
    same = grad[0] == grad[0, 0]
    assert abs(float(grad[0, 0]) - p) <= p * (2.0 ** -8 + 2.0 ** -16)
    if p:
        assert not bool(same[-1]) and abs(float(grad[0, -1]) + 1.0) <= 2.0 ** -8
    else:
        assert bool(same[-1])
    assert bool(same[:-1].all())
    assert float(store[0]) == 5.0 and bool((store[V + 1:] == 5.0).all())
