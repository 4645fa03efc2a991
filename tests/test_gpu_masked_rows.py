"""Rows of logits masked in part by large negative numbers, in stretches that whole threads, warps and parts of a row see nothing but:
such a logit has probability 0, whatever the number, as one of -inf has.  So the results are those of the row with -inf in these places: the
same bits, since a term of 0 is added in either case."""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


def rows(dtype, vocab, value):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = (torch.randn(4, vocab, device="cuda", generator=gen) * 3).to(dtype)
    z[0, : vocab - 20] = value
    z[1, 20:] = value
    z[2, 5::2] = value
    z[3, vocab // 3:vocab - 1] = value
    tokens = torch.tensor([vocab - 3, 7, 4, 1], device="cuda")
    return z, tokens, gen


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [-1e6, -1e10, -1e20, -1e30, -3e38])
@pytest.mark.parametrize("vocab", [101, 3001, 50257, 131072, 300007])
def test_policy(ctx, dtype, value, vocab):
    z, tokens, gen = rows(dtype, vocab, value)
    masked = torch.where(z.float() < -1e5, -math.inf, z.float()).to(dtype)
    p = L.Policy(ctx, kl=0.1)
    one = torch.ones(4, device="cuda")
    old = p.logprob(masked, tokens)[0] - 0.05
    got, want = (p.step(x, tokens, old, one, one, old) for x in (z, masked))
    back = [p.backward(x, tokens, want[2], old, one, one, old) for x in (z, masked)]
    for x, y in zip((*got, back[0], *p.logprob(z, tokens)), (*want, back[1], *p.logprob(masked, tokens))):
        assert bool(y.isfinite().all()) and torch.equal(x, y)
    assert torch.allclose(got[1].double(), torch.log_softmax(masked.double(), 1).gather(1, tokens[:, None])[:, 0], rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [-1e6, -1e10, -1e30, -3e38])
@pytest.mark.parametrize("vocab", [101, 3001, 50257])
def test_distillation(ctx, dtype, value, vocab):
    z, tokens, gen = rows(dtype, vocab, value)
    masked = torch.where(z.float() < -1e5, -math.inf, z.float()).to(dtype)
    d = L.Distillation(ctx, 1.0)
    top = torch.zeros(4, 1, device="cuda")
    got, want = (d.step(x, top, tokens[:, None], torch.ones(4, device="cuda")) for x in (z, masked))
    for x, y in zip(got, want):
        assert bool(y.isfinite().all()) and torch.equal(x, y)
