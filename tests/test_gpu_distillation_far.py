"""The distillation loss on logits far from zero: rows masked throughout by the type's lowest value or by -1e9 (their softmax is
uniform), offsets of all logits, rows of -inf throughout.  Against the definition in 64 bits.

Tolerances.  A probability depends on distances from the row's largest logit M only, D_v = (M - z_v) / T in powers of two:
three roundings of 2^-24 D and 2^-21 for the hardware's 2^x.  The sum over the row is off by the mean of that and by
(V / 128 + 16) 2^-24 for its additions; `e` below.  The lse adds M / T, its roundings 2^-23 of each.  The loss is a sum of
distances again.  Where the lse is given, its own rounding belongs to the input: exp(z / T - lse) of that float value."""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8 + 2.0 ** -24}
LOG2E = 1 / math.log(2)
VOCAB, TOP = 1003, 6


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


def inputs(dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(8, VOCAB, device="cuda", generator=gen) * 3
    low = torch.finfo(dtype).min
    z[0] = low                              # masked throughout
    z[1] = -1e9
    z[2] -= 1e4                             # all far off; what a bfloat16 keeps of it is the row
    z[3] += 1e4
    z[4] = -1e30
    z[5] = low
    z[5, 700] = low / 2                     # one less low than the others
    z[6] = -1e9
    z[6, 100:300] = 0.25 * torch.arange(200, device="cuda") - 2e3
    t = torch.randn(8, TOP, device="cuda", generator=gen) * 2
    i = torch.stack([torch.randperm(VOCAB, device="cuda", generator=gen)[:TOP] for _ in range(8)])
    i[5, 0] = 700
    i[6] = 100 + torch.arange(TOP, device="cuda") * 39
    return z.to(dtype), t, i, torch.randn(8, device="cuda", generator=gen)


@pytest.mark.parametrize("temp", [1.0, 2.0, 0.5])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_far_logits(ctx, dtype, temp):
    z, t, i, gl = inputs(dtype)
    d = L.Distillation(ctx, temp)
    loss, lse, grad = d.step(z, t, i, gl)
    loss2, lse2 = d.forward(z, t, i)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)

    x = z.double() / temp
    top = x.amax(1, keepdim=True)
    far = (top - x) * LOG2E
    s = torch.exp(x - top).sum(1, keepdim=True)
    q = torch.exp(x - top) / s
    e = ((q * far).sum(1, keepdim=True) + 1) * 2.0 ** -22 + 2.0 ** -21 + (VOCAB / 128 + 16) * 2.0 ** -24
    p = torch.softmax(t.double() / temp, 1)
    dense = torch.zeros_like(x).scatter_add_(1, i, p)

    exact_lse = (top + s.log())[:, 0]
    fits = exact_lse.abs() <= torch.finfo(F32).max
    assert bool(torch.isinf(lse[~fits]).all())
    room = e[:, 0] + 2.0 ** -23 * (top[:, 0].abs() + exact_lse.abs()) + 2.0 ** -22 * s.log()[:, 0]
    assert bool(((lse.double() - exact_lse).abs() <= room)[fits].all())

    gap = (top - x).gather(1, i)
    exact_loss = temp * temp * (p * (p.log() + gap + s.log())).sum(1)
    room = temp * temp * (e + 2.0 ** -20 * ((p * (p.log().abs() + gap + 1)).sum(1, keepdim=True) + s.log()))[:, 0]
    seen = exact_loss <= torch.finfo(F32).max
    assert bool(((loss.double() - exact_loss).abs() <= room)[seen].all()), (loss, exact_loss)
    assert bool(torch.isposinf(loss[~seen]).all())

    gain = (gl.double() * temp)[:, None]
    want = gain * (q - dense)
    room = gain.abs() * (q * (2 * e + far * 2.0 ** -22 + 2.0 ** -21) + dense * 2.0 ** -19) + ROUND[dtype] * want.abs() + 1e-38
    assert bool(((grad.double() - want).abs() <= room).all()), (grad.double() - want).abs().amax(1)

    # from the kept lse, as the float it is
    kept = d.backward(z, t, i, lse, gl)
    up = x - lse.double()[:, None]
    q = torch.exp(up)
    want = gain * (q - dense)
    room = gain.abs() * (q * (up.abs() * LOG2E * 2.0 ** -22 + 2.0 ** -21) + dense * 2.0 ** -19) + ROUND[dtype] * want.abs() + 1e-38
    assert bool(((kept.double() - want).abs() <= room)[fits].all()), (kept.double() - want).abs().amax(1)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_row_of_minus_infinity(ctx, dtype):
    """No token has a probability: the lse is -inf, the loss infinite, and the gradient what the teacher asks for."""
    z, t, i, gl = inputs(dtype, 1)
    z[3] = -math.inf
    d = L.Distillation(ctx, 2.0)
    loss, lse, grad = d.step(z, t, i, gl)
    assert float(lse[3]) == -math.inf and float(loss[3]) == math.inf
    want = torch.zeros(VOCAB, dtype=torch.float64, device="cuda").scatter_add_(0, i[3], torch.softmax(t[3].double() / 2, 0)) * gl[3].double() * -2
    for g in (grad, d.backward(z, t, i, lse, gl)):
        assert bool(((g[3].double() - want).abs() <= (2.0 ** -19 + ROUND[dtype]) * want.abs()).all())

@pytest.mark.parametrize("temp", [1.0, 0.5])
def test_a_teacher_of_lowest_values_is_uniform(ctx, temp):
    z, t, i, gl = inputs(F32, 2)
    z, i = z.nan_to_num().clamp(-10, 10), i.clone()
    t[0] = torch.finfo(F32).min
    t[1] = torch.finfo(F32).min
    t[1, 2] = -math.inf
    d = L.Distillation(ctx, temp)
    even = t.clone()
    even[0], even[1] = 0.0, 0.0
    even[1, 2] = -math.inf
    for a, b in zip(d.step(z, t, i, gl), d.step(z, even, i, gl)):
        assert torch.equal(a, b)                                   # distances from the largest entry are what counts
