"""The policy loss's gradient from a kept log-sum-exp where that float says little: rows far from zero, and ratios next to a border.
Against the definition in 64 bits, and against the step's gradient of the same rows.

Tolerances, as in the distillation loss's test of far logits.  A probability depends on distances from the row's largest logit M only, D_v =
(M - z_v) / T in powers of two: three roundings of 2^-24 D and 2^-21 for the hardware's 2^x; the sum S over the row is off by the mean
of that and by (V / 128 + 16) 2^-24 for its additions, `e` below.  The log-probability is a distance less log S: off by l = e + 2^-22 (its
two terms + 1); ratio, slope and gradient follow as in test_gpu_policy.py.
"""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

from test_gpu_policy import inputs as near_inputs

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8 + 2.0 ** -24}
LOG2E = 1 / math.log(2)
TEMPERATURES = [0.6, 0.7, 1.0, 2.0]


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


def far_inputs(dtype, vocab):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = torch.randn(11, vocab, device="cuda", generator=gen) * 3
    low, most = torch.finfo(dtype).min, vocab // 3
    z[0] = low                                       # masked throughout by the type's lowest value, by -1e9, by -1e30
    z[1] = -1e9
    z[2] = -1e30
    z[3] = 1e30
    z[3, most:] = -math.inf
    z[4] -= 1e4                                      # all far off
    z[5] += 1e6
    z[6] += 200
    z[7] -= 3e7
    z[8] = low
    z[8, 7] = low / 2                                # one less low than the others
    z[9] = -1e9                                      # a mask around what counts, which is far from zero itself
    z[9, :most] = -0.25 * torch.arange(most, device="cuda") - 2e3
    tokens = torch.randint(0, most, (11,), device="cuda", generator=gen)
    tokens[8] = 7
    tokens[9] = 5
    tokens[10] = 9                                   # near zero: as it always was
    return z.to(dtype), tokens, torch.randn(11, device="cuda", generator=gen), torch.randn(11, device="cuda", generator=gen)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("temp", TEMPERATURES)
@pytest.mark.parametrize("vocab", [100, 5003, 70001])
def test_rows_far_from_zero(ctx, dtype, temp, vocab):
    p = L.Policy(ctx, 0.2, 0.28, 0.1, temp)
    z, tokens, advantage, gl = far_inputs(dtype, vocab)
    x = z.double() / temp
    top = x.amax(1, keepdim=True)
    far = ((top - x) * LOG2E).nan_to_num(posinf=0.0)
    s = torch.exp(x - top).sum(1, keepdim=True)
    q = torch.exp(x - top) / s
    gap = (top - x).gather(1, tokens[:, None])[:, 0]
    logp = -gap - s.log()[:, 0]
    old, reference = (logp - 0.1).float(), (logp + 0.3).float()
    _, _, lse = p.forward(z, tokens, old, advantage, reference)
    kept = p.backward(z, tokens, lse, old, advantage, gl, reference)
    stepped = p.step(z, tokens, old, advantage, gl, reference)[3]
    own = z.clone()
    assert torch.equal(p.backward(own, tokens, lse, old, advantage, gl, reference, grad=own), kept)

    e = ((q * far).sum(1) + 1) * 2.0 ** -22 + 2.0 ** -21 + (vocab / 128 + 16) * 2.0 ** -24
    l = e + 2.0 ** -22 * (gap + s.log()[:, 0] + 1)
    a, ratio, away = advantage.double(), torch.exp(logp - old.double()), reference.double() - logp
    slope = -ratio * a - p.kl * torch.expm1(away)    # about e^0.1: inside the borders
    slope_error = a.abs() * ratio * (l + 2.0 ** -23 * ((logp - old.double()).abs() + 3)) + p.kl * torch.exp(away) * (l + 2.0 ** -22 * (away.abs() + 2))
    gain = (gl.double() / temp)[:, None]
    one = torch.zeros_like(q).scatter_(1, tokens[:, None], 1.0)
    want = gain * slope[:, None] * (one - q)
    room = gain.abs() * slope_error[:, None] * (one - q).abs() + (gain * slope[:, None]).abs() * (
        q * (2 * e[:, None] + far * 2.0 ** -22 + 2.0 ** -21) + (one + q) * 2.0 ** -22) + ROUND[dtype] * want.abs() + 1e-38
    for got in (stepped, kept):
        # the last row is near zero, where the kept lse is what the gradient is taken from
        err = (got.double() - want).abs()[:10]
        assert bool((err <= room[:10]).all()), (err - room[:10]).amax(1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("temp", TEMPERATURES)
@pytest.mark.parametrize("clip,high", [(0.0, None), (0.0, 0.5), (0.2, 0.28), (1.0, 0.0)])
def test_ratios_next_to_a_border(ctx, dtype, temp, clip, high):
    """What forward counts as not clipped has its gradient from either call, a few steps of the float around a border."""
    p = L.Policy(ctx, clip, high, 0.0, temp)
    z, tokens, _, advantage, _, gl = near_inputs(4000, 100, dtype, torch.int64, 11, p)
    logp, lse = p.logprob(z, tokens)
    gen = torch.Generator(device="cuda").manual_seed(5)
    for border in (1.0, 1 - p.clip, 1 + p.clip_high):
        if border <= 0:
            continue
        old = logp - math.log(border)
        for steps in (0, 4):
            shift = torch.randint(-steps, steps + 1, old.shape, device="cuda", generator=gen)
            close = old + shift * (old.abs() + 1) * 2.0 ** -24
            grad = p.step(z, tokens, close, advantage, gl)[3].double()
            kept = p.backward(z, tokens, lse, close, advantage, gl).double()
            assert torch.equal(kept.abs().amax(1) > 0, grad.abs().amax(1) > 0)
            # twice `e` of test_gpu_policy.py, which is below 2^-16 for logits of this size
            room = 1.5 * (gl * advantage / temp).double().abs()[:, None] * 2.0 ** -15 + 2 * ROUND[dtype] * grad.abs()
            assert bool(((kept - grad).abs() <= room).all())
        if border == 1.0:
            assert torch.equal(p.backward(z, tokens, lse, old, advantage, gl).abs().amax(1) > 0, tokens >= 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("temp", TEMPERATURES)
def test_tokens_far_below_their_row(ctx, dtype, temp):
    """The row is near zero, the sampled token masked by a large number: its log-probability is lost in a difference of floats as well.  The ratio to an
    `old` of the same call is that call's, so the gradient is the step's to the bit."""
    p = L.Policy(ctx, 0.2, 0.28, 0.05, temp)
    masks = [-300.0, -3e3, -1e5, -3e7, -1e9, -1e30, torch.finfo(dtype).min, -math.inf]
    rows = 20 * len(masks)
    z, tokens, _, advantage, _, gl = near_inputs(rows, 1000, dtype, torch.int64, 12, p)
    tokens = tokens.clamp(min=0)
    z[torch.arange(rows), tokens] = torch.tensor(masks, device="cuda").repeat_interleave(20).to(dtype)
    logp, lse = p.logprob(z, tokens)
    assert float(lse.abs().max()) < 64
    old, reference = logp - 0.1, logp.clamp(min=-1e38) + 0.3
    grad = p.step(z, tokens, old, advantage, gl, reference)[3]
    kept = p.backward(z, tokens, lse, old, advantage, gl, reference)
    same = (kept == grad) | (kept.isnan() & grad.isnan())
    assert bool(same.all()), (~same).any(1).nonzero()[:, 0]
