"""Clipped policy loss on sampled tokens against a plain implementation in 64 bits.

Tolerances.  As in the distillation loss, exponents are powers of two of x = z log2(e) / T, rounded to float: an exponential is off by
X 2^-22 (X the largest |x| and |lse| of the row, in powers of two) plus 2^-21 for the hardware's 2^x, a sum over the vocabulary by
(V / 128 + 16) 2^-24.  `e` is their sum.  Then
  |lse error| <= e + 2^-23 |lse|;  |logp error| <= l = e + 2^-22 |logp|  (from a kept lse 2^-23 (|lse| + |logp|) more);
  the ratio is off by r = l + 2^-23 (|logp - old| + 2) of itself, exp(gap) by l + 2^-22 and the gap's own 2^-24;
  |loss error| <= |A| ratio (r + 2^-23) + kl (|exp(gap) - 1| l + 2^-22 (exp(gap) + |gap| + 1)), the slope's the same with exp(gap) l;
  |grad error| <= |grad_loss| / T (slope error + |slope| 2^-22) (where not clipped) + |slope grad_loss| / T p 2 e, and the stored type's rounding.
"""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8 + 2.0 ** -24}


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


def exact(p, z, tokens, old, advantage, reference):
    """(loss, logp, lse, slope, probabilities, rows with a token) in double."""
    z = z.double() / p.temperature
    there = (tokens >= 0) & (tokens < z.shape[1])
    at = torch.where(there, tokens.long(), 0)[:, None]
    lse = torch.logsumexp(z, 1)
    logp = torch.where(lse == -math.inf, -math.inf, z.gather(1, at)[:, 0] - lse)
    a, ratio = advantage.double(), torch.exp(logp - old.double())
    clipped = ratio.clamp(1 - p.clip, 1 + p.clip_high)
    active = ratio * a <= clipped * a
    surrogate = torch.where(a == 0, 0.0, torch.minimum(ratio * a, clipped * a))
    loss, slope = -surrogate, torch.where(a == 0, 0.0, -ratio * a * active)
    if p.kl:
        gap = reference.double() - logp
        loss, slope = loss + p.kl * (torch.expm1(gap) - gap), slope - p.kl * torch.expm1(gap)
    q = torch.where((lse == -math.inf)[:, None], 0.0, torch.exp(z - lse[:, None]))
    return torch.where(there, loss, 0.0), torch.where(there, logp, 0.0), lse, torch.where(there, slope, 0.0), q, there


def errors(p, z, logp, lse, old, advantage, reference, kept):
    """(e, l, loss error, slope error) of the rows."""
    x = (z.double() / p.temperature).nan_to_num(neginf=0.0).abs().amax(1)
    x = torch.maximum(x, lse.abs()) / math.log(2)
    e = x * 2.0 ** -22 + 2.0 ** -21 + (z.shape[1] / 128 + 16) * 2.0 ** -24
    l = e + 2.0 ** -22 * logp.abs() + kept * 2.0 ** -23 * (lse.abs() + logp.abs())
    far = (logp - old.double()).abs()
    size = advantage.double().abs() * torch.exp(logp - old.double())
    loss = slope = size * (l + 2.0 ** -23 * (far + 3))
    if p.kl:
        gap = reference.double() - logp
        loss = loss + p.kl * (torch.expm1(gap).abs() * l + 2.0 ** -22 * (torch.exp(gap) + gap.abs() + 1))
        slope = slope + p.kl * torch.exp(gap) * (l + 2.0 ** -22 * (gap.abs() + 2))
    return e, l, loss, slope


def check(ctx, p, z, tokens, old, advantage, reference, gl, grad=None):
    logp0, lse0 = p.logprob(z, tokens)
    loss, logp, lse = p.forward(z, tokens, old, advantage, reference)
    g1 = p.backward(z, tokens, lse, old, advantage, gl, reference)
    loss2, logp2, lse2, g2 = p.step(z, tokens, old, advantage, gl, reference, grad=grad)
    for a, b in ((logp0, logp), (lse0, lse), (loss2, loss), (logp2, logp), (lse2, lse)):
        assert torch.equal(a, b)
    wloss, wlogp, wlse, slope, q, there = exact(p, z, tokens, old, advantage, reference)
    one = torch.zeros_like(q).scatter_(1, torch.where(there, tokens.long(), 0)[:, None], there.double()[:, None])
    for g, kept in ((g1, 1), (g2, 0)):
        e, l, loss_error, slope_error = errors(p, z, wlogp, wlse, old, advantage, reference, kept)
        if not kept:
            assert bool(((lse.double() - wlse).abs() <= e + 2.0 ** -23 * wlse.abs()).all())
            assert bool(((logp.double() - wlogp).abs() <= l * there).all())
            assert bool(((loss.double() - wloss).abs() <= (loss_error + 2.0 ** -24 * wloss.abs()) * there).all())
        gain = (gl.double() / p.temperature)[:, None]
        want = gain * slope[:, None] * (one - q)
        bound = gain.abs() * (slope_error * there)[:, None] * (one - q).abs() + (gain * slope[:, None]).abs() * (
            q * 2 * e[:, None] + (one + q) * 2.0 ** -22) + ROUND[z.dtype] * want.abs() + 1e-38
        assert g.dtype == z.dtype
        err = (g.double() - want).abs()
        assert bool((err <= bound).all()), float((err - bound).max())


def inputs(rows, vocab, dtype, index, seed, p):
    """Rows like a batch of answers: sampled tokens, a policy that has moved since, no row next to a border of the ratio."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    z = (rand(rows, vocab) * 3).to(dtype)
    tokens = (z.float() / p.temperature - torch.empty_like(z, dtype=F32).exponential_(generator=gen).log()).argmax(1)
    logp = torch.log_softmax(z.double() / p.temperature, 1).gather(1, tokens[:, None])[:, 0]
    moved = rand(rows).double() * 0.3
    for border in (1 - p.clip, 1 + p.clip_high):
        if border > 0:
            moved += 0.002 * ((moved - math.log(border)).abs() < 0.001)
    old, reference = (logp - moved).float(), (logp + rand(rows) * 0.4).float()
    tokens[rand(rows) > 1.2] = -1
    return z, tokens.to(index), old, rand(rows), reference if p.kl else None, rand(rows)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,index,temp,kl", [
    (1, 1, torch.int64, 1.0, 0.0), (3, 7, torch.int32, 2.0, 0.1), (5, 16, torch.int64, 1.0, 0.1), (40, 100, torch.int32, 0.7, 0.0),
    (333, 1000, torch.int64, 1.0, 0.04), (9, 5003, torch.int32, 2.0, 0.3), (70, 50257, torch.int64, 1.0, 0.02),
    (2, 131075, torch.int32, 1.0, 0.1), (1, 300007, torch.int64, 1.0, 0.0), (2, 1000003, torch.int64, 0.9, 0.1), (200, 131072, torch.int32, 1.0, 0.1),
    (600, 2049, torch.int32, 1.0, 0.0), (20000, 33, torch.int64, 1.0, 0.1),
])
def test_against_64_bits(ctx, dtype, rows, vocab, index, temp, kl):
    p = L.Policy(ctx, 0.2, 0.28, kl, temp)
    check(ctx, p, *inputs(rows, vocab, dtype, index, rows + vocab, p))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("clip,high", [(0.0, None), (0.1, 0.5), (1.0, 0.0), (3.0, 100.0)])
def test_clipping(ctx, dtype, clip, high):
    p = L.Policy(ctx, clip, high, 0.0)
    z, tokens, old, advantage, _, gl = inputs(500, 100, dtype, torch.int64, 1, p)
    check(ctx, p, z, tokens, old, advantage, None, gl)
    check(ctx, p, z, tokens, old - 5.0, advantage, None, gl)         # ratios of about 150
    check(ctx, p, z, tokens, old + 5.0, advantage, None, gl)
    # on the policy itself the ratio is 1, inside or on every border: the gradient is the plain policy gradient
    logp, lse = p.logprob(z, tokens)
    loss, _, _, grad = p.step(z, tokens, logp, advantage, gl)
    there = tokens >= 0
    assert torch.equal(loss, torch.where(there, -advantage, 0.0))
    assert torch.equal(grad.float().abs().amax(1) > 0, there)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_without_a_token_and_of_no_weight(ctx, dtype):
    p = L.Policy(ctx, kl=0.1)
    z, tokens, old, advantage, reference, gl = inputs(8, 777, dtype, torch.int64, 2, p)
    tokens = tokens.clamp(min=0)
    tokens[0], tokens[1], tokens[2] = -1, 777, -(2 ** 40)
    check(ctx, p, z, tokens, old, advantage, reference, gl)
    old[0] = advantage[1] = reference[2] = gl[0] = math.nan
    old[1], advantage[0] = -math.inf, math.inf
    advantage[3], gl[4] = 0.0, 0.0
    old[3] = -math.inf                                               # an infinite ratio of an advantage of zero
    loss, logp, lse, grad = p.step(z, tokens, old, advantage, gl, reference)
    back = p.backward(z, tokens, lse, old, advantage, gl, reference)
    for t in (loss, logp, grad, back):
        assert not bool(t[:3].any())
    assert bool(loss.isfinite().all()) and bool(grad.isfinite().all()) and bool(back.isfinite().all())
    assert not bool(grad[4].any()) and bool(grad[3].any())
    z[0] = math.nan                                                  # nothing of its logits reaches the gradient
    assert not bool(p.step(z, tokens, old, advantage, gl, reference, grad=z)[3][:3].any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_vocabulary_and_rows_far_from_zero(ctx, dtype):
    p = L.Policy(ctx, kl=0.1)
    low = torch.finfo(dtype).min
    z, tokens, old, advantage, reference, gl = inputs(7, 3001, dtype, torch.int32, 3, p)
    tokens = tokens.clamp(0, 2899)
    z[:, 2900:] = -math.inf
    z[0, 8:2000] = low
    z[0, tokens[0].long()] = 1.0
    z[3, :2800] = -math.inf                                          # whole stretches of threads see nothing
    tokens[3] = 2850
    logp = p.logprob(z, tokens)[0]
    old, reference = logp - 0.1, logp + 0.3
    check(ctx, p, z, tokens, old, advantage, reference, gl)
    # masked throughout by a large number: uniform over what is equal
    for value in (-1e9, low, 1e30):
        y = torch.full((2, 500), value, device="cuda", dtype=dtype)
        y[:, 100:] = -math.inf
        t = torch.tensor([3, 99], device="cuda")
        want = torch.full((2,), -math.log(100.0), device="cuda")
        logp, _ = p.logprob(y, t)
        assert torch.allclose(logp, want, rtol=1e-6)
        loss, logp2, _, grad = p.step(y, t, want, torch.ones(2, device="cuda"), torch.ones(2, device="cuda"), want)
        assert torch.equal(logp2, logp) and torch.allclose(loss, -torch.ones(2, device="cuda"), atol=1e-5)
        flat = torch.zeros(2, 500, device="cuda")
        flat[:, :100] = 0.01
        flat[[0, 1], [3, 99]] = -0.99
        assert torch.allclose(grad.float(), flat, rtol=2.0 ** -7, atol=1e-6)
    # the token itself ruled out: probability 0, no surrogate gradient, an infinite divergence
    y = z[:1].clone()
    y[0, 5] = -math.inf
    q = L.Policy(ctx)
    loss, logp, lse, grad = q.step(y, torch.tensor([5], device="cuda"), old[:1], advantage[:1].abs(), gl[:1])
    assert float(loss) == 0.0 and float(logp) == -math.inf and not bool(grad.any()) and math.isfinite(lse)
    assert not bool(q.backward(y, torch.tensor([5], device="cuda"), lse, old[:1], advantage[:1].abs(), gl[:1]).any())
    assert float(p.forward(y, torch.tensor([5], device="cuda"), old[:1], advantage[:1], reference[:1])[0]) == math.inf
    y[0, 77] = math.nan
    assert math.isnan(p.forward(y, torch.tensor([6], device="cuda"), old[:1], advantage[:1], reference[:1])[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift,stride,gshift,gstride", [(0, 1008, 0, 1008), (1, 1003, 1, 1003), (3, 1001, 0, 1000), (0, 1024, 5, 1001)])
def test_strides_and_alignment(ctx, dtype, shift, stride, gshift, gstride):
    p = L.Policy(ctx, kl=0.05)
    z, tokens, old, advantage, reference, gl = inputs(9, 1000, dtype, torch.int64, 4, p)
    raw = torch.zeros(shift + 9 * stride, device="cuda", dtype=dtype)
    zs = raw.as_strided((9, 1000), (stride, 1), shift)
    zs.copy_(z)
    store = torch.full((gshift + 9 * gstride + 9,), 5.0, device="cuda", dtype=dtype)
    gs = store.as_strided((9, 1000), (gstride, 1), gshift)
    check(ctx, p, zs, tokens, old, advantage, reference, gl, grad=gs)
    untouched = torch.ones_like(store, dtype=torch.bool)
    untouched.as_strided((9, 1000), (gstride, 1), gshift).fill_(False)
    assert bool((store[untouched] == 5.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [100, 50257, 131075])
def test_gradient_in_place(ctx, dtype, vocab):
    p = L.Policy(ctx, kl=0.05)
    z, tokens, old, advantage, reference, gl = inputs(300, vocab, dtype, torch.int64, 5, p)
    loss, _, lse, want = p.step(z, tokens, old, advantage, gl, reference)
    kept = p.backward(z, tokens, lse, old, advantage, gl, reference)
    for _ in range(3):
        a, b = z.clone(), z.clone()
        assert p.backward(a, tokens, lse, old, advantage, gl, reference, grad=a) is a
        loss2, _, _, _ = p.step(b, tokens, old, advantage, gl, reference, grad=b)
        assert torch.equal(b, want) and torch.equal(loss, loss2) and torch.equal(a, kept)


def test_log_probabilities_are_those_of_cross_entropy(ctx):
    z = torch.randn(50, 999, device="cuda") * 3
    t = torch.randint(0, 999, (50,), device="cuda")
    logp, _ = L.Policy(ctx).logprob(z, t)
    assert torch.allclose(logp.double(), -torch.nn.functional.cross_entropy(z.double(), t, reduction="none"), rtol=0, atol=2e-5)
    loss, _ = L.Distillation(ctx).forward(z, torch.zeros(50, 1, device="cuda"), t[:, None])
    assert torch.allclose(loss, -logp, rtol=0, atol=2e-5)


def test_gradient_against_differences(ctx):
    p = L.Policy(ctx, 0.2, 0.3, 0.2, 2.0)
    z, tokens, old, advantage, reference, _ = inputs(60, 50, F32, torch.int64, 7, p)
    one = torch.ones(60, device="cuda")
    u = torch.randn(z.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    g = p.step(z, tokens, old, advantage, one, reference)[3]

    def slope(h):
        return (p.forward(z + h * u, tokens, old, advantage, reference)[0].double()
                - p.forward(z - h * u, tokens, old, advantage, reference)[0].double()) / (2 * h)

    h = 2.0 ** -6
    near = lambda h: p.logprob(z + h * u, tokens)[0] - old  # noqa: E731
    same = torch.ones(60, device="cuda", dtype=torch.bool)           # rows that cross no border on the way
    for border in (math.log(0.8), math.log(1.3)):
        same &= (near(-2 * h) > border) == (near(2 * h) > border)
    want = (g.double() * u.double()).sum(1)
    a, b = slope(h), slope(2 * h)
    # truncation: a third of the difference of the slopes to leading order; rounding: a loss of size 3 is off by 2^-18, over h
    assert int(same.sum()) > 40 and bool(((a - want).abs() <= (a - b).abs() + 2.0 ** -18 / h)[same].all())


def test_streams_and_graphs(ctx):
    p = L.Policy(ctx, kl=0.1)
    z, tokens, old, advantage, reference, gl = inputs(40, 1003, BF16, torch.int64, 8, p)

    def f(stream=None):
        loss, logp, lse = p.forward(z, tokens, old, advantage, reference, stream=stream)
        return (loss, logp, lse, p.backward(z, tokens, lse, old, advantage, gl, reference, stream=stream),
                *p.step(z, tokens, old, advantage, gl, reference, stream=stream))

    want = f()
    torch.cuda.synchronize()
    both = [f(s) for s in [torch.cuda.Stream() for _ in range(2)] for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in both for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = f()
    for _ in range(2):
        z.normal_()
        tokens.copy_(torch.randint_like(tokens, -1, 1003))
        gl.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, f()))
    ctx.stats()


def test_rows_past_32_bits(ctx):
    """Logits of more than 2^32 elements: rows of 1000 of a batch 2^32 elements apart."""
    store = torch.empty((1 << 32) + 2048, device="cuda", dtype=BF16)
    p = L.Policy(ctx, kl=0.1)
    z, tokens, old, advantage, reference, gl = inputs(2, 1000, BF16, torch.int64, 9, p)
    wide = store.as_strided((2, 1000), (1 << 32, 1))
    wide.copy_(z)
    want = p.step(z, tokens, old, advantage, gl, reference)
    assert all(torch.equal(a, b) for a, b in zip(want, p.step(wide, tokens, old, advantage, gl, reference, grad=wide)))


def test_refusals(ctx):
    p = L.Policy(ctx, kl=0.1)
    z, tokens, old, advantage, reference, gl = inputs(4, 300, F32, torch.int64, 10, p)
    for bad in (lambda: L.Policy(ctx, -0.1), lambda: L.Policy(ctx, 0.1, math.inf), lambda: L.Policy(ctx, kl=-1.0),
                lambda: L.Policy(ctx, kl=math.nan), lambda: L.Policy(ctx, temperature=0.0),
                lambda: p.forward(z, tokens, old, advantage), lambda: p.forward(z, tokens, None, advantage, reference),
                lambda: p.step(z, tokens, old, None, gl, reference), lambda: p.forward(z, tokens[:3], old, advantage, reference),
                lambda: p.forward(z, tokens, old[:3], advantage, reference), lambda: p.forward(z, tokens, old, advantage.double(), reference),
                lambda: p.forward(z.t(), tokens, old, advantage, reference), lambda: p.logprob(z, tokens.cpu()),
                lambda: p.logprob(z, torch.stack([tokens, tokens], 1)[:, 0]),
                lambda: p.step(z, tokens, old, advantage, gl.cpu(), reference),
                lambda: p.step(z, tokens, old, advantage, gl, reference, grad=z.bfloat16())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: p.logprob(z.half(), tokens), lambda: p.logprob(z, tokens.float())):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(B.OmniError) as err:
        L.Policy(ctx, temperature=math.inf).logprob(z, tokens)
    assert err.value.status == B.ERR_BAD_CONFIG
    empty = p.step(z[:0], tokens[:0], old[:0], advantage[:0], gl[:0], reference[:0])
    assert empty[3].shape == (0, 300)
