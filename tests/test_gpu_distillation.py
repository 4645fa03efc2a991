"""Distillation loss from a teacher's top logits against a plain implementation in 64 bits.

Tolerances.  Exponents are taken in powers of two: x = z log2(e) / T, rounded to float, so an
exponential is off by X 2^-22 relative (X the largest |x| and |lse| of the row, in powers of two; two
roundings) plus 2^-21 for the hardware's 2^x; a sum over the vocabulary adds at most
(V / 128 + 16) 2^-24 relative (what one thread adds up, and the tree above it).  Their sum is `e` below:
  |lse error| <= e + 2^-23 |lse|;  |loss error| <= T^2 (e + 2^-20 (X + 16));
  |grad error| <= |g| T (q e + p 2^-19) and the rounding of the stored type.
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


def exact(z, t, index, temp):
    """(loss, lse, q, p dense, has a target) in double."""
    z = z.double() / temp
    vocab = z.shape[1]
    there = (index >= 0) & (index < vocab)
    t = torch.where(there, t.double() / temp, -math.inf)
    target = (t > -math.inf).any(1) | t.isnan().any(1)
    p = torch.where(target[:, None], torch.softmax(t, 1), 0.0)
    at = index.long().clamp(0, vocab - 1)
    lse = torch.logsumexp(z, 1)
    loss = temp * temp * torch.where(p > 0, p * (p.log() - z.gather(1, at) + lse[:, None]), 0.0).sum(1)
    dense = torch.zeros_like(z).scatter_add_(1, at, torch.where(there, p, 0.0))
    return loss, lse, torch.exp(z - lse[:, None]), dense, target


def check(ctx, z, t, index, temp, gl, grad=None):
    d = L.Distillation(ctx, temp)
    loss, lse = d.forward(z, t, index)
    g1 = d.backward(z, t, index, lse, gl)
    loss2, lse2, g2 = d.step(z, t, index, gl, grad=grad)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    wl, ws, q, p, target = exact(z, t, index, temp)
    vocab = z.shape[1]
    x = (z.double() / temp).nan_to_num(neginf=0.0).abs().amax(1)
    x = torch.maximum(x, ws.abs()) / math.log(2)
    e = x * 2.0 ** -22 + 2.0 ** -21 + (vocab / 128 + 16) * 2.0 ** -24
    assert bool(((lse.double() - ws).abs() <= e + 2.0 ** -23 * ws.abs()).all())
    assert bool(((loss.double() - wl).abs() <= temp * temp * (e + 2.0 ** -20 * (x + 16))).all())
    gain = (gl.double() * temp * target)[:, None]
    want = gain * (q - p)
    # the backward call starts from the rounded lse: 2^-24 |lse| more
    bound = gain.abs() * (q * 2 * e[:, None] + p * 2.0 ** -19) + ROUND[z.dtype] * want.abs() + 1e-38
    for g in (g1, g2):
        assert g.dtype == z.dtype
        err = (g.double() - want).abs()
        assert bool((err <= bound).all()), float((err - bound).max())


def inputs(rows, vocab, top, dtype, index, seed, temp=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn(rows, vocab, device="cuda", generator=gen) * 3).to(dtype)
    t, i = torch.topk(z.float() + torch.randn(rows, vocab, device="cuda", generator=gen), top, dim=1)
    gl = torch.randn(rows, device="cuda", generator=gen)
    return z, t, i.to(index), gl


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,top,index,temp", [
    (1, 1, 1, torch.int64, 1.0), (3, 7, 2, torch.int32, 2.0), (5, 16, 16, torch.int64, 1.0), (4, 100, 5, torch.int32, 4.0),
    (33, 1000, 64, torch.int64, 1.0), (9, 5003, 256, torch.int32, 2.0), (7, 50257, 33, torch.int64, 0.5),
    (2, 131075, 100, torch.int32, 1.0), (1, 300007, 8, torch.int64, 1.0), (2, 1000003, 8, torch.int64, 1.0), (200, 131072, 4, torch.int32, 1.0), (600, 2049, 3, torch.int32, 1.0),
])
def test_against_64_bits(ctx, dtype, rows, vocab, top, index, temp):
    check(ctx, *inputs(rows, vocab, top, dtype, index, rows + vocab)[:3], temp,
          inputs(rows, vocab, top, dtype, index, rows + vocab)[3])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_entries_that_are_not_there(ctx, dtype):
    z, t, i, gl = inputs(6, 777, 9, dtype, torch.int64, 1)
    i[0] = -1                      # no entry at all
    i[1, 3:] = -1                  # some
    i[2, 0] = 777                  # outside on the other side
    t[3, 4:] = -math.inf           # there, with no probability
    t[4] = -math.inf               # all without: no target
    check(ctx, z, t, i, 2.0, gl)
    loss, _, grad = L.Distillation(ctx, 2.0).step(z, t, i, gl)
    for r in (0, 4):
        assert float(loss[r]) == 0.0 and not bool(grad[r].any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_vocabulary_and_repeated_entries(ctx, dtype):
    z, t, i, gl = inputs(5, 3001, 12, dtype, torch.int32, 2)
    i = i.clamp(max=2899)
    z[:, 2900:] = -math.inf
    z[0, 8:2000] = torch.finfo(dtype).min   # the type's lowest value: probability 0, no NaN
    i[0] = 3
    i[1, 4], i[1, 7], i[2, :] = i[1, 2], i[1, 2], 17
    z[3, :2800] = -math.inf                 # whole stretches of threads see nothing
    i[3] = 2850
    check(ctx, z, t, i, 1.0, gl)


def test_infinite_and_not_a_number(ctx):
    z, t, i, gl = inputs(4, 640, 4, F32, torch.int64, 3)
    z[0, i[0, 0]] = -math.inf               # the teacher wants what the student rules out
    z[1, 77] = math.nan
    t[2, 1] = math.nan
    loss, lse, grad = L.Distillation(ctx).step(z, t, i, gl)
    assert math.isinf(loss[0]) and bool(grad[0].isfinite().all())
    assert math.isnan(lse[1]) and math.isnan(loss[1]) and math.isnan(loss[2]) and bool(grad[2][i[2]].isnan().all())
    assert bool(grad[3].isfinite().all()) and math.isfinite(loss[3])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift,stride,gshift,gstride", [(0, 1008, 0, 1008), (1, 1003, 1, 1003), (3, 1001, 0, 1000), (0, 1024, 5, 1001)])
def test_strides_and_alignment(ctx, dtype, shift, stride, gshift, gstride):
    z, t, i, gl = inputs(6, 1000, 10, dtype, torch.int64, 4)
    raw = torch.zeros(shift + 6 * stride, device="cuda", dtype=dtype)
    zs = raw[shift:].as_strided((6, 1000), (stride, 1), shift)
    zs.copy_(z)
    store = torch.full((gshift + 6 * gstride + 9,), 5.0, device="cuda", dtype=dtype)
    gs = store.as_strided((6, 1000), (gstride, 1), gshift)
    check(ctx, zs, t, i, 2.0, gl, grad=gs)
    untouched = torch.ones_like(store, dtype=torch.bool)
    untouched.as_strided((6, 1000), (gstride, 1), gshift).fill_(False)
    assert bool((store[untouched] == 5.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [1000, 50257, 131075])
def test_gradient_in_place(ctx, dtype, vocab):
    z, t, i, gl = inputs(5, vocab, 7, dtype, torch.int64, 5)
    d = L.Distillation(ctx, 2.0)
    loss, lse, want = d.step(z, t, i, gl)
    a, b = z.clone(), z.clone()
    d.backward(a, t, i, lse, gl, grad=a)
    loss2, _, _ = d.step(b, t, i, gl, grad=b)
    assert torch.equal(b, want) and torch.equal(loss, loss2)
    assert torch.equal(a, d.backward(z, t, i, lse, gl))


def test_cross_entropy_is_the_case_of_one_entry(ctx):
    z, _, _, _ = inputs(50, 999, 1, F32, torch.int64, 6)
    label = torch.randint(0, 999, (50, 1), device="cuda")
    loss, _ = L.Distillation(ctx).forward(z, torch.zeros(50, 1, device="cuda"), label)
    want = torch.nn.functional.cross_entropy(z.double(), label[:, 0], reduction="none")
    assert torch.allclose(loss.double(), want, rtol=0, atol=2e-5)


def test_gradient_against_differences(ctx):
    z, t, i, _ = inputs(4, 50, 6, F32, torch.int64, 7)
    d = L.Distillation(ctx, 2.0)
    u = torch.randn_like(z)
    _, _, g = d.step(z, t, i, torch.ones(4, device="cuda"))
    h = 2.0 ** -5
    slope = (d.forward(z + h * u, t, i)[0].double() - d.forward(z - h * u, t, i)[0].double()) / (2 * h)
    want = (g.double() * u.double()).sum(1)
    # truncation: h^2 / 6 of the third derivative, at most T^2 (|u| / T)^3 with |u| < 4; rounding: loss error / h
    assert bool(((slope - want).abs() <= h * h / 6 * 4 * 8 + 4 * 2.0 ** -17 / h).all())


def test_refusals(ctx):
    z, t, i, gl = inputs(4, 300, 5, F32, torch.int64, 8)
    d = L.Distillation(ctx)
    lse = torch.zeros(4, device="cuda")
    for bad in (lambda: d.forward(z, t[:3], i[:3]), lambda: d.forward(z, t, i[:, :4]), lambda: d.forward(z.t(), t, i),
                lambda: d.backward(z, t, i, lse[:3], gl), lambda: d.backward(z, t, i, lse, gl.double()),
                lambda: d.step(z, t, i, gl, grad=z.bfloat16()), lambda: d.step(z, t, i, gl.cpu()),
                lambda: L.Distillation(ctx, 0.0)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: d.forward(z.half(), t, i), lambda: d.forward(z, t.double(), i), lambda: d.forward(z, t, i.float())):
        with pytest.raises(TypeError):
            bad()
    many = torch.zeros(4, 257, device="cuda")
    with pytest.raises(B.OmniError) as err:
        d.forward(z, many, many.long())
    assert err.value.status == B.ERR_TOO_LARGE
    with pytest.raises(B.OmniError) as err:
        L.Distillation(ctx, math.inf).forward(z, t, i)
    assert err.value.status == B.ERR_BAD_CONFIG
    empty = d.step(z[:0], t[:0], i[:0], gl[:0])
    assert empty[2].shape == (0, 300)
