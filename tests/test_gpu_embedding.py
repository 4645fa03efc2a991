"""Embedding lookup and its gradient against a plain implementation in 64 bits.

Tolerances: a lookup is one product rounded to float (relative 2^-24) and, for bfloat16, once more
(2^-8).  A gradient row is a sum of m float terms, each rounded at most once per addition, times the
scale: |error| <= (m + 3) 2^-24 * scale * sum |terms|, then the rounding of the stored type; with
accumulate the old value takes part in the last addition.
"""
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


def tokens_of(n, vocab, kind, index, gen):
    if kind == "uniform":
        t = torch.randint(0, vocab, (n,), device="cuda", generator=gen)
    elif kind == "one":                       # every token the same: one run through all blocks
        t = torch.full((n,), vocab // 2, device="cuda")
    elif kind == "zipf":
        t = ((vocab + 1.0) ** torch.rand(n, device="cuda", generator=gen) - 1).long().clamp_(0, vocab - 1)
    else:                                     # outside the vocabulary on both sides
        t = torch.randint(-3, vocab + 3, (n,), device="cuda", generator=gen)
    return t.to(index)


def exact_grad(tokens, g, vocab, scale, padding):
    """(sum, sum of absolute terms, count) per row, in double."""
    t = tokens.long()
    keep = (t >= 0) & (t < vocab) & (t != padding)
    t, g = t[keep], g[keep].double() * scale
    s = torch.zeros(vocab, g.shape[1], dtype=torch.float64, device="cuda").index_add_(0, t, g)
    a = torch.zeros_like(s).index_add_(0, t, g.abs())
    return s, a, torch.bincount(t, minlength=vocab)[:, None]


def check_grad(got, tokens, g, vocab, scale, padding, old=None):
    s, a, m = exact_grad(tokens, g, vocab, scale, padding)
    if old is not None:
        s, a = s + old.double(), a + old.double().abs()
    err = (got.double() - s).abs()
    bound = (m + 3) * 2.0 ** -24 * a + ROUND[got.dtype] * s.abs()
    assert bool((err <= bound * 1.0001).all()), float((err - bound).max())


@pytest.mark.parametrize("table", [F32, BF16])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("n,vocab,dim,kind,index", [
    (1, 1, 1, "uniform", torch.int64), (1, 50, 8, "uniform", torch.int32), (33, 1000, 64, "wild", torch.int64),
    (257, 331, 99, "wild", torch.int32), (100, 2000, 768, "zipf", torch.int64), (65, 70, 1032, "uniform", torch.int32),
])
def test_lookup(ctx, table, act, n, vocab, dim, kind, index):
    gen = torch.Generator(device="cuda").manual_seed(n + vocab)
    w = torch.randn(vocab, dim, device="cuda", generator=gen).to(table)
    t = tokens_of(n, vocab, kind, index, gen)
    out = L.Embedding(ctx, vocab, dim, scale=1.7).forward(t, w, dtype=act)
    inside = (t >= 0) & (t < vocab)
    scale = float(torch.tensor(1.7, dtype=F32))
    want = w[t.long().clamp(0, vocab - 1)].double() * scale * inside[:, None]
    assert out.dtype == act and out.shape == (n, dim)
    assert bool(((out.double() - want).abs() <= ROUND[act] * want.abs() * 1.0001 + (2.0 ** -24) * want.abs()).all())


@pytest.mark.parametrize("shift,stride", [(0, 64), (1, 65), (4, 80), (0, 71)])
def test_lookup_of_strided_and_unaligned_tables(ctx, shift, stride):
    vocab, dim = 50, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    raw = torch.randn(shift + vocab * stride, device="cuda", generator=gen).to(BF16)
    w = raw[shift:shift + (vocab - 1) * stride + dim].as_strided((vocab, dim), (stride, 1))
    t = torch.randint(0, vocab, (3, 7), device="cuda", generator=gen)
    out = L.Embedding(ctx, vocab, dim).forward(t, w)
    assert out.shape == (3, 7, dim) and torch.equal(out, w[t])


@pytest.mark.parametrize("src", [F32, BF16])
@pytest.mark.parametrize("dst", [F32, BF16])
@pytest.mark.parametrize("n,vocab,dim,kind,index", [
    (1, 1, 1, "uniform", torch.int64), (0, 9, 16, "uniform", torch.int32), (31, 40, 8, "uniform", torch.int32),
    (32, 40, 8, "one", torch.int64), (33, 511, 24, "one", torch.int32), (1000, 513, 99, "wild", torch.int64),
    (5000, 1025, 40, "zipf", torch.int32), (4097, 7, 264, "uniform", torch.int64), (3000, 2000, 1, "zipf", torch.int64),
    (20000, 300, 520, "zipf", torch.int32), (40000, 30000, 64, "zipf", torch.int64), (33000, 12, 32, "one", torch.int32),
])
def test_gradient(ctx, src, dst, n, vocab, dim, kind, index):
    gen = torch.Generator(device="cuda").manual_seed(n + dim)
    t = tokens_of(n, vocab, kind, index, gen)
    g = torch.randn(n, dim, device="cuda", generator=gen).to(src)
    scale = 0.75
    padding = 3 if vocab > 3 else -1
    e = L.Embedding(ctx, vocab, dim, scale=scale, padding=padding)
    got = e.backward(t, g, dtype=dst)
    check_grad(got, t, g, vocab, scale, padding)
    assert torch.equal(got, e.backward(t, g, dtype=dst))          # the same call, the same bits
    old = torch.randn(vocab, dim, device="cuda", generator=gen).to(dst)
    acc = old.clone()
    e.backward(t, g, grad=acc, accumulate=True)
    check_grad(acc, t, g, vocab, scale, padding, old)
    named = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    inside = (t >= 0) & (t < vocab) & (t != padding)
    named[t[inside].long()] = True
    assert torch.equal(acc[~named], old[~named])                   # untouched rows keep their bits


def test_gradient_into_a_bucket_slice_with_unaligned_rows(ctx):
    vocab, dim, n = 37, 24, 400
    gen = torch.Generator(device="cuda").manual_seed(5)
    t = torch.randint(0, vocab, (n,), device="cuda", generator=gen)
    wide = torch.randn(n, 3 * dim + 1, device="cuda", generator=gen).to(BF16)
    g = wide[:, 1:1 + dim]                                         # rows start on 2-byte boundaries
    bucket = torch.full((vocab * dim + 10,), 7.0, device="cuda")
    grad = bucket[5:5 + vocab * dim].view(vocab, dim)
    L.Embedding(ctx, vocab, dim).backward(t, g, grad=grad)
    check_grad(grad, t, g, vocab, 1.0, -1)
    assert bool((bucket[:5] == 7.0).all()) and bool((bucket[-5:] == 7.0).all())


def test_gradient_keeps_infinities_and_nan_in_their_rows(ctx):
    t = torch.tensor([1, 2, 1, 3, 0], device="cuda")
    g = torch.ones(5, 8, device="cuda")
    g[1], g[3], g[4] = float("inf"), float("nan"), float("nan")
    got = L.Embedding(ctx, 6, 8, padding=0).backward(t, g)
    assert torch.equal(got[0], torch.zeros(8, device="cuda")) and bool((got[1] == 2).all())
    assert bool(torch.isposinf(got[2]).all()) and bool(torch.isnan(got[3]).all())
    assert bool((got[4:] == 0).all())


def test_gradient_against_differences(ctx):
    """d/dW of <lookup(W), c> along a direction, by a central difference of the float lookup."""
    vocab, dim, n = 20, 16, 64
    gen = torch.Generator(device="cuda").manual_seed(9)
    w, u = torch.randn(2, vocab, dim, device="cuda", generator=gen)
    t = torch.randint(0, vocab, (n,), device="cuda", generator=gen)
    c = torch.randn(n, dim, device="cuda", generator=gen)
    e = L.Embedding(ctx, vocab, dim, scale=2.0)
    f = lambda x: float((e.forward(t, x).double() * c.double()).sum())  # noqa: E731
    h = 2.0 ** -4                                                  # the lookup is linear: no truncation error
    slope = (f(w + h * u) - f(w - h * u)) / (2 * h)
    want = float((e.backward(t, c).double() * u.double()).sum())
    # w +- h u is rounded to float (|w| < 8: 2^-22), and the products: n dim terms of size 2 |c|, over 2 h
    assert abs(slope - want) <= n * dim * 2 * 4 * 2.0 ** -21 / (2 * h)


def test_on_another_stream(ctx):
    s = torch.cuda.Stream()
    t = torch.randint(0, 500, (3000,), device="cuda")
    g = torch.randn(3000, 64, device="cuda")
    e = L.Embedding(ctx, 500, 64)
    here = e.backward(t, g)
    s.wait_stream(torch.cuda.current_stream())
    there = e.backward(t, g, stream=s)
    with torch.cuda.stream(s):
        again = e.backward(t, g)
    s.synchronize()
    assert torch.equal(here, there) and torch.equal(here, again)


def test_refusals(ctx):
    e = L.Embedding(ctx, 10, 8)
    t, w = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(10, 8, device="cuda")
    with pytest.raises(TypeError):
        e.forward(t.float(), w)
    with pytest.raises(TypeError):
        e.forward(t, w.half())
    with pytest.raises(ValueError):
        e.forward(t, w[:, :4])
    with pytest.raises(ValueError):
        e.forward(t, w.cpu())
    with pytest.raises(ValueError):
        e.forward(torch.zeros(4, 2, dtype=torch.int64, device="cuda")[:, 0], w)
    with pytest.raises(ValueError):
        e.backward(t, torch.zeros(3, 8, device="cuda"))
    with pytest.raises(ValueError):
        e.backward(t, torch.zeros(4, 8, device="cuda"), accumulate=True)
    with pytest.raises(ValueError):
        L.Embedding(ctx, 0, 8)
    with pytest.raises(B.OmniError) as err:
        L.Embedding(ctx, 10, 8, scale=float("nan")).forward(t, w)
    assert err.value.status == B.ERR_BAD_CONFIG
