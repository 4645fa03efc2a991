"""Norms of query and key heads with the rotation by positions against a plain implementation in 64 bits.

Tolerances.  e = 2^-24.  The mean of squares is a sum of dim positive terms in float, by chains of at most 16 and a tree of five: off
by (16 + 5 + 2) e of itself, its root by half of that and 3 e more: 15 e.  Weighing costs 3 e, cosine and sine are off by 2 e
plus the angle's own 2 pi 2^-51 of its turns and 2^-23 for the remainder in float, a pair's sum by 2 e: a result is off by at most
26 e (|n_a| + |n_b|), which `E` rounds up to 32, and half a step of the stored type.  In the gradient two such sums are
subtracted: their terms' sizes are added up.  A weight's gradient is a sum over rows and heads, by chains of at most
`rows * heads / 64 + 32` terms and a tree.
"""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
E = 32 * 2.0 ** -24
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


def turn(x, angle, pairs, interleaved):
    """x [b, n, h, d] in double, angle [b, n, pairs]; also the sizes |a| + |b| of each element's terms."""
    c, s = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    y, size = x.clone(), x.abs()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def angles(r, positions, axes):
    p = positions if positions.dim() == 3 else positions[None]
    axis = torch.tensor(axes or [0] * len(r.frequencies), device="cuda")
    return p.permute(1, 2, 0)[:, :, axis].double() * torch.tensor(r.frequencies, device="cuda", dtype=torch.float64)


def close(got, want, size):
    """`size`: what E is relative to."""
    bound = E * size + HALF[got.dtype] * want.abs() * 1.001 + 1e-37
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), float((err - bound).max())


def check(ctx, q, k, positions, weights, r, axes=None, lengths=None, seed=0):
    interleaved, eps = r.interleaved, r.eps
    b, n = q.shape[:2]
    pairs = len(r.frequencies)
    angle = angles(r, positions, axes)
    there = torch.ones(b, n, 1, 1, device="cuda", dtype=torch.bool)
    if lengths is not None:
        there = (torch.arange(n, device="cuda")[None] < lengths[:, None])[:, :, None, None]
    gen = torch.Generator(device="cuda").manual_seed(seed + 100)
    grads = [torch.randn(x.shape, device="cuda", generator=gen).to(x.dtype) for x in (q, k)]
    got = r.forward(q, k, positions, *weights, lengths=lengths)
    back = r.backward(q, k, positions, *grads, *weights, lengths=lengths)
    for x, w, dy, y, dx, dw in zip((q, k), weights, grads, got, back[:2], back[2:]):
        assert y.dtype == dx.dtype == x.dtype and y.shape == dx.shape == x.shape
        x, g = (torch.where(there, t.double(), 0.0) for t in (x, dy))
        scale = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) if w is not None else torch.ones_like(x[..., :1])
        weight = w.double() if w is not None else 1.0
        want, size = turn(torch.where(there, x * scale * weight, 0.0), angle, pairs, interleaved)
        close(y, want, size)
        dn, size = turn(g, -angle, pairs, interleaved)
        if w is None:
            assert dw is None
            close(dx, dn, size)
            continue
        unit = torch.where(there, x * scale, 0.0)
        want = scale * (dn * weight - unit * (dn * weight * unit).mean(-1, keepdim=True))
        size = scale * (size * abs(weight) + 2 * unit.abs() * (size * abs(weight) * unit.abs()).mean(-1, keepdim=True))
        close(dx, torch.where(there, want, 0.0), torch.where(there, size, 0.0))
        assert dw.dtype == F32 and dw.shape == w.shape
        terms = dn * unit
        chain = x.shape[0] * x.shape[1] * x.shape[2] / 64 + 64
        err = (dw.double() - terms.sum((0, 1, 2))).abs()
        bound = (E + chain * 2.0 ** -24) * terms.abs().sum((0, 1, 2)) + E * (turn(g, -angle, pairs, interleaved)[1] * unit.abs()).sum((0, 1, 2)) + 1e-37
        assert bool((err <= bound).all()), float((err - bound).max())


def inputs(b, n, h, hk, d, dtype, seed, weight=None, axes=1, far=1000):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    packed = (torch.randn(b, n, h + 2 * hk, d, device="cuda", generator=gen) * 2).to(dtype)
    positions = torch.randint(0, far, (axes, b, n), device="cuda", generator=gen)
    weights = (None, None)
    if weight is not None:
        weights = tuple((1 + 0.3 * torch.randn(d, device="cuda", generator=gen)).to(weight) for _ in range(2))
    return packed[:, :, :h], packed[:, :, h:h + hk], positions, weights


SHAPES = [  # batch, length, heads, kv_heads, dim, pairs
    (1, 1, 1, 1, 2, 1), (3, 1, 16, 4, 128, 64), (2, 5, 3, 1, 64, 32), (1, 77, 7, 7, 80, 40), (2, 33, 12, 4, 96, 24), (1, 19, 2, 1, 256, 128),
    (1, 700, 40, 8, 128, 64), (5, 301, 4, 2, 48, 8), (2, 45, 9, 3, 64, 9), (3, 130, 6, 6, 96, 12), (1, 260, 2, 1, 256, 100), (2, 7, 5, 5, 16, 3), (1, 3, 33, 5, 250, 125), (2, 130, 3, 1, 34, 11), (1, 5000, 2, 1, 16, 8), (1, 6000, 1, 1, 6, 2),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,weight", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, None), (BF16, None)])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_64_bits(ctx, shape, dtype, weight, interleaved):
    b, n, h, hk, d, pairs = shape
    q, k, positions, weights = inputs(b, n, h, hk, d, dtype, sum(shape), weight)
    check(ctx, q, k, positions, weights, L.Rotary(ctx, h, hk, d, L.Rotary.geometric(pairs), interleaved=interleaved))


@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_several_axes(ctx, dtype, index):
    axes = [0, 1, 2] * 5 + [3] * 5
    q, k, positions, weights = inputs(2, 45, 6, 2, 64, dtype, 1, dtype, axes=4)
    for interleaved in (False, True):
        check(ctx, q, k, positions.to(index), weights, L.Rotary(ctx, 6, 2, 64, L.Rotary.geometric(20), axes, interleaved), axes)


def test_far_and_negative_positions(ctx):
    """Angles of 2^31 radians and more: a table in float would lose the phase altogether."""
    q, k, positions, weights = inputs(1, 64, 2, 1, 64, F32, 2, F32)
    r = L.Rotary(ctx, 2, 1, 64, L.Rotary.geometric(32))
    for offset in (131072, 2 ** 24 + 1, 2 ** 31 - 2000, -(2 ** 31), -5):
        check(ctx, q, k, positions + offset, weights, r)
    # 2^40 radians keep 2^-11 of a radian in 64 bits, here as in the plain form
    got, want = r.forward(q, k, positions + 2 ** 40)[0], turn(q.double(), angles(r, positions + 2 ** 40, None), 32, False)[0]
    assert float((got - want).abs().max()) <= 4 * 2.0 ** -11 * float(q.abs().max())


@pytest.mark.parametrize("weight", [None, F32])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,pairs", [(64, 32), (50, 20)])
def test_lengths_and_what_stands_behind_them(ctx, dtype, weight, d, pairs):
    q, k, positions, weights = inputs(4, 37, 6, 2, d, dtype, 3, weight)
    lengths = torch.tensor([37, 0, 1, 20], device="cuda", dtype=torch.int32)
    r = L.Rotary(ctx, 6, 2, d, L.Rotary.geometric(pairs))
    check(ctx, q, k, positions, weights, r, lengths=lengths)
    clean = r.forward(q, k, positions, *weights, lengths=lengths)
    gq, gk = torch.randn_like(clean[0]), torch.randn_like(clean[1])
    clean_grads = r.backward(q, k, positions, gq, gk, *weights, lengths=lengths)
    behind = torch.arange(37, device="cuda")[None] >= lengths[:, None]
    for t in (q, k, gq, gk):
        t[behind] = math.nan
    dirty = r.forward(q, k, positions, *weights, lengths=lengths), r.backward(q, k, positions, gq, gk, *weights, lengths=lengths)
    for a, b in zip((*clean, *clean_grads), (*dirty[0], *dirty[1])):
        assert (a is None and b is None) or torch.equal(a, b)
    assert not bool(dirty[0][0][behind].any()) and not bool(dirty[1][1][behind].any())
    far = torch.tensor([99, -3, 1, 20], device="cuda", dtype=torch.int32)       # clamped
    assert torch.equal(r.forward(q, k, positions, *weights, lengths=far)[1], clean[1])
    for a, b in zip(clean_grads, r.backward(q, k, positions, gq, gk, *weights, lengths=far)):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,n,d,pairs,kind", [
    (1000, 5, 64, 32, "any"), (1024, 3, 48, 5, "any"), (1025, 3, 48, 24, "any"), (70, 40, 42, 9, "any"), (33, 300, 128, 64, "empty but one"),
    (33, 300, 128, 64, "empty"), (2000, 7, 30, 15, "empty"), (64, 50, 32, 16, "full"), (5, 1500, 16, 8, "any"),
])
def test_padded_batches(ctx, dtype, b, n, d, pairs, kind):
    """Many sequences, most of them short or empty: the backward pass walks the rows that are there alone."""
    q, k, positions, weights = inputs(b, n, 5, 2, d, dtype, b + n, F32)
    gen = torch.Generator(device="cuda").manual_seed(b)
    lengths = torch.randint(-1, n + 2, (b,), device="cuda", generator=gen).int()
    if kind != "any":
        lengths.fill_(n if kind == "full" else 0)
    if kind == "empty but one":
        lengths[17] = 1
    r = L.Rotary(ctx, 5, 2, d, L.Rotary.geometric(pairs))
    check(ctx, q, k, positions, weights, r, lengths=lengths.clamp(0, n))
    behind = torch.arange(n, device="cuda")[None] >= lengths[:, None]
    q[behind], k[behind] = math.nan, math.inf
    grads = [torch.full_like(x, 3.0) for x in (q, k)]
    out = r.backward(q, k, positions, q, k, *weights, lengths=lengths, grads=grads)
    assert all(bool(x.isfinite().all()) for x in out)
    assert not bool(grads[0][behind].any()) and not bool(grads[1][behind].any())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift,row,head", [(0, 0, 0), (1, 0, 0), (0, 3, 0), (0, 0, 1), (4, 8, 4)])
def test_strides_alignment_and_places_in_a_cache(ctx, dtype, shift, row, head):
    b, n, h, hk, d = 2, 9, 4, 2, 32
    q, k, positions, weights = inputs(b, n, h, hk, d, dtype, 4, dtype)
    r = L.Rotary(ctx, h, hk, d, L.Rotary.geometric(16))
    want = r.forward(q, k, positions, *weights)

    def odd(heads):
        strides = (n * (heads * (d + head) + row), heads * (d + head) + row, d + head, 1)
        store = torch.full((shift + b * strides[0] + 64,), 5.0, device="cuda", dtype=dtype)
        return store, store.as_strided((b, n, heads, d), strides, shift)

    (store_q, out_q), (store_k, out_k), (_, in_q), (_, in_k) = odd(h), odd(hk), odd(h), odd(hk)
    in_q.copy_(q)
    in_k.copy_(k)
    assert r.forward(in_q, in_k, positions, *weights, out=(out_q, out_k))[0] is out_q
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    grads = r.backward(q, k, positions, gq, gk, *weights)
    odd_grads = r.backward(in_q, in_k, positions, gq, gk, *weights)
    if shift == row == head == 0:
        assert torch.equal(out_q, want[0]) and torch.equal(out_k, want[1])
        assert all(torch.equal(x, y) for x, y in zip(grads, odd_grads))
    check(ctx, in_q, in_k, positions, weights, r)
    for store, out in ((store_q, out_q), (store_k, out_k)):
        untouched = torch.ones_like(store, dtype=torch.bool)
        untouched.as_strided(out.shape, out.stride(), shift).fill_(False)
        assert bool((store[untouched] == 5.0).all())
    # one step of a cache whose rows are far apart
    cache = torch.zeros(b, 20, hk, d, device="cuda", dtype=dtype)
    one = r.forward(q[:, :1], k[:, :1], positions[:, :, :1], *weights, out=(torch.empty_like(q[:, :1]), cache[:, 7:8]))
    assert torch.equal(cache[:, 7], r.forward(q[:, :1], k[:, :1], positions[:, :, :1], *weights)[1][:, 0]) and not bool(cache[:, 8:].any())
    assert one[1].data_ptr() == cache[:, 7:8].data_ptr()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("weight", [None, F32])
@pytest.mark.parametrize("d,pairs", [(64, 32), (42, 21), (64, 13), (128, 20), (256, 100)])
def test_in_place(ctx, dtype, weight, d, pairs):
    q, k, positions, weights = inputs(2, 50, 4, 2, d, dtype, 5, weight)
    r = L.Rotary(ctx, 4, 2, d, L.Rotary.geometric(pairs), interleaved=d == 42)
    want = r.forward(q, k, positions, *weights)
    gq, gk = torch.randn_like(want[0]), torch.randn_like(want[1])
    want_grads = r.backward(q, k, positions, gq, gk, *weights)
    got = r.backward(q, k, positions, gq, gk, *weights, grads=(gq, gk))
    assert got[0] is gq and all(a is None or torch.equal(a, b) for a, b in zip(got, want_grads))
    r.forward(q, k, positions, *weights, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_positions_of_any_strides(ctx):
    q, k, positions, weights = inputs(3, 20, 4, 2, 64, BF16, 6, F32)
    r = L.Rotary(ctx, 4, 2, 64, L.Rotary.geometric(32))
    shared = torch.arange(20, device="cuda")[None].expand(3, -1)
    assert torch.equal(r.forward(q, k, shared, *weights)[0], r.forward(q, k, shared.contiguous()[None].int(), *weights)[0])
    across = positions[0].t().contiguous().t()
    assert torch.equal(r.forward(q, k, across, *weights)[1], r.forward(q, k, positions, *weights)[1])
    every_other = torch.stack([positions, positions * 0], -1)[..., 0]
    assert torch.equal(r.forward(q, k, every_other, *weights)[1], r.forward(q, k, positions, *weights)[1])


def test_rows_past_32_bits(ctx):
    """A cache whose rows lie more than 2^32 elements apart."""
    store = torch.empty((1 << 32) + 4096, device="cuda", dtype=BF16)
    q, k, positions, weights = inputs(2, 1, 2, 2, 64, BF16, 7, BF16)
    wide = store.as_strided((2, 1, 2, 64), (1 << 32, 128, 64, 1))
    wide.copy_(k)
    r = L.Rotary(ctx, 2, 2, 64, L.Rotary.geometric(32))
    want, grads = r.forward(q, k, positions, *weights), r.backward(q, k, positions, k, k, *weights)
    assert all(torch.equal(a, b) for a, b in zip(grads, r.backward(q, wide, positions, k, wide, *weights)))
    r.forward(q, wide, positions, *weights, out=(q.clone(), wide))
    assert torch.equal(wide, want[1])


@pytest.mark.parametrize("weight", [None, F32])
def test_nothing(ctx, weight):
    r = L.Rotary(ctx, 4, 2, 64, L.Rotary.geometric(32))
    for b, n in ((0, 5), (3, 0)):
        q, k, positions, weights = inputs(b, n, 4, 2, 64, BF16, 8, weight)
        assert r.forward(q, k, positions, *weights)[0].shape == (b, n, 4, 64)
        dw = r.backward(q, k, positions, q, k, *weights)[2:]
        assert all(x is None or not bool(x.any()) for x in dw)
    ctx.stats()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,pairs", [(64, 32), (30, 10)])
def test_extreme_values(ctx, dtype, d, pairs):
    """Rows of zeros are zeros (eps keeps the norm finite), large rows keep unit size, NaN stays in its head."""
    q, k, positions, weights = inputs(1, 6, 4, 4, d, dtype, 9, F32)
    q[0, 0] = 0.0
    q[0, 1] *= 1e15
    q[0, 2] *= 1e-15
    check(ctx, q, k, positions, weights, L.Rotary(ctx, 4, 4, d, L.Rotary.geometric(pairs)))
    q[0, 3, 1, 5] = math.nan
    out, _ = L.Rotary(ctx, 4, 4, d, L.Rotary.geometric(pairs)).forward(q, k, positions, *weights)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, 3, 1] = True
    assert torch.equal(out.isnan(), bad) and not bool(out[0, 0].any())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,pairs", [(64, 8), (64, 5), (96, 12), (50, 7), (128, 60)])
def test_what_is_not_turned_stays_as_it_is(ctx, dtype, interleaved, d, pairs):
    """Elements behind the pairs pass through, infinities and NaN beside them too."""
    q, k, positions, _ = inputs(2, 9, 3, 3, d, dtype, 13)
    r = L.Rotary(ctx, 3, 3, d, L.Rotary.geometric(pairs), interleaved=interleaved)
    clean = r.forward(q, k, positions)[0]
    q[0, 1, 2, 2 * pairs + 1], q[1, 3, 0, d - 1], q[1, 4, 1, 2 * pairs] = math.nan, math.inf, -math.inf
    out, _ = r.forward(q, k, positions)
    back = r.backward(q, k, positions, q, k)[0]
    assert torch.equal(out[..., :2 * pairs], clean[..., :2 * pairs])
    for t in (out, back):
        assert torch.equal(t[..., 2 * pairs:].nan_to_num(7.0), q[..., 2 * pairs:].nan_to_num(7.0)) and int(t.isnan().sum()) == 1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shift", [0, 1, 2, 4])
@pytest.mark.parametrize("d,pairs", [(84, 42), (82, 41), (82, 40), (128, 20), (20, 10), (36, 18), (36, 4), (250, 123), (252, 126), (256, 126), (256, 127), (4, 1),
                                     (8, 4), (66, 1)])
def test_accesses_of_every_width(ctx, dtype, interleaved, shift, d, pairs):
    """Heads whose size, halves and boundaries allow 16, 8, 4 or 2 bytes at a time, among storage that stays as it is."""
    b, n, h, hk = 3, 41, 3, 2
    axes = [i % 2 for i in range(pairs)]
    r = L.Rotary(ctx, h, hk, d, L.Rotary.geometric(pairs), axes=axes, interleaved=interleaved)
    q, k, positions, weights = inputs(b, n, h, hk, d, dtype, d + pairs, dtype, axes=r.axes)
    lengths = torch.tensor([n, 0, 17], device="cuda", dtype=torch.int32)

    def place(heads):
        strides = (n * heads * d + shift, heads * d, d, 1)
        store = torch.full((shift + b * strides[0] + 16,), 5.0, device="cuda", dtype=dtype)
        return store, store.as_strided((b, n, heads, d), strides, shift)

    stores, places = zip(*(place(x) for x in (h, hk, h, hk)))
    inputs_at = tuple(p.copy_(x) for p, x in zip(places[2:], (q, k)))
    for w in (weights, (None, None)):
        check(ctx, *inputs_at, positions, w, r, axes, lengths)
        out = r.forward(*inputs_at, positions, *w, lengths=lengths, out=places[:2])
        back = r.backward(*inputs_at, positions, q, k, *w, lengths=lengths)
        assert all(torch.equal(x, y) for x, y in zip(out, r.forward(*inputs_at, positions, *w, lengths=lengths)))
        same = r.backward(*inputs_at, positions, q, k, *w, lengths=lengths, grads=places[:2])
        assert all(torch.equal(x, y) for x, y in zip(back[:2], same))
    for store, at in zip(stores, places):
        untouched = torch.ones_like(store, dtype=torch.bool)
        untouched.as_strided(at.shape, at.stride(), shift).fill_(False)
        assert bool((store[untouched] == 5.0).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(ctx, interleaved):
    q, k, positions, weights = inputs(1, 4, 3, 1, 32, F32, 10, F32)
    r = L.Rotary(ctx, 3, 1, 32, L.Rotary.geometric(12), interleaved=interleaved)
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda t: torch.randn(t.shape, device="cuda", generator=gen)  # noqa: E731
    gq, gk, uq, uk, uw, vw = (rand(t) for t in (q, k, q, k, *weights))

    def value(h):
        y = r.forward(q + h * uq, k + h * uk, positions, weights[0] + h * uw, weights[1] + h * vw)
        return float((y[0].double() * gq).sum() + (y[1].double() * gk).sum())

    h = 2.0 ** -6
    grads = r.backward(q, k, positions, gq, gk, *weights)
    want = sum(float((a.double() * b).sum()) for a, b in zip(grads, (uq, uk, uw, vw)))
    slope, wider = (value(h) - value(-h)) / (2 * h), (value(2 * h) - value(-2 * h)) / (4 * h)
    # truncation is a third of the difference of the two slopes to leading order; rounding: 16 vectors of 32 of size 3, 32 e each, over h
    assert abs(slope - want) <= abs(slope - wider) + 16 * 32 * 9 * E / h


def test_same_bits_on_streams_in_graphs_and_contexts(ctx):
    q, k, positions, weights = inputs(3, 600, 16, 4, 128, BF16, 11, BF16)
    r = L.Rotary(ctx, 16, 4, 128, L.Rotary.geometric(64))
    gq, gk = torch.randn_like(q), torch.randn_like(k)

    def f(rotary=r, stream=None):
        return (*rotary.forward(q, k, positions, *weights, stream=stream), *rotary.backward(q, k, positions, gq, gk, *weights, stream=stream))

    want = f()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [f(stream=s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in both for a, b in zip(got, want))
    plain = B.Omni(1, 1, 1, 1, flags=B.NO_BULK_COPY)
    assert all(torch.equal(a, b) for a, b in zip(f(L.Rotary(plain, 16, 4, 128, L.Rotary.geometric(64))), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = f()
    for seed in range(2):
        positions.copy_(torch.randint_like(positions, 5000))
        gq.normal_()
        q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, f()))


def test_refusals(ctx):
    q, k, positions, weights = inputs(2, 5, 4, 2, 64, BF16, 12, BF16)
    f = L.Rotary.geometric(32)
    r = L.Rotary(ctx, 4, 2, 64, f)
    for bad in (lambda: L.Rotary(ctx, 4, 2, 63, f), lambda: L.Rotary(ctx, 4, 2, 62, f), lambda: L.Rotary(ctx, 4, 0, 64, f),
                lambda: L.Rotary(ctx, 4, 2, 64, []), lambda: L.Rotary(ctx, 4, 2, 64, f, axes=[0]),
                lambda: L.Rotary(ctx, 4, 2, 64, f, axes=[4] * 32), lambda: L.Rotary(ctx, 4, 2, 64, f, eps=-1.0),
                lambda: r.forward(q[0], k, positions), lambda: r.forward(q[:, :, :3], k, positions),
                lambda: r.forward(q, k[:, :4], positions), lambda: r.forward(q, k, positions[:, :, :4]),
                lambda: r.forward(q, k, positions.cpu()), lambda: r.forward(q, k, positions, weights[0]),
                lambda: r.forward(q, k, positions, weights[0][:5], weights[1]),
                lambda: r.forward(q, k, positions, weights[0], weights[1].float()),
                lambda: r.forward(q, k, positions, lengths=torch.ones(2, device="cuda")),
                lambda: r.forward(q, k, positions, out=(k, k)), lambda: r.forward(q.transpose(2, 3), k, positions),
                lambda: r.backward(q, k, positions, k, k, *weights),
                lambda: r.backward(q, k, positions, q, k, *weights, weight_grads=(weights[0], weights[1].float()))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: r.forward(q.half(), k, positions), lambda: r.forward(q, k.float(), positions),
                lambda: r.forward(q, k, positions.float()), lambda: r.backward(q, k, positions, q.float(), k)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(B.OmniError) as err:
        L.Rotary(ctx, 4, 2, 258, f).forward(*(torch.zeros(1, 1, h, 258, device="cuda") for h in (4, 2)), positions[:, :1, :1])
    assert err.value.status == B.ERR_TOO_LARGE
    with pytest.raises(B.OmniError) as err:
        L.Rotary(ctx, 4, 2, 64, [math.inf]).forward(q, k, positions)
    assert err.value.status == B.ERR_BAD_CONFIG
