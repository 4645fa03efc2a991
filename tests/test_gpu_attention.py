"""Attention, forward and backward, against the formulas in 64 bits.

Tolerances, element by element.  Scores are exact products summed in float; a probability is off by
e = X 2^-21 + 2^-19 relative (X the largest |score| and |lse| in powers of two: rounding of the exponent, the
sum over dim <= 128 in float, the hardware's 2^x).  P and dS are rounded to bfloat16 (2^-8), and so is each result:
  |O error|  <= (2^-8 + 2 e) P |V|            + 2^-8 |O|
  |dV error| <= (2^-8 + e) P^T |dO|           + 2^-8 |dV|
  |dS error| <= 2^-8 |dS| + P ((e + 2^-17) (|dO| |V|^T + sum |dO O|))  =: E
  |dQ error| <= scale E |K|                   + 2^-8 |dQ|      (dK the same with E^T |Q|)
The backward pass is compared from the out and lse that it is given.
"""
import gc
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu
BF = 2.0 ** -8


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


def randn(shape, seed, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=gen) * std).bfloat16()


def allowed(q_len, kv_len, causal, ql, kl):
    i = torch.arange(q_len, device="cuda")[None, :, None]
    j = torch.arange(kv_len, device="cuda")[None, None, :]
    ql, kl = ql.long()[:, None, None], kl.long()[:, None, None]
    ok = (i < ql) & (j < kl)
    return (ok & (j <= i + kl - ql) if causal else ok)[:, None]


def first(x):
    return x.transpose(1, 2).double()


def shared(x, group):
    return first(x).repeat_interleave(group, 1)


def lens(q, k, q_lengths, kv_lengths):
    b = q.shape[0]
    full = lambda n: torch.full((b,), n, device="cuda", dtype=torch.int32)  # noqa: E731
    return (full(q.shape[1]) if q_lengths is None else q_lengths.clamp(0, q.shape[1]),
            full(k.shape[1]) if kv_lengths is None else kv_lengths.clamp(0, k.shape[1]))


def exact_forward(q, k, v, causal, scale, ql, kl):
    """(out, lse, bound of out) with heads first, in double; what stands behind the lengths is ignored."""
    group = q.shape[2] // k.shape[2]
    ok = allowed(q.shape[1], k.shape[1], causal, ql, kl)
    s = torch.where(ok, first(q).nan_to_num() @ shared(k, group).nan_to_num().transpose(2, 3) * scale, -math.inf)
    lse = torch.logsumexp(s, 3)
    p = torch.where(ok, torch.exp(s - lse[..., None].clamp(min=-1e300)), 0.0)
    vv = shared(v, group).nan_to_num()
    out = p @ vv
    x = torch.where(ok, s, 0.0).abs().amax() / math.log(2) + 8
    e = float(x) * 2.0 ** -21 + 2.0 ** -19
    return out, lse, (BF + 2 * e) * (p @ vv.abs()) + BF * out.abs(), e


def check_forward(got, lse, q, k, v, causal, scale, ql, kl):
    out, wl, bound, e = exact_forward(q, k, v, causal, scale, ql, kl)
    err = (first(got) - out).abs()
    assert bool((err <= bound * 1.001 + 1e-30).all()), float((err - bound).max())
    empty = wl == -math.inf
    assert torch.equal(lse == -math.inf, empty) and not bool(got.transpose(1, 2)[empty].any())
    assert bool(((lse.double() - wl)[~empty].abs() <= e + 2.0 ** -23 * wl[~empty].abs()).all())


def check_backward(grads, q, k, v, out, lse, do, causal, scale, ql, kl):
    group = q.shape[2] // k.shape[2]
    ok = allowed(q.shape[1], k.shape[1], causal, ql, kl) & (lse != -math.inf)[..., None]
    qq, kk, vv, dd, oo = first(q).nan_to_num(), shared(k, group).nan_to_num(), shared(v, group).nan_to_num(), first(do).nan_to_num(), first(out).nan_to_num()
    s = qq @ kk.transpose(2, 3) * scale
    p = torch.where(ok, torch.exp(s - lse.double()[..., None]), 0.0)
    x = torch.where(ok, s, 0.0).abs().amax() / math.log(2) + 8
    e = float(x) * 2.0 ** -21 + 2.0 ** -19
    dp, dpa = dd @ vv.transpose(2, 3), dd.abs() @ vv.abs().transpose(2, 3)
    ds = p * (dp - (dd * oo).sum(3, keepdim=True))
    err = BF * ds.abs() + p * (e + 2.0 ** -17) * (dpa + (dd * oo).abs().sum(3, keepdim=True))
    fold = lambda y: y.unflatten(1, (k.shape[2], group)).sum(2)  # noqa: E731
    wants = (scale * ds @ kk, fold(scale * ds.transpose(2, 3) @ qq), fold(p.transpose(2, 3) @ dd))
    bounds = (scale * err @ kk.abs(), fold(scale * err.transpose(2, 3) @ qq.abs()), fold((BF + e) * p.transpose(2, 3) @ dd.abs()))
    for name, g, w, bnd in zip(("dq", "dk", "dv"), grads, wants, bounds):
        d = (first(g) - w).abs()
        limit = bnd + BF * w.abs()
        assert bool((d <= limit * 1.001 + 1e-30).all()), (name, float((d - limit).max()))
    return wants, bounds


def run(ctx, q, k, v, do, causal, q_lengths=None, kv_lengths=None, scale=None):
    a = L.Attention(ctx, q.shape[2], k.shape[2], q.shape[3], causal=causal, scale=scale)
    ql, kl = lens(q, k, q_lengths, kv_lengths)
    out, lse = a.forward(q, k, v, q_lengths, kv_lengths)
    check_forward(out, lse, q, k, v, causal, a.scale, ql, kl)
    grads = a.backward(q, k, v, out, lse, do, q_lengths, kv_lengths)
    check_backward(grads, q, k, v, out, lse, do, causal, a.scale, ql, kl)
    again = a.backward(q, k, v, out, lse, do, q_lengths, kv_lengths)
    assert all(torch.equal(x, y) for x, y in zip(grads, again))          # the same call, the same bits
    ctx.stats()                                                          # no wait ran out
    return out, lse, grads


def tensors(batch, q_len, kv_len, heads, kv_heads, dim, seed=0):
    return (randn((batch, q_len, heads, dim), seed), randn((batch, kv_len, kv_heads, dim), seed + 1),
            randn((batch, kv_len, kv_heads, dim), seed + 2), randn((batch, q_len, heads, dim), seed + 3))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("batch,q_len,kv_len,heads,kv_heads,dim", [
    (1, 1, 1, 1, 1, 64), (2, 1, 700, 4, 2, 128), (1, 64, 64, 2, 1, 64), (1, 127, 129, 2, 2, 128), (1, 128, 128, 1, 1, 8),
    (2, 129, 127, 3, 1, 72), (1, 255, 257, 2, 2, 64), (3, 300, 300, 4, 1, 80), (1, 513, 400, 2, 1, 128), (1, 1100, 1100, 2, 2, 96),
    (1, 400, 1300, 4, 4, 16), (1, 1000, 65, 1, 1, 128), (70, 33, 33, 1, 1, 64),
    # few tiles on one side: the walk along the other is split
    (1, 5, 3000, 2, 1, 128), (2, 1, 1500, 3, 1, 64), (1, 3000, 11, 4, 1, 64), (1, 2500, 100, 2, 2, 80), (1, 300, 2600, 1, 1, 72),
])
def test_against_64_bits(ctx, batch, q_len, kv_len, heads, kv_heads, dim, causal):
    run(ctx, *tensors(batch, q_len, kv_len, heads, kv_heads, dim), causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_padded_batches_ignore_what_stands_behind_the_lengths(ctx, dim, causal):
    q, k, v, do = tensors(7, 333, 333, 4, 2, dim, 10)
    ql = torch.tensor([333, 0, 1, 64, 130, 256, 999], dtype=torch.int32, device="cuda")   # clamped to 333
    kl = torch.tensor([333, 200, 0, 65, 3, 300, -5], dtype=torch.int32, device="cuda")    # clamped to 0
    clean = run(ctx, q, k, v, do, causal, ql, kl)
    for b in range(7):
        for t, n in ((q, ql), (do, ql), (k, kl), (v, kl)):
            t[b, max(0, min(333, int(n[b]))):] = math.nan
    dirty = run(ctx, q, k, v, do, causal, ql, kl)
    for x, y in zip((clean[0], clean[1], *clean[2]), (dirty[0], dirty[1], *dirty[2])):
        assert torch.equal(x, y)


def test_large_scores_move_the_running_maximum(ctx):
    """Rows whose maximum grows from tile to tile, and scores far apart, without overflow."""
    q, k, v, do = tensors(1, 300, 700, 2, 1, 64, 20)
    k *= torch.linspace(0.1, 6, 700, device="cuda").bfloat16()[None, :, None, None]
    run(ctx, q, k, v, do, False)
    run(ctx, q * 4, k, v, do, True)
    run(ctx, q, k.flip(1).contiguous(), v, do, True, scale=0.5)


@pytest.mark.parametrize("dim", [64, 80])
def test_slices_of_a_projection_and_given_outputs(ctx, dim):
    b, n, h, hk = 2, 200, 4, 2
    packed = randn((b, n, h + 2 * hk, dim), 30)
    q, k, v = packed[:, :, :h], packed[:, :, h:h + hk], packed[:, :, h + hk:]
    do = randn((b, h, n, dim), 31).transpose(1, 2)                       # heads before rows
    a = L.Attention(ctx, h, hk, dim)
    grad = torch.full_like(packed, 9.0)
    store = torch.full((b, n, h, dim + 8), 9.0, device="cuda", dtype=torch.bfloat16)
    out, lse = a.forward(q, k, v, out=store[..., :dim])
    assert out.data_ptr() == store.data_ptr() and bool((store[..., dim:] == 9).all())
    grads = a.backward(q, k, v, out, lse, do, grads=(grad[:, :, :h], grad[:, :, h:h + hk], grad[:, :, h + hk:]))
    ql, kl = lens(q, k, None, None)
    check_forward(out, lse, q, k, v, True, a.scale, ql, kl)
    check_backward(grads, q, k, v, out, lse, do, True, a.scale, ql, kl)
    plain = a.backward(q.contiguous(), k.contiguous(), v.contiguous(), out.contiguous(), lse, do.contiguous())
    assert torch.equal(torch.cat(plain, 2), grad)


def test_a_nan_stays_with_the_rows_that_see_it(ctx):
    q, k, v, do = tensors(1, 256, 256, 1, 1, 64, 40)
    k[0, 200] = math.nan
    out, lse = L.Attention(ctx, 1, 1, 64).forward(q, k, v)
    assert bool(out[0, :128].isfinite().all()) and bool(lse[0, 0, :200].isfinite().all())
    assert bool(lse[0, 0, 200:].isnan().all()) and bool(out[0, 200:].isnan().all())


@pytest.mark.parametrize("causal", [False, True])
def test_gradient_against_differences(ctx, causal):
    """Slope of <O(x), c> along a direction, by central differences of the forward formula in 64 bits."""
    q, k, v, c = tensors(1, 40, 50, 2, 1, 64, 50)
    a = L.Attention(ctx, 2, 1, 64, causal=causal)
    out, lse = a.forward(q, k, v)
    grads = a.backward(q, k, v, out, lse, c)
    ql, kl = lens(q, k, None, None)
    _, bounds = check_backward(grads, q, k, v, out, lse, c, causal, a.scale, ql, kl)
    h = 1e-5
    for i, (g, bound) in enumerate(zip(grads, bounds)):
        u = torch.randn(g.shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(i))

        def f(sign):
            x = [t.double() for t in (q, k, v)]
            x[i] = x[i] + sign * h * u
            return float((exact_forward(*x, causal, a.scale, ql, kl)[0] * first(c)).sum())

        slope = (f(1) - f(-1)) / (2 * h)
        # the product's own bound along u; out is rounded to bfloat16 in D: 2^-8 of sum |dO O| per row, P |K| scale of it
        rounded = (first(c) * first(out)).abs().sum(3).sum() * BF * a.scale * 8 if i < 2 else 0.0
        room = float((bound * u.transpose(1, 2).abs()).sum() + BF * (first(g).abs() * u.transpose(1, 2).abs()).sum() + rounded)
        got = float((g.double() * u).sum())
        assert abs(got - slope) <= room, (i, got, slope, room)
        assert room < 1.5 * float((g.double().abs() * u.abs()).sum())     # the room says something


def test_on_another_stream(ctx):
    q, k, v, do = tensors(2, 260, 260, 2, 1, 64, 60)
    a = L.Attention(ctx, 2, 1, 64)
    out, lse = a.forward(q, k, v)
    here = a.backward(q, k, v, out, lse, do)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out2, lse2 = a.forward(q, k, v, stream=s)
    there = a.backward(q, k, v, out2, lse2, do, stream=s)
    s.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(x, y) for x, y in zip(here, there))


def test_in_a_captured_graph(ctx):
    q, k, v, do = tensors(1, 300, 300, 2, 2, 64, 70)
    a = L.Attention(ctx, 2, 2, 64)
    out, lse = a.forward(q, k, v)
    want = a.backward(q, k, v, out, lse, do)
    torch.cuda.synchronize()
    gc.collect()                 # a context of another module that is freed during the capture would end it
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o2, l2 = a.forward(q, k, v)
        got = a.backward(q, k, v, o2, l2, do)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, o2) and all(torch.equal(x, y) for x, y in zip(want, got))


def test_sizes_of_zero(ctx):
    a = L.Attention(ctx, 2, 1, 64)
    for q_len, kv_len in ((0, 5), (5, 0), (0, 0)):
        q, k, v, do = tensors(2, q_len, kv_len, 2, 1, 64, 80)
        out, lse = a.forward(q, k, v)
        assert not bool(out.any()) and bool((lse == -math.inf).all())
        assert not any(bool(g.any()) for g in a.backward(q, k, v, out, lse, do))
    q, k, v, do = tensors(0, 5, 5, 2, 1, 64, 81)
    a.backward(q, k, v, *a.forward(q, k, v), do)


def test_refusals(ctx):
    q, k, v, do = tensors(2, 20, 30, 4, 2, 64, 90)
    a = L.Attention(ctx, 4, 2, 64)
    out, lse = a.forward(q, k, v)
    n = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    for bad in (lambda: a.forward(q[:, :, :3], k, v), lambda: a.forward(q, k[:1], v[:1]), lambda: a.forward(q, k, v[:, :29]),
                lambda: a.forward(q, k, v, n.long()), lambda: a.forward(q, k, v, n[:1]), lambda: a.forward(q.cpu(), k, v),
                lambda: a.backward(q, k, v, out, lse[:, :, :19], do), lambda: a.backward(q, k, v, out, lse, do[:, :19]),
                lambda: L.Attention(ctx, 3, 2, 64)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        a.forward(q.float(), k, v)

    def status(f):
        with pytest.raises(B.OmniError) as err:
            f()
        return err.value.status

    big = randn((1, 4, 2, 136), 0)
    assert status(lambda: L.Attention(ctx, 2, 2, 136).forward(big, big, big)) == B.ERR_TOO_LARGE
    odd = randn((1, 4, 2, 60), 0)
    assert status(lambda: L.Attention(ctx, 2, 2, 60).forward(odd, odd, odd)) == B.ERR_BAD_CONFIG
    assert status(lambda: L.Attention(ctx, 4, 2, 64, scale=-1.0).forward(q, k, v)) == B.ERR_BAD_CONFIG
    shifted = randn((2 * 20 * 4 * 64 + 1,), 0)[1:].view(2, 20, 4, 64)
    assert status(lambda: a.forward(shifted, k, v)) == B.ERR_ALIGN
    thin = randn((2, 20, 4, 68), 0)[..., :64]
    assert status(lambda: a.forward(thin, k, v)) == B.ERR_ALIGN
