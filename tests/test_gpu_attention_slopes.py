"""The gradient of attention against differences of the forward formula in 64 bits, along the gradient's own signs, where
the slope is the sum of its absolute values and an error of two percent shows.

With A_ij = u_i . K_j (or Q_i . u_j), a slope along u is scale sum dS_ij A_ij, so that what the kernels may be off by is
  scale sum E_ij |A_ij|              E the bound of dS (P and dS as bfloat16, see test_gpu_attention.py)
  scale sum_i d_i |sum_j P_ij A_ij|  d_i = 2^-8 sum_c |dO_ic O_ic|: D is taken from the bfloat16 output
  2^-8 sum |g u|                     the gradient as bfloat16
and for V, with A_ij = dO_i . u_j, sum (2^-8 + e) P_ij |A_ij| + 2^-8 sum |g u|."""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

from test_gpu_attention import BF, allowed, exact_forward, first, shared, tensors

pytestmark = pytest.mark.gpu


def slope_of(x, i, u, c, causal, scale, ql, kl, h=1e-5):
    def f(sign):
        y = [t.double() for t in x]
        y[i] = y[i] + sign * h * u
        return float((exact_forward(*y, causal, scale, ql, kl)[0] * first(c)).sum())

    return (f(1) - f(-1)) / (2 * h)


def room_of(x, i, u, g, c, causal, scale, ql, kl):
    q, k, v = x
    group = q.shape[2] // k.shape[2]
    out, lse, _, e = exact_forward(q, k, v, causal, scale, ql, kl)
    ok = allowed(q.shape[1], k.shape[1], causal, ql, kl)
    qq, kk, vv, dd = first(q), shared(k, group), shared(v, group), first(c)
    p = torch.where(ok, torch.exp(qq @ kk.transpose(2, 3) * scale - lse[..., None].clamp(min=-1e300)), 0.0)
    stored = BF * float((g.double().abs() * u.abs()).sum())
    if i == 2:
        return float(((BF + e) * p * (dd @ shared(u, group).transpose(2, 3)).abs()).sum()) + stored
    a = first(u) @ kk.transpose(2, 3) if i == 0 else qq @ shared(u, group).transpose(2, 3)
    ds = p * (dd @ vv.transpose(2, 3) - (dd * out).sum(3, keepdim=True))
    size = (dd * out).abs().sum(3, keepdim=True)
    off = BF * ds.abs() + p * (e + 2.0 ** -17) * (dd.abs() @ vv.abs().transpose(2, 3) + size)
    rounded = BF * size[..., 0] * (p * a).sum(3).abs()
    return scale * float((off * a.abs()).sum() + rounded.sum()) + stored


CASES = [(1, 40, 50, 2, 1, 64, False), (1, 40, 50, 2, 1, 64, True), (2, 150, 150, 4, 2, 128, True), (1, 300, 140, 3, 3, 80, True),
         (1, 3, 1500, 2, 1, 64, False)]


@pytest.mark.parametrize("batch,q_len,kv_len,heads,kv_heads,dim,causal", CASES)
def test_slope_along_the_gradient(batch, q_len, kv_len, heads, kv_heads, dim, causal):
    q, k, v, c = tensors(batch, q_len, kv_len, heads, kv_heads, dim, 50)
    a = L.Attention(B.Omni(1, 1, 1, 1), heads, kv_heads, dim, causal=causal)
    out, lse = a.forward(q, k, v)
    grads = a.backward(q, k, v, out, lse, c)
    ql, kl = (torch.full((batch,), n, dtype=torch.int32, device="cuda") for n in (q_len, kv_len))
    for i, g in enumerate(grads):
        u = g.double().sign()
        got = float((g.double() * u).sum())
        slope = slope_of((q, k, v), i, u, c, causal, a.scale, ql, kl)
        room = room_of((q, k, v), i, u, g, c, causal, a.scale, ql, kl)
        assert abs(got - slope) <= room, (i, got, slope, room)
        assert room < 0.02 * slope, (i, room, slope)                 # a wrong term, sign or factor would not fit in
