"""The operators together, as a worker uses them: a small student's gradients against autograd in 64 bits, the
weighted aggregation of the workers' gradients against one worker with the whole batch, and a falling loss.

Tolerances (norm of the difference over the norm): activations, gradients and buckets are bfloat16, each
rounding 2^-9 root mean square at most; a gradient has about ten of them in a row behind it, sqrt(10) 2^-9 < 1 %, and twice
that is asked for.  Two ways through the same data differ by the buckets' roundings (K and one): 1 %.
"""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import student as S

pytestmark = pytest.mark.gpu
CFG = S.Config(vocab=333, dim=64, heads=4, kv_heads=2, head_dim=16, length=40, top=5)


def plain_loss(cfg, params, batch):
    """The model's mean loss in double, by elementary operations."""
    e, w_qkv, w_o = params
    n, length = batch.tokens.shape
    x = e[batch.tokens] * math.sqrt(cfg.dim)
    qkv = (x @ w_qkv).view(n, length, cfg.heads + 2 * cfg.kv_heads, cfg.head_dim).transpose(1, 2)
    q, k, v = qkv.split([cfg.heads, cfg.kv_heads, cfg.kv_heads], 1)
    group = cfg.heads // cfg.kv_heads
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    i = torch.arange(length, device=x.device)
    ok = (i[None, :] <= i[:, None])[None, None] & (i[None, :] < batch.lengths.long()[:, None])[:, None, None, :]
    s = (q @ k.transpose(2, 3) * cfg.head_dim ** -0.5).masked_fill(~ok, -math.inf)
    out = (torch.softmax(s, 3) @ v).transpose(1, 2).reshape(n * length, -1)
    z = (x.reshape(n * length, -1) + out @ w_o) @ e.t() / cfg.temperature
    there = batch.top_index[:, 0] >= 0
    p = torch.softmax(batch.top_logits.double() / cfg.temperature, 1)
    log_q = torch.log_softmax(z, 1).gather(1, batch.top_index.clamp(min=0))
    return (cfg.temperature ** 2 * (p * (p.log() - log_q)).sum(1))[there].sum() / there.sum()


def distance(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("ragged", [False, True])
def test_gradients_against_autograd_in_64_bits(ragged):
    omni = B.Omni(1, 6, 1, 6)
    student = S.Student(omni, CFG)
    batch = S.Teacher(CFG).batch(6, ragged)
    loss = float(student.gradient(0, batch))
    params = [p.double().requires_grad_() for p in student.views(student.theta_lp)]
    want = plain_loss(CFG, params, batch)
    value = float(want.detach())
    assert abs(loss - value) <= 0.02 * value
    for got, exact in zip(student.views(student.grads[0]), torch.autograd.grad(want, params)):
        assert distance(got, exact) <= 0.02
    omni.stats()


def test_weighted_gradients_of_workers_are_those_of_the_whole_batch():
    sizes = [2, 6, 19, 37]                                     # what 1 : 2 : 4 : 8 throughputs lead to
    many, one = B.Omni(4, 64, 2, 48), B.Omni(1, 64, 64, 64)
    many.set_batches(sizes)
    teacher = S.Teacher(CFG)
    parts = [teacher.batch(n) for n in sizes]
    whole = S.Batch(*(torch.cat([getattr(p, f) for p in parts]) for f in ("tokens", "lengths", "top_logits", "top_index")))
    a, b = S.Student(many, CFG), S.Student(one, CFG)
    start = a.theta.clone()
    la = a.step(parts, [1.0, 2.0, 4.0, 8.0], lr=1.0, momentum=0.0)
    lb = b.step([whole], [1.0], lr=1.0, momentum=0.0)
    assert abs(float(la) - float(lb)) <= 1e-3 * float(lb)
    for ta, tb, t0 in zip(a.views(a.theta), b.views(b.theta), a.views(start)):
        assert distance(ta - t0, tb - t0) <= 0.01
    assert torch.equal(a.theta_lp, a.theta.bfloat16())


@pytest.mark.parametrize("ragged", [False, True])
def test_training_lowers_the_loss_and_follows_the_throughputs(ragged):
    trace = S.train(steps=25, cfg=CFG, ragged=ragged)
    assert trace.loss[-1] < 0.5 * trace.loss[0], trace.loss
    assert trace.batches[0] == [16, 16, 16, 16] and all(sum(b) == 64 for b in trace.batches)
    assert trace.batches[-1] == sorted(trace.batches[-1]) and trace.batches[-1][3] > 2 * trace.batches[-1][0]
