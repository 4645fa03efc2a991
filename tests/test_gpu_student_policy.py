"""The operators of policy training together, as a worker uses them: head norms with rotation before attention, the clipped policy
loss on sampled tokens, AdamW on the workers' weighted gradients; and that the student without them is what it was.

Tolerances (norm of the difference over the norm): those of test_gpu_student.py, about ten bfloat16 roundings of 2^-9 root mean
square in a row and twice that, 2 %; and what the rounding of the logits does to their exponentials, which stand in the ratio of
every row and in its probabilities: a logit z is off by up to 2^-8 |z|, its exponential by as much of itself, and with it
the row's gradient, at most 2^-8 times the largest logit.  (The distillation's test divides its logits by a temperature of 2 and has no ratio.)
"""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import student as S

from test_gpu_student import distance

pytestmark = pytest.mark.gpu
CFG = S.Config(vocab=333, dim=64, heads=4, kv_heads=2, head_dim=16, length=40, top=5, rotary=True)


def turn(cfg, x, weight):
    """[sequences, heads, length, dim] in double."""
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
    half = cfg.head_dim // 2
    angle = torch.arange(x.shape[2], device=x.device)[:, None] * 10000.0 ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    z = torch.view_as_complex(torch.stack([n[..., :half], n[..., half:]], -1)) * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], -1)


def plain_logits(cfg, params, tokens, lengths):
    e, w_qkv, w_o, norms = params
    n, length = tokens.shape
    x = e[tokens] * math.sqrt(cfg.dim)
    qkv = (x @ w_qkv).view(n, length, cfg.heads + 2 * cfg.kv_heads, cfg.head_dim).transpose(1, 2)
    q, k, v = qkv.split([cfg.heads, cfg.kv_heads, cfg.kv_heads], 1)
    q, k = turn(cfg, q, norms[0]), turn(cfg, k, norms[1])
    group = cfg.heads // cfg.kv_heads
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    i = torch.arange(length, device=x.device)
    ok = (i[None, :] <= i[:, None])[None, None] & (i[None, :] < lengths.long()[:, None])[:, None, None, :]
    s = (q @ k.transpose(2, 3) * cfg.head_dim ** -0.5).masked_fill(~ok, -math.inf)
    out = (torch.softmax(s, 3) @ v).transpose(1, 2).reshape(n * length, -1)
    return (x.reshape(n * length, -1) + out @ w_o) @ e.t()


def plain_loss(cfg, params, batch):
    z = plain_logits(cfg, params, batch.tokens, batch.lengths)
    there = batch.actions >= 0
    logp = torch.log_softmax(z, 1).gather(1, batch.actions.clamp(min=0)[:, None])[:, 0]
    ratio = torch.exp(logp - batch.old.double())
    a = batch.advantage.double()
    surrogate = torch.minimum(ratio * a, ratio.clamp(1 - cfg.clip, 1 + cfg.clip) * a)
    gap = batch.reference.double() - logp
    return (-surrogate + cfg.kl * (torch.exp(gap) - gap - 1))[there].sum() / there.sum()


def samples(student, teacher, n, ragged, gen):
    """Sampled by another student, so that ratios are not 1; none within bfloat16's rounding of a border of the clipping."""
    other = S.Student(B.Omni(1, n, 1, n), CFG, seed=1)
    other.theta_lp.add_(torch.randn(other.theta_lp.shape, device="cuda", generator=gen) * 0.01)
    batch = other.sample(teacher.batch(n, ragged), other.views(other.theta_lp))
    logits, _ = student.forward(student.views(student.theta_lp), batch.tokens, batch.lengths)
    moved = student.policy.logprob(logits, batch.actions)[0] - batch.old
    for border in (math.log(1 - CFG.clip), math.log(1 + CFG.clip)):
        batch.old = torch.where((moved - border).abs() < 0.1, batch.old + 0.25, batch.old)
        moved = student.policy.logprob(logits, batch.actions)[0] - batch.old
    return batch


@pytest.mark.parametrize("ragged", [False, True])
def test_gradients_against_autograd_in_64_bits(ragged):
    omni = B.Omni(1, 6, 1, 6)
    student = S.Student(omni, CFG)
    gen = torch.Generator(device="cuda").manual_seed(3)
    student.views(student.theta_lp)[3].copy_(1 + 0.2 * torch.randn(2, CFG.head_dim, device="cuda", generator=gen))
    batch = samples(student, S.Teacher(CFG), 6, ragged, gen)
    loss = float(student.gradient(0, batch))
    params = [p.double().requires_grad_() for p in student.views(student.theta_lp)]
    want = plain_loss(CFG, params, batch)
    # terms of both signs: of their mean size; ratios are below 2 here
    with torch.no_grad():
        largest = float(plain_logits(CFG, params, batch.tokens, batch.lengths)[batch.actions >= 0].abs().max())
    room = 0.02 + 2.0 ** -8 * largest
    assert abs(loss - float(want.detach())) <= room * float(2 * batch.advantage.abs().sum() / (batch.actions >= 0).sum() + abs(want.detach()))
    for got, exact in zip(student.views(student.grads[0]), torch.autograd.grad(want, params)):
        assert distance(got, exact) <= room
    omni.stats()


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8"])
def test_a_step_of_all_workers(optimizer):
    """The parameters move by AdamW's first step on the weighted mean of the buckets: its sign, almost, times the rate."""
    omni = B.Omni(4, 16, 1, 12)
    omni.set_batches([1, 2, 5, 8])
    student, teacher = S.Student(omni, CFG, optimizer=optimizer), S.Teacher(CFG)
    first = student.views(student.theta_lp.clone())
    batches = [student.sample(teacher.batch(n), first) for n in (1, 2, 5, 8)]
    start = [p.clone() for p in student.views(student.theta)]
    student.step(batches, [1.0, 2.0, 4.0, 8.0], lr=1e-3)
    assert student.adamw.steps == 1 and sum(omni.batches) == 16
    for i, (p, p0, lp, decay) in enumerate(zip(student.views(student.theta), start, student.views(student.theta_lp), (0.01, 0.01, 0.01, 0.0))):
        g = sum(b / 16 * student.views(student.grads[k])[i].double() for k, b in enumerate((1, 2, 5, 8)))
        want = p0.double() * (1 - 1e-3 * decay) - 1e-3 * g / (g.abs() + 1e-8)
        # the aggregate is off by four roundings, 2^-22 of its terms, which matters where they cancel; the quotient by 2^-20, theta by two roundings
        terms = sum(b / 16 * student.views(student.grads[k])[i].double().abs() for k, b in enumerate((1, 2, 5, 8)))
        near = 1e-3 * 1e-8 * 2.0 ** -21 * terms / (g.abs() + 1e-8) ** 2 + 1e-3 * 2.0 ** -19 + 2.0 ** -22 * p0.abs()
        assert bool(((p.double() - want).abs() <= near).all())
        assert torch.equal(lp, p.bfloat16())


def test_the_whole_loop_runs():
    for optimizer, lr in (("adamw", 2e-3), ("adamw8", 2e-3), ("sgd", 0.1)):
        trace = S.train(steps=6, cfg=CFG, ragged=True, objective="policy", optimizer=optimizer, lr=lr)
        assert len(trace.reward) == 6 and all(math.isfinite(x) for x in trace.loss) and all(sum(b) == 64 for b in trace.batches)
        assert trace.batches[-1] == sorted(trace.batches[-1])
    with pytest.raises(ValueError):
        S.train(steps=1, cfg=CFG, objective="reward")
    with pytest.raises(ValueError):
        S.Student(B.Omni(1, 1, 1, 1), CFG, optimizer="lion")


def test_sampled_tokens_are_on_the_policy():
    """The ratio of a first step is exactly 1: the log-probabilities of a step are those of the sampling call, bit for bit."""
    student, teacher = S.Student(B.Omni(1, 8, 1, 8), CFG), S.Teacher(CFG)
    first = student.views(student.theta_lp.clone())
    batch = student.sample(teacher.batch(8, True), first)
    assert torch.equal(batch.old, batch.reference)
    logits, _ = student.forward(first, batch.tokens, batch.lengths)
    loss, logp, _, _ = student.policy.step(logits, batch.actions, batch.old, batch.advantage, torch.ones_like(batch.old), batch.reference)
    assert torch.equal(logp, batch.old) and torch.equal(loss, -batch.advantage)
    assert bool((batch.actions.view(8, -1) >= 0).sum(1).eq(batch.lengths).all())
