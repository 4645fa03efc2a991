"""A small language model trained by K workers of different speed, from a teacher's top logits.

The whole synchronous loop on one GPU: every worker computes the gradient of its own batch of
sequences with the operators of ``language`` (embedding, attention, distillation loss; the plain matrix
products are torch's), in bfloat16 into its gradient bucket, and ``Omni.step_bsp`` aggregates the K
buckets with the weights lambda_k = b_k / B, updates the float parameters and their bfloat16 copy,
which the next forward pass reads, and re-batches from the workers' throughputs.

A worker's loss is the mean over its own targets, so the weighted mean of the workers' gradients is the
gradient of the mean over the global batch when all sequences have as many targets.

The model: tied embedding E (scaled by sqrt(dim) at the bottom), one attention block with shared
key/value heads and a residual connection, logits = y E^T.  With ``Config.rotary`` the heads of queries and
keys are normed and rotated by their positions.

Other objective, other update: with ``objective="policy"`` the student samples tokens, is rewarded where the
teacher lists them, and follows the clipped policy loss with a divergence from its first self; with
``optimizer="adamw"`` or ``"adamw8"`` the workers' weighted gradients go through AdamW with moments of 32 or 8 bits
instead of SGD.

    python -m paper_2503_17469_b200.student --steps 30
    python -m paper_2503_17469_b200.student --steps 30 --rotary --objective policy --optimizer adamw8 --lr 0.003
"""
from __future__ import annotations

import argparse
import math
from dataclasses import dataclass, field
from typing import List, Optional, Sequence

import torch

from . import binding as B
from . import language as L
from . import workloads as W


@dataclass
class Config:
    vocab: int = 1000
    dim: int = 128
    heads: int = 4
    kv_heads: int = 2
    head_dim: int = 32
    length: int = 64          # padded length of a sequence
    top: int = 8              # teacher's logits per position
    temperature: float = 2.0
    rotary: bool = False      # norms of query and key heads, and their rotation
    clip: float = 0.2         # of the policy objective, as its divergence's weight
    kl: float = 0.02

    @property
    def shapes(self):
        """Embedding (and head), query/key/value projection, output projection; weights of the two norms."""
        return [(self.vocab, self.dim), (self.dim, (self.heads + 2 * self.kv_heads) * self.head_dim),
                (self.heads * self.head_dim, self.dim)] + [(2, self.head_dim)] * self.rotary


@dataclass
class Batch:
    tokens: torch.Tensor      # int64 [sequences, length]
    lengths: torch.Tensor     # int32 [sequences]
    top_logits: torch.Tensor  # float32 [sequences * length, top]
    top_index: torch.Tensor   # int64, -1 behind the length


@dataclass
class Samples:
    tokens: torch.Tensor      # int64 [sequences, length]
    lengths: torch.Tensor     # int32 [sequences]
    actions: torch.Tensor     # int64 [sequences * length], -1 behind the length
    old: torch.Tensor         # float32, log-probabilities when they were sampled
    reference: torch.Tensor   # and under the reference
    advantage: torch.Tensor
    reward: torch.Tensor      # mean over the sampled tokens


@dataclass
class Trace:
    loss: List[float] = field(default_factory=list)            # mean over the global batch, per step
    reward: List[float] = field(default_factory=list)          # of the policy objective, the same mean
    batches: List[List[int]] = field(default_factory=list)     # b_k used in the step


class Teacher:
    """A fixed table of top logits per token, and the sequences that go with it."""

    def __init__(self, cfg: Config, seed: int = 0, device="cuda"):
        self.cfg, self.device = cfg, device
        self.gen = torch.Generator(device=device).manual_seed(seed)
        noise = torch.randn(cfg.vocab, cfg.vocab, device=device, generator=self.gen) * 3
        self.logits, self.index = torch.topk(noise, cfg.top, dim=1)

    def batch(self, sequences: int, ragged: bool = False) -> Batch:
        c = self.cfg
        tokens = torch.randint(0, c.vocab, (sequences, c.length), device=self.device, generator=self.gen)
        lengths = torch.full((sequences,), c.length, dtype=torch.int32, device=self.device)
        if ragged:
            lengths = torch.randint(1, c.length + 1, (sequences,), device=self.device, generator=self.gen).int()
        there = torch.arange(c.length, device=self.device)[None] < lengths[:, None]
        flat = tokens.view(-1)
        index = torch.where(there.view(-1, 1), self.index[flat], -1)
        return Batch(tokens, lengths, self.logits[flat], index)

    @staticmethod
    def reward(batch: Batch, actions: torch.Tensor) -> torch.Tensor:
        """1 where the teacher lists the action."""
        return (batch.top_index == actions[:, None]).any(1).float()


class Student:
    """Parameters of the model in one flat bucket, K gradient buckets, and the pass that fills one of them."""

    def __init__(self, omni: "B.Omni", cfg: Config, seed: int = 1, device="cuda", optimizer: str = "sgd"):
        if optimizer not in ("sgd", "adamw", "adamw8"):
            raise ValueError("optimizer is sgd, adamw or adamw8")
        self.omni, self.cfg = omni, cfg
        self.layout = W.pack_buckets([math.prod(s) for s in cfg.shapes], 2, None)
        gen = torch.Generator(device=device).manual_seed(seed)
        n = self.layout.total
        self.theta = torch.zeros(n, device=device)
        for i, (part, shape) in enumerate(zip(self.views(self.theta), cfg.shapes)):
            if i == 3:                                                                  # the norms' weights
                part.fill_(1.0)
                continue
            part.normal_(0.0, cfg.dim ** -0.5 if shape[0] == cfg.vocab else shape[0] ** -0.5, generator=gen)
        self.theta_lp = self.theta.bfloat16()
        self.momentum = torch.zeros(n, device=device)
        self.grads = [torch.zeros(n, device=device, dtype=torch.bfloat16) for _ in range(omni.K)]
        self.buckets = B.BucketSet.from_flat(self.layout, self.theta, self.grads, self.momentum, self.theta_lp)
        self.embedding = L.Embedding(omni, cfg.vocab, cfg.dim, scale=math.sqrt(cfg.dim))
        self.attention = L.Attention(omni, cfg.heads, cfg.kv_heads, cfg.head_dim, causal=True)
        self.distillation = L.Distillation(omni, cfg.temperature)
        self.policy = L.Policy(omni, cfg.clip, kl=cfg.kl)
        self.gen = gen
        if cfg.rotary:
            self.rotary = L.Rotary(omni, cfg.heads, cfg.kv_heads, cfg.head_dim, L.Rotary.geometric(cfg.head_dim // 2))
        self.adamw = None
        if optimizer != "sgd":
            workers = [self.views(g) for g in self.grads]
            self.adamw = L.AdamW(omni, self.views(self.theta), list(zip(*workers)), self.views(self.theta_lp), betas=(0.9, 0.95),
                                 weight_decay=[0.01] * 3 + [0.0] * cfg.rotary, bits=8 if optimizer == "adamw8" else 32)

    def views(self, flat) -> List[torch.Tensor]:
        return [flat[start:start + n].view(self.cfg.shapes[i]) for i, start, n in self.layout.tensor_slices()]

    def forward(self, params, tokens, lengths):
        """(logits [rows, vocab], what the backward pass needs) with bfloat16 parameters."""
        c = self.cfg
        e, w_qkv, w_o = params[:3]
        sequences, length = tokens.shape
        rows = sequences * length
        heads = c.heads + 2 * c.kv_heads

        x = self.embedding.forward(tokens, e)                                           # [sequences, length, dim]
        x2 = x.view(rows, c.dim)
        qkv = (x2 @ w_qkv).view(sequences, length, heads, c.head_dim)
        q, k, v = qkv[:, :, :c.heads], qkv[:, :, c.heads:c.heads + c.kv_heads], qkv[:, :, c.heads + c.kv_heads:]
        turned = None
        if c.rotary:
            positions = torch.arange(length, device=tokens.device)[None].expand(sequences, -1)
            turned = (positions, *params[3])
            q, k = self.rotary.forward(q, k, *turned, lengths=lengths)
        out, lse = self.attention.forward(q, k, v, lengths, lengths)
        out2 = out.view(rows, -1)
        y = torch.addmm(x2, out2, w_o)
        return y @ e.t(), (tokens, lengths, x2, qkv, q, k, v, turned, out, lse, out2, y)

    def backward(self, params, grads, d_logits, saved) -> None:
        """The parameters' gradients into `grads`."""
        c = self.cfg
        e, w_qkv, w_o = params[:3]
        g_e, g_qkv, g_o = grads[:3]
        tokens, lengths, x2, qkv, q, k, v, turned, out, lse, out2, y = saved
        dy = d_logits @ e
        torch.mm(d_logits.t(), y, out=g_e)                                              # the head's part of the tied gradient
        torch.mm(out2.t(), dy, out=g_o)
        d_out = (dy @ w_o.t()).view(out.shape)
        d_qkv = torch.empty_like(qkv)
        d_q, d_k, d_v = d_qkv[:, :, :c.heads], d_qkv[:, :, c.heads:c.heads + c.kv_heads], d_qkv[:, :, c.heads + c.kv_heads:]
        self.attention.backward(q, k, v, out, lse, d_out, lengths, lengths, grads=(d_q, d_k, d_v))
        if c.rotary:
            self.rotary.backward(qkv[:, :, :c.heads], qkv[:, :, c.heads:c.heads + c.kv_heads], turned[0], d_q, d_k, *turned[1:], lengths=lengths,
                                 grads=(d_q, d_k), weight_grads=tuple(grads[3]))
        d_qkv2 = d_qkv.view(x2.shape[0], -1)
        torch.mm(x2.t(), d_qkv2, out=g_qkv)
        dx = torch.addmm(dy, d_qkv2, w_qkv.t())
        self.embedding.backward(tokens, dx, grad=g_e, accumulate=True)                  # and the lookup's part

    @staticmethod
    def _weights(lengths, rows: int):
        """(targets of the batch, the weight of each row in their mean); rows without a target do not count."""
        targets = lengths.sum().float()
        return targets, (1.0 / targets).expand(rows).contiguous()

    def gradient(self, worker: int, batch) -> torch.Tensor:
        """The worker's pass: its bucket receives the gradient of its mean loss, which is returned (on the device)."""
        params, grads = self.views(self.theta_lp), self.views(self.grads[worker])
        logits, saved = self.forward(params, batch.tokens, batch.lengths)
        targets, weight = self._weights(batch.lengths, len(logits))
        if isinstance(batch, Samples):
            loss, _, _, d_logits = self.policy.step(logits, batch.actions, batch.old, batch.advantage, weight, batch.reference, grad=logits)
        else:
            loss, _, d_logits = self.distillation.step(logits, batch.top_logits, batch.top_index, weight, grad=logits)
        self.backward(params, grads, d_logits, saved)
        return loss.sum() / targets

    def sample(self, batch: Batch, reference) -> Samples:
        """One token for each position from the student's own probabilities; the advantage is the reward less its mean."""
        logits, _ = self.forward(self.views(self.theta_lp), batch.tokens, batch.lengths)
        actions = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=self.gen)[:, 0]
        there = batch.top_index[:, 0] >= 0
        actions = torch.where(there, actions, -1)
        old, _ = self.policy.logprob(logits, actions)
        ref, _ = self.policy.logprob(self.forward(reference, batch.tokens, batch.lengths)[0], actions)
        reward = Teacher.reward(batch, actions) * there
        mean = reward.sum() / there.sum()
        return Samples(batch.tokens, batch.lengths, actions, old, ref, (reward - mean) * there, mean)

    def step(self, batches, throughputs: Sequence[float], lr: float, momentum: Optional[float] = None) -> torch.Tensor:
        """One iteration of Algorithm 1: every worker's gradient, then aggregation, update and re-batch.  ``momentum`` is SGD's, 0.9 by default."""
        if momentum is not None and self.adamw is not None:
            raise ValueError("momentum: AdamW has none")
        used = self.omni.batches
        losses = torch.stack([self.gradient(k, b) for k, b in enumerate(batches)])
        if self.adamw is None:
            self.omni.step_bsp(self.buckets, throughputs, lr, 0.9 if momentum is None else momentum)
        else:
            self.adamw.step(lr, used)
            self.omni.rebatch(throughputs)
        share = torch.tensor(used, device=losses.device, dtype=torch.float32) / sum(used)
        return (losses * share).sum()


def train(steps: int = 30, throughputs: Sequence[float] = (1.0, 2.0, 4.0, 8.0), global_batch: int = 64, lr: float = 0.5,
          cfg: Optional[Config] = None, seed: int = 0, ragged: bool = False, objective: str = "distillation",
          optimizer: str = "sgd") -> Trace:
    """Trains a student on fresh sequences for `steps` steps of the synchronous loop."""
    if objective not in ("distillation", "policy"):
        raise ValueError("objective is distillation or policy")
    cfg = cfg or Config()
    K = len(throughputs)
    omni = B.Omni(K, global_batch, max(1, global_batch // K // 8), 3 * global_batch // K)
    teacher, student = Teacher(cfg, seed), Student(omni, cfg, seed + 1, optimizer=optimizer)
    first = student.views(student.theta_lp.clone())
    trace, losses, rewards = Trace(), [], []
    for _ in range(steps):
        b = omni.batches
        trace.batches.append(b)
        batches = [teacher.batch(n, ragged) for n in b]
        if objective == "policy":
            batches = [student.sample(x, first) for x in batches]
            rewards.append(sum(n / sum(b) * x.reward for n, x in zip(b, batches)))
        losses.append(student.step(batches, throughputs, lr))
    omni.stats()                                                                        # raises if a wait ran out
    trace.loss = torch.stack(losses).tolist() if losses else []
    trace.reward = torch.stack(rewards).tolist() if rewards else []
    return trace


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=30)
    p.add_argument("--global-batch", type=int, default=64)
    p.add_argument("--lr", type=float, default=0.5)
    p.add_argument("--ragged", action="store_true", help="sequences of different lengths")
    p.add_argument("--rotary", action="store_true", help="norms and rotation of the query and key heads")
    p.add_argument("--objective", choices=("distillation", "policy"), default="distillation")
    p.add_argument("--optimizer", choices=("sgd", "adamw", "adamw8"), default="sgd")
    a = p.parse_args()
    t = train(a.steps, global_batch=a.global_batch, lr=a.lr, cfg=Config(rotary=a.rotary), ragged=a.ragged, objective=a.objective,
              optimizer=a.optimizer)
    for i, (loss, b) in enumerate(zip(t.loss, t.batches)):
        print(f"step {i:3d}  loss {loss:8.4f}  batches {b}" + (f"  reward {t.reward[i]:.4f}" if t.reward else ""))


if __name__ == "__main__":
    main()
