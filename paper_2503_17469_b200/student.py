"""A small language model trained by K workers of different speed, from a teacher's top logits.

The whole synchronous loop on one GPU: every worker computes the gradient of its own batch of
sequences with the operators of ``language`` (embedding, attention, distillation loss; the plain matrix
products are torch's), in bfloat16 into its gradient bucket, and ``Omni.step_bsp`` aggregates the K
buckets with the weights lambda_k = b_k / B, updates the float parameters and their bfloat16 copy,
which the next forward pass reads, and re-batches from the workers' throughputs.

A worker's loss is the mean over its own targets, so the weighted mean of the workers' gradients is the
gradient of the mean over the global batch when all sequences have as many targets.

The model: tied embedding E (scaled by sqrt(dim) at the bottom), one attention block with shared
key/value heads and a residual connection, logits = y E^T.

    python -m paper_2503_17469_b200.student --steps 30
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

    @property
    def shapes(self):
        """Embedding (and head), query/key/value projection, output projection."""
        return [(self.vocab, self.dim), (self.dim, (self.heads + 2 * self.kv_heads) * self.head_dim),
                (self.heads * self.head_dim, self.dim)]


@dataclass
class Batch:
    tokens: torch.Tensor      # int64 [sequences, length]
    lengths: torch.Tensor     # int32 [sequences]
    top_logits: torch.Tensor  # float32 [sequences * length, top]
    top_index: torch.Tensor   # int64, -1 behind the length


@dataclass
class Trace:
    loss: List[float] = field(default_factory=list)            # mean over the global batch, per step
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


class Student:
    """Parameters of the model in one flat bucket, K gradient buckets, and the pass that fills one of them."""

    def __init__(self, omni: "B.Omni", cfg: Config, seed: int = 1, device="cuda"):
        self.omni, self.cfg = omni, cfg
        self.layout = W.pack_buckets([math.prod(s) for s in cfg.shapes], 2, None)
        gen = torch.Generator(device=device).manual_seed(seed)
        n = self.layout.total
        self.theta = torch.zeros(n, device=device)
        for part, shape in zip(self.views(self.theta), cfg.shapes):
            part.normal_(0.0, cfg.dim ** -0.5 if shape[0] == cfg.vocab else shape[0] ** -0.5, generator=gen)
        self.theta_lp = self.theta.bfloat16()
        self.momentum = torch.zeros(n, device=device)
        self.grads = [torch.zeros(n, device=device, dtype=torch.bfloat16) for _ in range(omni.K)]
        self.buckets = B.BucketSet.from_flat(self.layout, self.theta, self.grads, self.momentum, self.theta_lp)
        self.embedding = L.Embedding(omni, cfg.vocab, cfg.dim, scale=math.sqrt(cfg.dim))
        self.attention = L.Attention(omni, cfg.heads, cfg.kv_heads, cfg.head_dim, causal=True)
        self.distillation = L.Distillation(omni, cfg.temperature)

    def views(self, flat) -> List[torch.Tensor]:
        return [flat[start:start + n].view(self.cfg.shapes[i]) for i, start, n in self.layout.tensor_slices()]

    def gradient(self, worker: int, batch: Batch) -> torch.Tensor:
        """The worker's pass: its bucket receives the gradient of its mean loss, which is returned (on the device)."""
        c = self.cfg
        e, w_qkv, w_o = self.views(self.theta_lp)
        g_e, g_qkv, g_o = self.views(self.grads[worker])
        sequences, length = batch.tokens.shape
        rows = sequences * length
        heads = c.heads + 2 * c.kv_heads

        x = self.embedding.forward(batch.tokens, e)                                     # [sequences, length, dim]
        x2 = x.view(rows, c.dim)
        qkv = (x2 @ w_qkv).view(sequences, length, heads, c.head_dim)
        q, k, v = qkv[:, :, :c.heads], qkv[:, :, c.heads:c.heads + c.kv_heads], qkv[:, :, c.heads + c.kv_heads:]
        out, lse = self.attention.forward(q, k, v, batch.lengths, batch.lengths)
        out2 = out.view(rows, -1)
        y = torch.addmm(x2, out2, w_o)
        logits = y @ e.t()

        targets = batch.lengths.sum().float()
        weight = (1.0 / targets).expand(rows).contiguous()                              # rows without a target do not count
        loss, _, d_logits = self.distillation.step(logits, batch.top_logits, batch.top_index, weight, grad=logits)

        dy = d_logits @ e
        torch.mm(d_logits.t(), y, out=g_e)                                              # the head's part of the tied gradient
        torch.mm(out2.t(), dy, out=g_o)
        d_out = (dy @ w_o.t()).view(out.shape)
        d_qkv = torch.empty_like(qkv)
        self.attention.backward(q, k, v, out, lse, d_out, batch.lengths, batch.lengths,
                                grads=(d_qkv[:, :, :c.heads], d_qkv[:, :, c.heads:c.heads + c.kv_heads], d_qkv[:, :, c.heads + c.kv_heads:]))
        d_qkv2 = d_qkv.view(rows, -1)
        torch.mm(x2.t(), d_qkv2, out=g_qkv)
        dx = torch.addmm(dy, d_qkv2, w_qkv.t())
        self.embedding.backward(batch.tokens, dx, grad=g_e, accumulate=True)            # and the lookup's part
        return loss.sum() / targets

    def step(self, batches: Sequence[Batch], throughputs: Sequence[float], lr: float, momentum: float = 0.9) -> torch.Tensor:
        """One iteration of Algorithm 1: every worker's gradient, then aggregation, update and re-batch."""
        used = self.omni.batches
        losses = torch.stack([self.gradient(k, b) for k, b in enumerate(batches)])
        self.omni.step_bsp(self.buckets, throughputs, lr, momentum)
        share = torch.tensor(used, device=losses.device, dtype=torch.float32) / sum(used)
        return (losses * share).sum()


def train(steps: int = 30, throughputs: Sequence[float] = (1.0, 2.0, 4.0, 8.0), global_batch: int = 64, lr: float = 0.5,
          cfg: Optional[Config] = None, seed: int = 0, ragged: bool = False) -> Trace:
    """Trains a student on fresh sequences for `steps` steps of the synchronous loop."""
    cfg = cfg or Config()
    K = len(throughputs)
    omni = B.Omni(K, global_batch, max(1, global_batch // K // 8), 3 * global_batch // K)
    teacher, student = Teacher(cfg, seed), Student(omni, cfg, seed + 1)
    trace, losses = Trace(), []
    for _ in range(steps):
        b = omni.batches
        trace.batches.append(b)
        losses.append(student.step([teacher.batch(n, ragged) for n in b], throughputs, lr))
    omni.stats()                                                                        # raises if a wait ran out
    trace.loss = torch.stack(losses).tolist() if losses else []
    return trace


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=30)
    p.add_argument("--global-batch", type=int, default=64)
    p.add_argument("--lr", type=float, default=0.5)
    p.add_argument("--ragged", action="store_true", help="sequences of different lengths")
    a = p.parse_args()
    t = train(a.steps, global_batch=a.global_batch, lr=a.lr, ragged=a.ragged)
    for i, (loss, b) in enumerate(zip(t.loss, t.batches)):
        print(f"step {i:3d}  loss {loss:8.4f}  batches {b}")


if __name__ == "__main__":
    main()
