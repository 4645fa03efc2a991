"""Operators of a language model's training pass: embedding, attention, distillation loss.

What a worker computes its gradients with, on torch tensors of one CUDA device.  Each class keeps an
operator's constants and an ``Omni`` context (launch counts, errors, the status word of bounded
waits); its calls allocate their outputs with torch unless they are given, take scratch memory from torch's
caching allocator, enqueue on ``stream`` (a torch stream, default the current one) and do not
synchronise.  The formulas, types and limits stand in ``include/omni.h``.  There is no fallback.

Arguments that do not fit together raise ``ValueError`` or ``TypeError`` before anything is
enqueued; what the library refuses raises ``OmniError``.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional

import torch

from . import binding as B

_DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16}
_INDEX = {torch.int32: B.I32, torch.int64: B.I64}


def _code(t, codes, what: str) -> int:
    c = codes.get(t.dtype)
    if c is None:
        raise TypeError(f"{what}: dtype {t.dtype} is none of {', '.join(map(str, codes))}")
    return c


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _on(device, **tensors) -> None:
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} is on {t.device}, not on {device}")


def _rows(t, what: str) -> int:
    """Stride between the rows of a matrix whose rows are contiguous."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: a matrix with contiguous rows is wanted, got shape {tuple(t.shape)}, strides {t.stride()}")
    stride = t.stride(0)
    return stride if stride >= t.shape[1] else t.shape[1] if t.shape[0] <= 1 else stride


class _Operator:
    def __init__(self, ctx: "B.Omni"):
        self.ctx = ctx
        self._lib = B.lib()

    def _stream(self, stream):
        return B.Omni._stream(stream)

    @staticmethod
    def _allocating(stream):
        """Outputs and scratch belong to the stream that uses them."""
        return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)

    def _check(self, rc: int) -> None:
        if rc != B.OK:
            self.ctx._check(rc)


class Embedding(_Operator):
    """Lookup ``scale * weight[tokens]`` and its dense gradient.  ``padding``: a token that gets no gradient."""

    def __init__(self, ctx: "B.Omni", vocab: int, dim: int, scale: float = 1.0, padding: int = -1):
        super().__init__(ctx)
        _need(vocab >= 1 and dim >= 1, "vocab and dim are at least 1")
        self.vocab, self.dim, self.scale, self.padding = vocab, dim, scale, padding

    def forward(self, tokens, weight, dtype=None, out=None, stream=None):
        """``tokens``: int32 or int64, any shape, contiguous; ``weight``: [vocab, dim] float32 or bfloat16.
        Returns ``tokens.shape + (dim,)`` of ``dtype`` (default the table's)."""
        _need(tokens.is_contiguous(), "tokens: a contiguous tensor is wanted")
        _need(tuple(weight.shape) == (self.vocab, self.dim), f"weight: shape {(self.vocab, self.dim)} is wanted")
        n = tokens.numel()
        if out is None:
            with self._allocating(stream):
                out = torch.empty(*tokens.shape, self.dim, dtype=dtype or weight.dtype, device=tokens.device)
        _need(tuple(out.shape) == (*tokens.shape, self.dim) and out.is_contiguous(),
              "out: a contiguous tensor of the tokens' shape and dim is wanted")
        _on(tokens.device, weight=weight, out=out)
        self._check(self._lib.omni_embed_forward(
            self.ctx._h, tokens.data_ptr(), _code(tokens, _INDEX, "tokens"), n, weight.data_ptr(),
            _code(weight, _DTYPES, "weight"), _rows(weight, "weight"), self.vocab, self.dim, self.scale, out.data_ptr(),
            _code(out, _DTYPES, "out"), self.dim, self._stream(stream)))
        return out

    def backward(self, tokens, grad_out, dtype=torch.float32, grad=None, accumulate: bool = False, stream=None):
        """Gradient of the table, [vocab, dim] of ``dtype``; into ``grad`` if given (for example a view of a
        gradient bucket), added to it with ``accumulate``.  ``grad_out``: ``tokens.shape + (dim,)``,
        or a matrix of as many rows, rows contiguous."""
        _need(tokens.is_contiguous(), "tokens: a contiguous tensor is wanted")
        n = tokens.numel()
        g = grad_out if grad_out.dim() == 2 else grad_out.view(n, self.dim)
        _need(tuple(g.shape) == (n, self.dim), f"grad_out: {n} rows of {self.dim} are wanted")
        _need(grad is not None or not accumulate, "accumulate needs a gradient to add to")
        size = C.c_uint64()
        self._check(self._lib.omni_embed_workspace(n, self.vocab, self.dim, C.byref(size)))
        with self._allocating(stream):
            if grad is None:
                grad = torch.empty(self.vocab, self.dim, dtype=dtype, device=tokens.device)
            scratch = torch.empty(max(16, size.value), dtype=torch.uint8, device=tokens.device)
        _need(tuple(grad.shape) == (self.vocab, self.dim), f"grad: shape {(self.vocab, self.dim)} is wanted")
        _on(tokens.device, grad_out=g, grad=grad)
        self._check(self._lib.omni_embed_backward(
            self.ctx._h, tokens.data_ptr(), _code(tokens, _INDEX, "tokens"), n, g.data_ptr(),
            _code(g, _DTYPES, "grad_out"), _rows(g, "grad_out"), self.vocab, self.dim, self.scale, self.padding,
            grad.data_ptr(), _code(grad, _DTYPES, "grad"), _rows(grad, "grad"), accumulate, scratch.data_ptr(),
            scratch.numel(), self._stream(stream)))
        return grad


class Attention(_Operator):
    """Softmax attention on bfloat16 ``[batch, length, head, dim]`` tensors, forward and backward.

    ``heads`` query heads share ``kv_heads`` key/value heads in groups; ``causal`` aligns queries and
    keys at their ends; ``scale`` defaults to dim ** -0.5.  Any strides with a contiguous last dimension, multiples of 8
    elements (slices of one projection's output, for example)."""

    def __init__(self, ctx: "B.Omni", heads: int, kv_heads: int, dim: int, causal: bool = True, scale: Optional[float] = None):
        super().__init__(ctx)
        _need(heads >= 1 and kv_heads >= 1 and heads % kv_heads == 0, "heads is a multiple of kv_heads")
        self.heads, self.kv_heads, self.dim, self.causal = heads, kv_heads, dim, causal
        self.scale = dim ** -0.5 if scale is None else scale

    def _shape(self, q, k, q_lengths, kv_lengths):
        batch = q.shape[0]
        for name, t in (("q_lengths", q_lengths), ("kv_lengths", kv_lengths)):
            if t is not None:
                _need(t.dtype == torch.int32 and t.is_contiguous() and tuple(t.shape) == (batch,) and t.device == q.device,
                      f"{name}: contiguous int32 [batch] on the tensors' device is wanted")
        return B.omni_attn(batch, q.shape[1], k.shape[1], self.heads, self.kv_heads, self.dim, self.causal, self.scale,
                           None if q_lengths is None else q_lengths.data_ptr(),
                           None if kv_lengths is None else kv_lengths.data_ptr())

    def _view(self, t, what: str, like, length: int, heads: int):
        if t.dtype != torch.bfloat16:
            raise TypeError(f"{what}: dtype {t.dtype} is not bfloat16")
        _need(tuple(t.shape) == (like.shape[0], length, heads, self.dim) and (self.dim == 1 or t.stride(3) == 1),
              f"{what}: shape {(like.shape[0], length, heads, self.dim)} with a contiguous last dimension is wanted")
        _on(like.device, **{what: t})
        return B.omni_attn_view(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))

    def forward(self, q, k, v, q_lengths=None, kv_lengths=None, out=None, stream=None):
        """Returns (out like q, lse float32 [batch, heads, q_len])."""
        _need(q.dim() == 4 and k.dim() == 4, "q and k: [batch, length, head, dim] is wanted")
        a = self._shape(q, k, q_lengths, kv_lengths)
        with self._allocating(stream):
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            lse = torch.empty(a.batch, self.heads, a.q_len, device=q.device)
        self._check(self._lib.omni_attn_forward(
            self.ctx._h, C.byref(a), C.byref(self._view(q, "q", q, a.q_len, self.heads)),
            C.byref(self._view(k, "k", q, a.kv_len, self.kv_heads)), C.byref(self._view(v, "v", q, a.kv_len, self.kv_heads)),
            C.byref(self._view(out, "out", q, a.q_len, self.heads)), lse.data_ptr(), self._stream(stream)))
        return out, lse

    def backward(self, q, k, v, out, lse, grad_out, q_lengths=None, kv_lengths=None, grads=None, stream=None):
        """Returns the gradients of (q, k, v); into ``grads``, a tuple of three, if given.  ``out`` and ``lse`` are the
        forward call's."""
        _need(q.dim() == 4 and k.dim() == 4, "q and k: [batch, length, head, dim] is wanted")
        a = self._shape(q, k, q_lengths, kv_lengths)
        _need(lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (a.batch, self.heads, a.q_len)
              and lse.device == q.device, "lse: contiguous float32 [batch, heads, q_len] is wanted")
        with self._allocating(stream):
            dq, dk, dv = grads or (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
            # the library's own query: rows of whole tiles, two floats each
            size = C.c_uint64()
            self._check(self._lib.omni_attn_workspace(C.byref(a), C.byref(size)))
            scratch = torch.empty(max(16, size.value), dtype=torch.uint8, device=q.device)
        rows = [C.byref(self._view(t, name, q, a.q_len, self.heads))
                for t, name in ((q, "q"), (out, "out"), (grad_out, "grad_out"), (dq, "grads[0]"))]
        keys = [C.byref(self._view(t, name, q, a.kv_len, self.kv_heads))
                for t, name in ((k, "k"), (v, "v"), (dk, "grads[1]"), (dv, "grads[2]"))]
        self._check(self._lib.omni_attn_backward(
            self.ctx._h, C.byref(a), rows[0], keys[0], keys[1], rows[1], lse.data_ptr(), rows[2], rows[3], keys[2], keys[3],
            scratch.data_ptr(), scratch.numel(), self._stream(stream)))
        return dq, dk, dv


class Distillation(_Operator):
    """KL divergence (times temperature squared) of the student's softmax from a teacher's top logits, per row.
    An index of -1 marks an entry that is not there; a row without entries has loss 0 and no gradient."""

    def __init__(self, ctx: "B.Omni", temperature: float = 1.0):
        super().__init__(ctx)
        _need(temperature > 0, "temperature is positive")
        self.temperature = temperature

    def _describe(self, logits, top_logits, top_index):
        _need(logits.dim() == 2 and top_logits.dim() == 2 and top_logits.shape == top_index.shape
              and top_logits.shape[0] == logits.shape[0],
              "logits [rows, vocab], top_logits and top_index [rows, top] are wanted")
        if top_logits.dtype != torch.float32:
            raise TypeError("top_logits: float32 is wanted")
        stride = _rows(top_logits, "top_logits")
        _need(_rows(top_index, "top_index") == stride, "top_logits and top_index: the same stride is wanted")
        _on(logits.device, top_logits=top_logits, top_index=top_index)
        return B.omni_distill(logits.data_ptr(), logits.shape[0], _rows(logits, "logits"), logits.shape[1],
                              _code(logits, _DTYPES, "logits"), top_logits.data_ptr(), top_index.data_ptr(), stride,
                              top_logits.shape[1], _code(top_index, _INDEX, "top_index"), self.temperature)

    @staticmethod
    def _row_values(t, logits, what: str):
        _need(t.dtype == torch.float32 and t.is_contiguous() and tuple(t.shape) == (logits.shape[0],),
              f"{what}: contiguous float32 [rows] is wanted")
        _on(logits.device, **{what: t})
        return t.data_ptr()

    def _grad_like(self, logits, grad):
        if grad is None:
            grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        _need(grad.shape == logits.shape and grad.dtype == logits.dtype, "grad: the logits' shape and dtype are wanted")
        _on(logits.device, grad=grad)
        return grad

    def forward(self, logits, top_logits, top_index, stream=None):
        """Returns (loss, lse), float32 [rows] each."""
        d = self._describe(logits, top_logits, top_index)
        with self._allocating(stream):
            loss, lse = torch.empty(2, logits.shape[0], device=logits.device)
        self._check(self._lib.omni_distill_forward(self.ctx._h, C.byref(d), loss.data_ptr(), lse.data_ptr(), self._stream(stream)))
        return loss, lse

    def backward(self, logits, top_logits, top_index, lse, grad_loss, grad=None, stream=None):
        """Gradient of the logits from ``lse`` of the forward call and ``grad_loss`` [rows]; ``grad`` may be ``logits``."""
        d = self._describe(logits, top_logits, top_index)
        with self._allocating(stream):
            grad = self._grad_like(logits, grad)
        self._check(self._lib.omni_distill_backward(
            self.ctx._h, C.byref(d), self._row_values(lse, logits, "lse"), self._row_values(grad_loss, logits, "grad_loss"),
            grad.data_ptr(), _rows(grad, "grad"), self._stream(stream)))
        return grad

    def step(self, logits, top_logits, top_index, grad_loss, grad=None, stream=None):
        """Forward and backward in one pass; returns (loss, lse, gradient of the logits)."""
        d = self._describe(logits, top_logits, top_index)
        with self._allocating(stream):
            loss, lse = torch.empty(2, logits.shape[0], device=logits.device)
            grad = self._grad_like(logits, grad)
        self._check(self._lib.omni_distill_step(
            self.ctx._h, C.byref(d), self._row_values(grad_loss, logits, "grad_loss"), loss.data_ptr(), lse.data_ptr(),
            grad.data_ptr(), _rows(grad, "grad"), self._stream(stream)))
        return loss, lse, grad
