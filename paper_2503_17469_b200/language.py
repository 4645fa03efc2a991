"""Operators of a language model's training pass: embedding, attention, distillation loss.

What a worker computes its gradients with, on torch tensors of the current CUDA device.  Each class keeps an
operator's constants and an ``Omni`` context (launch counts, errors, the status word of bounded
waits); its calls allocate their outputs with torch unless they are given, take scratch memory from torch's
caching allocator, enqueue on ``stream`` (a torch stream, default the current one) and do not
synchronise.  The formulas, types and limits stand in ``include/omni.h``.  There is no fallback.

The results carry no autograd graph, whatever the arguments require: a call is one direction, and the gradients are the
``backward`` and ``step`` calls' (inside a ``torch.autograd.Function``, for example).  Tensors that belong to another stream than
``stream`` are the caller's to order and to keep, as with torch's own calls.  A captured graph takes the host's part off
short calls; the context has to have been used before the capture.

Arguments that do not fit together raise ``ValueError`` or ``TypeError`` before anything is
enqueued; what the library refuses raises ``OmniError``.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from . import binding as B

_DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16}
_INDEX = {torch.int32: B.I32, torch.int64: B.I64}
_like, _float, _bf16, _byte = torch.empty_like, torch.float32, torch.bfloat16, torch.uint8
_ref = C.byref


# The current device, and the raw handle of its current stream (what ``Omni._stream`` wraps) without an object around it.
_device = torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)


def _code(t, codes, what: str) -> int:
    c = codes.get(t.dtype)
    if c is None:
        raise TypeError(f"{what}: dtype {t.dtype} is none of {', '.join(map(str, codes))}")
    return c


def _elsewhere(**tensors):
    """For the messages of tensors that are not on the current device, whose stream takes the call."""
    return ValueError(", ".join(f"{k} on {t.device}" for k, t in tensors.items() if t is not None) + ": the current CUDA device is wanted")


def _too_large():
    """For sizes that the library takes as 32 bits: ctypes would cut them."""
    return ValueError("a size of 2**31 or more")


def _rows(t, what: str) -> int:
    """Stride between the rows of a matrix whose rows are contiguous; that of a single row is its length, whatever it was cut from."""
    n, m = t.shape
    stride, one = t.stride()
    if one != 1 and m > 1:
        raise ValueError(f"{what}: contiguous rows are wanted, got strides {t.stride()}")
    return stride if n > 1 else m


# The checks below stand in the calls themselves, without helpers and keyword arguments, and a
# message is only put together where it is raised: a call's host time is most of a short operator's.
class _Operator:
    def __init__(self, ctx: "B.Omni"):
        self.ctx = ctx
        self._lib = B.lib()
        self._sizes = {}       # scratch bytes by problem size

    @staticmethod
    def _on_stream(stream):
        """Outputs and scratch belong to the stream that uses them."""
        return torch.cuda.stream(stream)

    def _check(self, rc: int) -> None:
        if rc != B.OK:
            self.ctx._check(rc)


class Embedding(_Operator):
    """Lookup ``scale * weight[tokens]`` and its dense gradient.  ``padding``: a token that gets no gradient."""

    def __init__(self, ctx: "B.Omni", vocab: int, dim: int, scale: float = 1.0, padding: int = -1):
        super().__init__(ctx)
        if vocab < 1 or dim < 1:
            raise ValueError("vocab and dim are at least 1")
        if (vocab | dim) >> 31:
            raise _too_large()
        self.vocab, self.dim, self.scale, self.padding = vocab, dim, scale, padding
        self._table = torch.Size((vocab, dim))

    def forward(self, tokens, weight, dtype=None, out=None, stream=None):
        """``tokens``: int32 or int64, any shape, contiguous; ``weight``: [vocab, dim] float32 or bfloat16.
        Returns ``tokens.shape + (dim,)`` of ``dtype`` (default the table's)."""
        if stream is not None:
            with self._on_stream(stream):
                return self.forward(tokens, weight, dtype, out)
        shape = (*tokens.shape, self.dim)
        if out is None:
            out = weight.new_empty(shape, dtype=dtype or weight.dtype)
        elif out.shape != shape or not out.is_contiguous():
            raise ValueError(f"out: a contiguous tensor of shape {shape} is wanted")
        if weight.shape != self._table:
            raise ValueError(f"weight: shape {tuple(self._table)} is wanted")
        if not tokens.is_contiguous():
            raise ValueError("tokens: a contiguous tensor is wanted")
        device = tokens.get_device()
        if not tokens.is_cuda or not weight.get_device() == out.get_device() == device == _device():
            raise _elsewhere(tokens=tokens, weight=weight, out=out)
        self._check(self._lib.omni_embed_forward(
            self.ctx._h, tokens.data_ptr(), _code(tokens, _INDEX, "tokens"), tokens.numel(), weight.data_ptr(),
            _code(weight, _DTYPES, "weight"), _rows(weight, "weight"), self.vocab, self.dim, self.scale, out.data_ptr(),
            _code(out, _DTYPES, "out"), self.dim, _raw_stream(device)))
        return out

    def backward(self, tokens, grad_out, dtype=torch.float32, grad=None, accumulate: bool = False, stream=None):
        """Gradient of the table, [vocab, dim] of ``dtype``; into ``grad`` if given (for example a view of a
        gradient bucket), added to it with ``accumulate``.  ``grad_out``: ``tokens.shape + (dim,)``,
        or a matrix of as many rows, rows contiguous."""
        if stream is not None:
            with self._on_stream(stream):
                return self.backward(tokens, grad_out, dtype, grad, accumulate)
        n = tokens.numel()
        try:
            g = grad_out if grad_out.dim() == 2 else grad_out.view(n, self.dim)
        except RuntimeError:           # other sizes, or strides that are no matrix's
            g = None
        if g is None or g.shape != (n, self.dim):
            raise ValueError(f"grad_out: {n} rows of {self.dim} are wanted")
        if not tokens.is_contiguous():
            raise ValueError("tokens: a contiguous tensor is wanted")
        if grad is None:
            if accumulate:
                raise ValueError("accumulate needs a gradient to add to")
            grad = g.new_empty(self._table, dtype=dtype)
        elif grad.shape != self._table:
            raise ValueError(f"grad: shape {tuple(self._table)} is wanted")
        device = tokens.get_device()
        if not tokens.is_cuda or not g.get_device() == grad.get_device() == device == _device():
            raise _elsewhere(tokens=tokens, grad_out=g, grad=grad)
        size = self._sizes.get(n)
        if size is None:
            need = C.c_uint64()
            self._check(self._lib.omni_embed_workspace(n, self.vocab, self.dim, _ref(need)))
            size = self._sizes[n] = max(16, need.value)
        scratch = g.new_empty(size, dtype=_byte)
        self._check(self._lib.omni_embed_backward(
            self.ctx._h, tokens.data_ptr(), _code(tokens, _INDEX, "tokens"), n, g.data_ptr(),
            _code(g, _DTYPES, "grad_out"), _rows(g, "grad_out"), self.vocab, self.dim, self.scale, self.padding,
            grad.data_ptr(), _code(grad, _DTYPES, "grad"), _rows(grad, "grad"), accumulate, scratch.data_ptr(),
            size, _raw_stream(device)))
        return grad


class Attention(_Operator):
    """Softmax attention on bfloat16 ``[batch, length, head, dim]`` tensors, forward and backward.

    ``heads`` query heads share ``kv_heads`` key/value heads in groups; ``causal`` aligns queries and
    keys at their ends; ``scale`` defaults to dim ** -0.5.  Any strides with a contiguous last
    dimension, multiples of 8 elements (slices of one projection's output, for example)."""

    def __init__(self, ctx: "B.Omni", heads: int, kv_heads: int, dim: int, causal: bool = True, scale: Optional[float] = None):
        super().__init__(ctx)
        if heads < 1 or kv_heads < 1 or heads % kv_heads:
            raise ValueError("heads is a multiple of kv_heads")
        if (heads | dim) >> 31:
            raise _too_large()
        self.heads, self.kv_heads, self.dim, self.causal = heads, kv_heads, dim, causal
        self.scale = dim ** -0.5 if scale is None else scale

    def _describe(self, q, k, q_lengths, kv_lengths):
        """(sizes, shape of the query side, shape of the key side) of a call."""
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("q and k: [batch, length, head, dim] is wanted")
        batch, q_len = q.shape[:2]
        kv_len = k.shape[1]
        if (batch | q_len | kv_len) >> 31:
            raise _too_large()
        if not q.is_cuda or q.get_device() != _device():
            raise _elsewhere(q=q)
        at = [None, None]
        for i, t in enumerate((q_lengths, kv_lengths)):
            if t is not None:
                if t.dtype != torch.int32 or not t.is_contiguous() or t.shape != (batch,) or t.get_device() != q.get_device():
                    raise ValueError("q_lengths and kv_lengths: contiguous int32 [batch] on the tensors' device is wanted")
                at[i] = t.data_ptr()
        return (B.omni_attn(batch, q_len, kv_len, self.heads, self.kv_heads, self.dim, self.causal, self.scale, *at),
                (batch, q_len, self.heads, self.dim), (batch, kv_len, self.kv_heads, self.dim))

    @staticmethod
    def _view(t, what: str, shape, device: int):
        if t.dtype != _bf16:
            raise TypeError(f"{what}: dtype {t.dtype} is not bfloat16")
        batch, row, head, one = t.stride()
        if t.shape != shape or one != 1 or t.get_device() != device:
            raise ValueError(f"{what}: shape {shape} with a contiguous last dimension on the current device is wanted, "
                             f"got {tuple(t.shape)}, strides {t.stride()}, on {t.device}")
        return B.omni_attn_view(t.data_ptr(), batch, row, head)

    def _scratch_bytes(self, query, a, rows, kv_len, forward: bool) -> int:
        key = (forward, rows[0], rows[1], kv_len)
        size = self._sizes.get(key)
        if size is None:
            need = C.c_uint64()
            self._check(query(_ref(a), _ref(need)))
            size = self._sizes[key] = need.value
        return size

    def forward(self, q, k, v, q_lengths=None, kv_lengths=None, out=None, stream=None):
        """Returns (out like q, lse float32 [batch, heads, q_len])."""
        if stream is not None:
            with self._on_stream(stream):
                return self.forward(q, k, v, q_lengths, kv_lengths, out)
        a, rows, keys = self._describe(q, k, q_lengths, kv_lengths)
        device, view = q.get_device(), self._view
        if out is None:
            out = _like(q)
        lse = q.new_empty((rows[0], self.heads, rows[1]), dtype=_float)
        size = self._scratch_bytes(self._lib.omni_attn_forward_workspace, a, rows, keys[1], True)
        scratch = q.new_empty(size, dtype=_byte) if size else None
        self._check(self._lib.omni_attn_forward(
            self.ctx._h, _ref(a), _ref(view(q, "q", rows, device)), _ref(view(k, "k", keys, device)),
            _ref(view(v, "v", keys, device)), _ref(view(out, "out", rows, device)), lse.data_ptr(),
            scratch.data_ptr() if size else None, size, _raw_stream(device)))
        return out, lse

    def backward(self, q, k, v, out, lse, grad_out, q_lengths=None, kv_lengths=None, grads=None, stream=None):
        """Returns the gradients of (q, k, v); into ``grads``, a tuple of three, if given.  ``out`` and
        ``lse`` are the forward call's."""
        if stream is not None:
            with self._on_stream(stream):
                return self.backward(q, k, v, out, lse, grad_out, q_lengths, kv_lengths, grads)
        a, rows, keys = self._describe(q, k, q_lengths, kv_lengths)
        device, view = q.get_device(), self._view
        if lse.dtype != _float or not lse.is_contiguous() or lse.shape != (rows[0], self.heads, rows[1]) or lse.get_device() != device:
            raise ValueError("lse: contiguous float32 [batch, heads, q_len] is wanted")
        if grads is None:
            grads = (_like(q), _like(k), _like(v))
        size = self._scratch_bytes(self._lib.omni_attn_workspace, a, rows, keys[1], False)
        scratch = q.new_empty(max(16, size), dtype=_byte)
        dq, dk, dv = grads
        self._check(self._lib.omni_attn_backward(
            self.ctx._h, _ref(a), _ref(view(q, "q", rows, device)), _ref(view(k, "k", keys, device)),
            _ref(view(v, "v", keys, device)), _ref(view(out, "out", rows, device)), lse.data_ptr(),
            _ref(view(grad_out, "grad_out", rows, device)), _ref(view(dq, "grads[0]", rows, device)),
            _ref(view(dk, "grads[1]", keys, device)), _ref(view(dv, "grads[2]", keys, device)), scratch.data_ptr(), size,
            _raw_stream(device)))
        return dq, dk, dv


class Distillation(_Operator):
    """KL divergence (times temperature squared) of the student's softmax from a teacher's top logits, per row.
    An index of -1 marks an entry that is not there; a row without entries has loss 0 and no gradient."""

    def __init__(self, ctx: "B.Omni", temperature: float = 1.0):
        super().__init__(ctx)
        if not temperature > 0:
            raise ValueError("temperature is positive")
        self.temperature = temperature

    def _describe(self, logits, top_logits, top_index):
        if top_logits.dtype != _float:
            raise TypeError("top_logits: float32 is wanted")
        rows, vocab = logits.shape
        n, top = top_logits.shape
        if n != rows or top_index.shape != (n, top):
            raise ValueError("logits [rows, vocab], top_logits and top_index [rows, top] are wanted")
        if (vocab | top) >> 31:
            raise _too_large()
        stride = _rows(top_logits, "top_logits")
        if _rows(top_index, "top_index") != stride:
            raise ValueError("top_logits and top_index: the same stride is wanted")
        if not logits.is_cuda or not logits.get_device() == top_logits.get_device() == top_index.get_device() == _device():
            raise _elsewhere(logits=logits, top_logits=top_logits, top_index=top_index)
        return B.omni_distill(logits.data_ptr(), rows, _rows(logits, "logits"), vocab, _code(logits, _DTYPES, "logits"),
                              top_logits.data_ptr(), top_index.data_ptr(), stride, top, _code(top_index, _INDEX, "top_index"),
                              self.temperature)

    @staticmethod
    def _row_values(t, logits, what: str) -> int:
        if t.dtype != _float or not t.is_contiguous() or t.shape != logits.shape[:1] or t.get_device() != logits.get_device():
            raise ValueError(f"{what}: contiguous float32 [rows] on the logits' device is wanted")
        return t.data_ptr()

    @staticmethod
    def _grad_like(logits, grad):
        if grad is None:
            return _like(logits)
        if grad.shape != logits.shape or grad.dtype != logits.dtype or grad.get_device() != logits.get_device():
            raise ValueError("grad: the logits' shape, dtype and device are wanted")
        return grad

    def forward(self, logits, top_logits, top_index, stream=None):
        """Returns (loss, lse), float32 [rows] each."""
        if stream is not None:
            with self._on_stream(stream):
                return self.forward(logits, top_logits, top_index)
        d = self._describe(logits, top_logits, top_index)
        loss = logits.new_empty(d.rows, dtype=_float)
        lse = _like(loss)
        self._check(self._lib.omni_distill_forward(self.ctx._h, _ref(d), loss.data_ptr(), lse.data_ptr(), _raw_stream(logits.get_device())))
        return loss, lse

    def backward(self, logits, top_logits, top_index, lse, grad_loss, grad=None, stream=None):
        """Gradient of the logits from ``lse`` of the forward call and ``grad_loss`` [rows]; ``grad`` may be ``logits``.

        Without ``grad`` the result is dense.  For logits that are columns of wider rows (a padded vocabulary) a ``grad`` of
        the logits' own strides is written faster: 8192 x 50257 bfloat16 of 50304, 301 against 1412 us, a ``step`` 319 against 873."""
        if stream is not None:
            with self._on_stream(stream):
                return self.backward(logits, top_logits, top_index, lse, grad_loss, grad)
        d = self._describe(logits, top_logits, top_index)
        grad = self._grad_like(logits, grad)
        self._check(self._lib.omni_distill_backward(
            self.ctx._h, _ref(d), self._row_values(lse, logits, "lse"), self._row_values(grad_loss, logits, "grad_loss"),
            grad.data_ptr(), _rows(grad, "grad"), _raw_stream(logits.get_device())))
        return grad

    def step(self, logits, top_logits, top_index, grad_loss, grad=None, stream=None):
        """Forward and backward in one pass; returns (loss, lse, gradient of the logits).  ``grad`` as in ``backward``."""
        if stream is not None:
            with self._on_stream(stream):
                return self.step(logits, top_logits, top_index, grad_loss, grad)
        d = self._describe(logits, top_logits, top_index)
        weights = self._row_values(grad_loss, logits, "grad_loss")
        loss, lse = _like(grad_loss), _like(grad_loss)
        grad = self._grad_like(logits, grad)
        self._check(self._lib.omni_distill_step(self.ctx._h, _ref(d), weights, loss.data_ptr(), lse.data_ptr(),
                                                grad.data_ptr(), _rows(grad, "grad"), _raw_stream(logits.get_device())))
        return loss, lse, grad
