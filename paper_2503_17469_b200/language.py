"""Operators of a language model's training pass: embedding, head norms with rotation, attention, distillation and policy
losses; AdamW on the workers' gradients.

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
from array import array
from typing import Optional

import torch

from . import binding as B

_DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16}
_INDEX = {torch.int32: B.I32, torch.int64: B.I64}
_like, _float, _bf16, _byte = torch.empty_like, torch.float32, torch.bfloat16, torch.uint8
_numel, _contiguous, _where, _address = torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.get_device, torch.Tensor.data_ptr
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


class Rotary(_Operator):
    """Norms of query and key heads with the rotation by positions, on float32 or bfloat16 ``[batch, length, head, dim]`` tensors.

    ``frequencies``: radians per position of each rotated pair (``Rotary.geometric`` gives the usual ones), at most dim / 2;
    elements behind the pairs are not rotated.  ``axes``: the position axis of each pair, for positions of
    several axes (time, height, width).  ``interleaved``: pairs are neighbours, otherwise element i and i + pairs.  Any strides with a
    contiguous last dimension; 16-byte boundaries run faster.  Like its context, an object takes one call at a time."""

    def __init__(self, ctx: "B.Omni", heads: int, kv_heads: int, dim: int, frequencies, axes=None, interleaved: bool = False,
                 eps: float = 1e-6):
        super().__init__(ctx)
        frequencies = [float(f) for f in frequencies]
        axes = [0] * len(frequencies) if axes is None else [int(a) for a in axes]
        if heads < 1 or kv_heads < 1 or dim < 2 or dim % 2:
            raise ValueError("heads and kv_heads are at least 1, dim is even")
        if (heads | kv_heads | dim) >> 31:
            raise _too_large()
        if not 1 <= len(frequencies) <= dim // 2 or len(axes) != len(frequencies):
            raise ValueError("between 1 and dim / 2 frequencies, and an axis for each, are wanted")
        if min(axes) < 0 or max(axes) >= B.ROTARY_MAX_AXES:
            raise ValueError(f"axes are 0 to {B.ROTARY_MAX_AXES - 1}")
        if not 0.0 <= eps < float("inf"):
            raise ValueError("eps is finite and not negative")
        self.heads, self.kv_heads, self.dim, self.interleaved, self.eps = heads, kv_heads, dim, interleaved, eps
        self.frequencies, self.axes = frequencies, max(axes) + 1
        self._tables = ((C.c_double * len(frequencies))(*frequencies), (C.c_int32 * len(axes))(*axes))
        # What a call passes, made once and filled at each call: its fields' cost is most of a single token's.
        self._call = B.omni_rotary(0, 0, heads, kv_heads, dim, len(frequencies), self.axes, interleaved, 0, 0, 0, eps, *self._tables)
        self._call_ref = _ref(self._call)
        self._views = [B.omni_attn_view() for _ in range(6)]
        self._view_refs = [_ref(v) for v in self._views]

    @staticmethod
    def geometric(pairs: int, base: float = 10000.0):
        """base ** (-i / pairs), i = 0 .. pairs - 1."""
        return [base ** (-i / pairs) for i in range(pairs)]

    def _describe(self, q, k, positions, q_weight, k_weight, lengths):
        """Fills the call's sizes; (shape of the queries, shape of the keys, dtype, device)."""
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("q and k: [batch, length, head, dim] is wanted")
        batch, length = q.shape[:2]
        if (batch | length) >> 31:
            raise _too_large()
        device = q.get_device()
        if not q.is_cuda or not device == positions.get_device() == _device():
            raise _elsewhere(q=q, positions=positions)
        shape = positions.shape
        if shape == (batch, length) and self.axes == 1:
            axis, strides = 0, positions.stride()
        elif shape == (self.axes, batch, length):
            axis, *strides = positions.stride()
        else:
            raise ValueError(f"positions: shape {(self.axes, batch, length)} is wanted" + ", or without the first" * (self.axes == 1))
        weight, at = B.F32, (None, None)
        if q_weight is not None and k_weight is not None:
            weight, at = _code(q_weight, _DTYPES, "q_weight"), (q_weight.data_ptr(), k_weight.data_ptr())
            for w in (q_weight, k_weight):
                if w.shape != (self.dim,) or not w.is_contiguous() or w.dtype != q_weight.dtype or w.get_device() != device:
                    raise ValueError("q_weight and k_weight: contiguous [dim] of one dtype on the tensors' device is wanted")
        elif q_weight is not None or k_weight is not None:
            raise ValueError("q_weight and k_weight: both or neither")
        if lengths is not None and (lengths.dtype != torch.int32 or not lengths.is_contiguous() or lengths.shape != (batch,)
                                    or lengths.get_device() != device):
            raise ValueError("lengths: contiguous int32 [batch] on the tensors' device is wanted")
        r = self._call
        r.batch, r.length = batch, length
        r.dtype, r.weight_dtype, r.position_type = _code(q, _DTYPES, "q"), weight, _code(positions, _INDEX, "positions")
        r.positions, r.position_axis = positions.data_ptr(), axis
        r.position_batch, r.position_row = strides
        r.q_weight, r.k_weight = at
        r.lengths = None if lengths is None else lengths.data_ptr()
        return (batch, length, self.heads, self.dim), (batch, length, self.kv_heads, self.dim), q.dtype, device

    def _view(self, i: int, t, what: str, shape, dtype, device: int):
        if t.dtype is not dtype:
            raise TypeError(f"{what}: dtype {t.dtype} is not that of q, {dtype}")
        v = self._views[i]
        if t.shape != shape or t.get_device() != device:
            one = 0
        else:
            v.batch, v.row, v.head, one = t.stride()
        if one != 1:
            raise ValueError(f"{what}: shape {shape} with a contiguous last dimension on the current device is wanted, "
                             f"got {tuple(t.shape)}, strides {t.stride()}, on {t.device}")
        v.data = t.data_ptr()
        return self._view_refs[i]

    def forward(self, q, k, positions, q_weight=None, k_weight=None, lengths=None, out=None, stream=None):
        """Returns normed and rotated (q, k); into ``out``, a tuple of two, if given (q and k themselves, or places in a cache).
        ``positions``: int32 or int64 [batch, length], or [axes, batch, length], any strides.  Without weights there is no norm.
        Rows behind ``lengths`` (int32 [batch]) are zeros."""
        if stream is not None:
            with self._on_stream(stream):
                return self.forward(q, k, positions, q_weight, k_weight, lengths, out)
        rows, keys, dtype, device = self._describe(q, k, positions, q_weight, k_weight, lengths)
        view = self._view
        out_q, out_k = (_like(q), _like(k)) if out is None else out
        self._check(self._lib.omni_rotary_forward(
            self.ctx._h, self._call_ref, view(0, q, "q", rows, dtype, device), view(1, k, "k", keys, dtype, device),
            view(2, out_q, "out[0]", rows, dtype, device), view(3, out_k, "out[1]", keys, dtype, device), _raw_stream(device)))
        return out_q, out_k

    def backward(self, q, k, positions, grad_q, grad_k, q_weight=None, k_weight=None, lengths=None, grads=None, dtype=torch.float32,
                 weight_grads=None, stream=None):
        """Gradients of (q, k, q_weight, k_weight) from those of the forward call's results; q and k are the forward call's arguments.
        Into ``grads`` (a tuple of two; grad_q and grad_k themselves will do) and ``weight_grads`` (a tuple of two [dim]) if given;
        the weights' are of ``dtype`` otherwise, and None without weights."""
        if stream is not None:
            with self._on_stream(stream):
                return self.backward(q, k, positions, grad_q, grad_k, q_weight, k_weight, lengths, grads, dtype, weight_grads)
        rows, keys, kind, device = self._describe(q, k, positions, q_weight, k_weight, lengths)
        view = self._view
        dq, dk = (_like(q), _like(k)) if grads is None else grads
        if q_weight is None:
            dqw = dkw = scratch = None
            at, code, size = (None, None, None), B.F32, 0
        else:
            dqw, dkw = (q_weight.new_empty(self.dim, dtype=dtype) for _ in range(2)) if weight_grads is None else weight_grads
            code = _code(dqw, _DTYPES, "weight_grads")
            for w in (dqw, dkw):
                if w.shape != (self.dim,) or not w.is_contiguous() or w.dtype != dqw.dtype or w.get_device() != device:
                    raise ValueError("weight_grads: contiguous [dim] of one dtype on the current device is wanted")
            size = self._sizes.get(0)
            if size is None:
                need = C.c_uint64()
                self._check(self._lib.omni_rotary_workspace(self._call_ref, _ref(need)))
                size = self._sizes[0] = need.value
            scratch = q.new_empty(size, dtype=_byte)
            at = (dqw.data_ptr(), dkw.data_ptr(), scratch.data_ptr())
        self._check(self._lib.omni_rotary_backward(
            self.ctx._h, self._call_ref, view(0, q, "q", rows, kind, device), view(1, k, "k", keys, kind, device),
            view(2, grad_q, "grad_q", rows, kind, device), view(3, grad_k, "grad_k", keys, kind, device),
            view(4, dq, "grads[0]", rows, kind, device), view(5, dk, "grads[1]", keys, kind, device), at[0], at[1], code, at[2], size,
            _raw_stream(device)))
        return dq, dk, dqw, dkw


class Policy(_Operator):
    """Clipped policy loss on sampled tokens, with ``kl`` times a divergence from a reference policy, per row of logits.
    The ratio to the sampling policy is clipped to 1 - ``clip`` .. 1 + ``clip_high`` (default ``clip``).  A token of -1 marks a row
    without one (a prompt's, padding): loss 0, log-probability 0 and no gradient, whatever its other values are.  Like its context, an object
    takes one call at a time."""

    def __init__(self, ctx: "B.Omni", clip: float = 0.2, clip_high: Optional[float] = None, kl: float = 0.0, temperature: float = 1.0):
        super().__init__(ctx)
        high = clip if clip_high is None else clip_high
        if not (0 <= clip < float("inf") and 0 <= high < float("inf") and 0 <= kl < float("inf")):
            raise ValueError("clip, clip_high and kl are finite and not negative")
        if not temperature > 0:
            raise ValueError("temperature is positive")
        self.clip, self.clip_high, self.kl, self.temperature = clip, high, kl, temperature
        self._call = B.omni_policy()                  # filled at each call
        self._call_ref = _ref(self._call)

    def _describe(self, logits, tokens, valued: bool = False, old=None, advantage=None, reference=None):
        rows, vocab = logits.shape
        if tokens.shape != (rows,) or not tokens.is_contiguous():
            raise ValueError("logits [rows, vocab] and contiguous tokens [rows] are wanted")
        if vocab >> 31:
            raise _too_large()
        device = tokens.get_device()
        if not logits.is_cuda or not logits.get_device() == device == _device():
            raise _elsewhere(logits=logits, tokens=tokens)
        d, n = self._call, (rows,)
        d.logits, d.rows, d.row_stride, d.vocab, d.dtype = logits.data_ptr(), rows, _rows(logits, "logits"), vocab, _code(logits, _DTYPES, "logits")
        d.tokens, d.index_type, d.temperature = tokens.data_ptr(), _code(tokens, _INDEX, "tokens"), self.temperature
        if valued:
            d.clip_low, d.clip_high, d.kl = self.clip, self.clip_high, self.kl
            if old is None or advantage is None or (self.kl and reference is None):
                raise ValueError("old, advantage and, with kl, the reference's log-probabilities are wanted")
            d.old, d.advantage = self._row_values(old, n, device, "old"), self._row_values(advantage, n, device, "advantage")
            d.reference = self._row_values(reference, n, device, "reference") if self.kl else None
        return n, device

    @staticmethod
    def _row_values(t, shape, device: int, what: str) -> int:
        if t.dtype is not _float or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
            raise ValueError(f"{what}: contiguous float32 [rows] on the logits' device is wanted")
        return t.data_ptr()

    _grad_like = staticmethod(Distillation._grad_like)

    def logprob(self, logits, tokens, stream=None):
        """Returns (log-probabilities of the tokens, lse), float32 [rows] each: ``old`` and ``reference`` of the calls below come
        from here, with the logits of the sampling and of the reference policy."""
        if stream is not None:
            with self._on_stream(stream):
                return self.logprob(logits, tokens)
        n, device = self._describe(logits, tokens)
        logp = logits.new_empty(n, dtype=_float)
        lse = _like(logp)
        self._check(self._lib.omni_policy_logprob(self.ctx._h, self._call_ref, logp.data_ptr(), lse.data_ptr(), _raw_stream(device)))
        return logp, lse

    def forward(self, logits, tokens, old, advantage, reference=None, stream=None):
        """Returns (loss, log-probabilities, lse), float32 [rows] each.  ``old``, ``advantage``, ``reference`` (wanted if ``kl`` is
        not 0): float32 [rows]."""
        if stream is not None:
            with self._on_stream(stream):
                return self.forward(logits, tokens, old, advantage, reference)
        _, device = self._describe(logits, tokens, True, old, advantage, reference)
        loss, logp, lse = _like(old), _like(old), _like(old)
        self._check(self._lib.omni_policy_forward(self.ctx._h, self._call_ref, loss.data_ptr(), logp.data_ptr(), lse.data_ptr(),
                                                  _raw_stream(device)))
        return loss, logp, lse

    def backward(self, logits, tokens, lse, old, advantage, grad_loss, reference=None, grad=None, stream=None):
        """Gradient of the logits from ``lse`` of the forward call and ``grad_loss`` [rows]; ``grad`` may be ``logits``.  Rows that are far from
        zero (an ``lse`` or a token's logit of 128 and more), or whose ratio stands within rounding of a border, take their own sum instead, in one more walk."""
        if stream is not None:
            with self._on_stream(stream):
                return self.backward(logits, tokens, lse, old, advantage, grad_loss, reference, grad)
        n, device = self._describe(logits, tokens, True, old, advantage, reference)
        grad = self._grad_like(logits, grad)
        self._check(self._lib.omni_policy_backward(
            self.ctx._h, self._call_ref, self._row_values(lse, n, device, "lse"), self._row_values(grad_loss, n, device, "grad_loss"),
            grad.data_ptr(), _rows(grad, "grad"), _raw_stream(device)))
        return grad

    def step(self, logits, tokens, old, advantage, grad_loss, reference=None, grad=None, stream=None):
        """Forward and backward in one pass; returns (loss, log-probabilities, lse, gradient of the logits).  ``grad`` as in
        ``backward``."""
        if stream is not None:
            with self._on_stream(stream):
                return self.step(logits, tokens, old, advantage, grad_loss, reference, grad)
        n, device = self._describe(logits, tokens, True, old, advantage, reference)
        weights = self._row_values(grad_loss, n, device, "grad_loss")
        loss, logp, lse = _like(old), _like(old), _like(old)
        grad = self._grad_like(logits, grad)
        self._check(self._lib.omni_policy_step(self.ctx._h, self._call_ref, weights, loss.data_ptr(), logp.data_ptr(), lse.data_ptr(),
                                               grad.data_ptr(), _rows(grad, "grad"), _raw_stream(device)))
        return loss, logp, lse, grad


class AdamW(_Operator):
    """AdamW on a list of tensors, in one launch, from the batch-weighted gradients of K workers.

    ``params``: float32 tensors; ``grads[i][k]``: worker k's gradient of tensor i, float32 or bfloat16; ``copies``: bfloat16 tensors
    that receive the rounded parameters, or None.  All contiguous, of the current device, and kept alive by this object, which
    notes where they lie: they are updated in place and are not to be replaced, and a graph that a step was captured into needs the object
    for as long as it is replayed.  ``weight_decay``: one for all or one for each.
    ``bits``: 32, or 8 for moments in one byte each with stochastic rounding (formats and formulas in ``include/omni.h``).
    ``state``: (m, v) float32 tensors, or (m, v, tops) uint8, uint8 and int16 [blocks, 2], for each tensor, to go on from; zeros
    by default.  ``state`` and ``steps`` (how many have been made) are what a checkpoint holds."""

    def __init__(self, ctx: "B.Omni", params, grads, copies=None, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, bits: int = 32,
                 state=None, steps: int = 0):
        super().__init__(ctx)
        params, grads = list(params), [list(g) for g in grads]
        copies = [None] * len(params) if copies is None else list(copies)
        decay = [float(weight_decay)] * len(params) if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        if bits not in (8, 32):
            raise ValueError("bits are 8 or 32")
        if not len(params) == len(grads) == len(copies) == len(decay):
            raise ValueError("params, grads, copies and weight_decay: as many of each are wanted")
        if not (0 <= betas[0] < 1 and 0 <= betas[1] < 1 and 0 <= eps < float("inf")) or steps < 0:
            raise ValueError("betas are in [0, 1), eps is finite and not negative, steps is not negative")
        self.K = len(grads[0]) if grads else 1
        if not 1 <= self.K <= B.MAX_K or any(len(g) != self.K for g in grads):
            raise ValueError(f"every tensor has the gradients of as many workers, 1 to {B.MAX_K}")
        self._at = _device()
        if state is None:
            state = [self._zeros(p, bits) for p in params]
        self.state = [tuple(s) for s in state]
        if len(self.state) != len(params):
            raise ValueError("state: as many as params are wanted")
        dtype = grads[0][0].dtype if grads else _float
        code = B.F32 if not grads else _code(grads[0][0], _DTYPES, "grads")
        moments = (_float, _float) if bits == 32 else (_byte, _byte, torch.int16)
        described = (B.omni_adamw_tensor * max(1, len(params)))()
        self._tables = []
        for i, (p, gs, c, s) in enumerate(zip(params, grads, copies, self.state)):
            n, shape = p.numel(), p.shape
            if len(s) != len(moments):
                raise ValueError(f"state[{i}]: {len(moments)} tensors are wanted")
            blocks = torch.Size((-(-n // B.ADAMW_BLOCK), 2))
            for what, t, kind, size in (("params", p, _float, shape), ("copies", c, _bf16, shape), *(("grads", g, dtype, shape) for g in gs),
                                        *(("state", t, kind, blocks if kind == torch.int16 else shape) for t, kind in zip(s, moments))):
                if t is None and what == "copies":
                    continue
                if t.dtype != kind:
                    raise TypeError(f"{what}[{i}]: dtype {t.dtype}, {kind} is wanted")
                if t.shape != size or not t.is_contiguous():
                    raise ValueError(f"{what}[{i}]: a contiguous tensor of shape {tuple(size)} is wanted, got {tuple(t.shape)}, strides {t.stride()}")
                if not t.is_cuda or t.get_device() != self._at:
                    raise _elsewhere(**{what: t})
            table = (C.c_void_p * self.K)(*(g.data_ptr() for g in gs))
            self._tables.append(table)
            described[i] = B.omni_adamw_tensor(p.data_ptr(), None if c is None else c.data_ptr(), table, s[0].data_ptr(), s[1].data_ptr(),
                                               s[2].data_ptr() if bits == 8 else None, n, decay[i])
        self._keep = (params, grads, copies)
        self.betas, self.eps, self.bits, self.steps = (float(betas[0]), float(betas[1])), float(eps), bits, int(steps)
        need = C.c_uint64()
        self._check(self._lib.omni_adamw_plan_bytes(described, len(params), self.K, code, bits, _ref(need)))
        host = torch.empty(need.value, dtype=_byte)
        self._check(self._lib.omni_adamw_plan(described, len(params), self.K, code, bits, host.data_ptr(), need.value))
        self._record = host
        self._record_dev = host.to(f"cuda:{self._at}")
        self._batches = C.c_int32 * self.K
        self._numels, self._pointers = [p.numel() for p in params], C.c_void_p * max(1, len(params))

    @staticmethod
    def _zeros(p, bits):
        if bits == 32:
            return tuple(torch.zeros(p.shape, dtype=_float, device=p.device) for _ in range(2))
        return (*(torch.zeros(p.shape, dtype=_byte, device=p.device) for _ in range(2)),
                torch.zeros((-(-p.numel() // B.ADAMW_BLOCK), 2), dtype=torch.int16, device=p.device))

    def step(self, lr: float, batches=None, clock=None, stream=None) -> None:
        """One step with the gradients that lie in ``grads`` now.  ``batches``: the K workers' batch sizes (of one worker: not needed).
        The step's number is ``steps`` + 1, which ``steps`` becomes; with ``clock``, an int64 tensor of one element on the device, it is what
        that holds when the step runs (1 for the first), and ``steps`` stays: for a captured graph that also adds 1 to the clock."""
        if batches is None:
            if self.K > 1:
                raise ValueError("batches: the workers' batch sizes are wanted")
            batches = (1,)
        if len(batches) != self.K:
            raise ValueError(f"batches: {self.K} of them are wanted")
        if sum(batches) >> 31 and any(b >> 31 not in (0, -1) for b in batches):       # the sum first: a fifth of the time
            raise _too_large()
        if self._at != _device():
            raise _elsewhere(params=self._record_dev)
        at = None
        if clock is not None:
            if clock.dtype != torch.int64 or clock.numel() != 1 or clock.get_device() != self._at:
                raise ValueError("clock: an int64 tensor of one element on the current device is wanted")
            at = clock.data_ptr()
        raw = _raw_stream(self._at) if stream is None else stream.cuda_stream
        self._check(self._lib.omni_adamw_step(self.ctx._h, self._record.data_ptr(), self._record_dev.data_ptr(), self._batches(*batches), lr,
                                              *self.betas, self.eps, self.steps + 1, at, raw))
        if clock is None:
            self.steps += 1

    def moments(self, out=None, stream=None):
        """[(m, v)] as float32, for each tensor: the state itself at 32 bits, at 8 bits what its codes stand for, into ``out`` if given."""
        if stream is not None:
            with self._on_stream(stream):
                return self.moments(out)
        if self._at != _device():
            raise _elsewhere(params=self._record_dev)
        if self.bits == 32:
            if out is None:
                return list(self.state)
            raise ValueError("out: moments of 32 bits are the state itself")
        if out is None:
            out = [tuple(torch.empty(s[0].shape, dtype=_float, device=s[0].device) for _ in range(2)) for s in self.state]
        # many short tensors: by functions that run over all of them, not tensor by tensor
        m, v = tuple(zip(*out)) or ((), ())
        tables = []
        for t in (m, v):
            if list(map(_numel, t)) != self._numels or not all(map(_contiguous, t)) or not {x.dtype for x in t} <= {_float} \
                    or not set(map(_where, t)) <= {self._at}:
                raise ValueError("out: for each tensor a pair of contiguous float32 tensors of its size on the current device is wanted")
            tables.append(self._pointers.from_buffer(array("Q", map(_address, t) if t else (0,))))
        self._check(self._lib.omni_adamw_moments(self.ctx._h, self._record.data_ptr(), self._record_dev.data_ptr(), *tables, _raw_stream(self._at)))
        return out
