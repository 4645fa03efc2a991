"""What the language-model operators check before they touch a device: status codes and workspace sizes, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

PTR = 1 << 20        # an aligned address that no call here gets to use


@pytest.fixture(scope="module")
def omni():
    return B.Omni(1, 1, 1, 1)


def embed_args(**kw):
    a = dict(tokens=PTR, index=B.I64, n=4, rows=PTR, rows_dtype=B.F32, rows_stride=8, vocab=10, dim=8, scale=1.0, table=PTR,
             table_dtype=B.F32, table_stride=8)
    a.update(kw)
    return a


def embed_forward(ctx, **kw):
    a = embed_args(**kw)
    return B.lib().omni_embed_forward(ctx, a["tokens"], a["index"], a["n"], a["table"], a["table_dtype"], a["table_stride"],
                                      a["vocab"], a["dim"], a["scale"], a["rows"], a["rows_dtype"], a["rows_stride"], None)


def embed_backward(ctx, workspace=PTR, size=1 << 30, **kw):
    a = embed_args(**kw)
    return B.lib().omni_embed_backward(ctx, a["tokens"], a["index"], a["n"], a["rows"], a["rows_dtype"], a["rows_stride"],
                                       a["vocab"], a["dim"], a["scale"], -1, a["table"], a["table_dtype"], a["table_stride"], 0,
                                       workspace, size, None)


@pytest.mark.parametrize("call", [embed_forward, embed_backward])
@pytest.mark.parametrize("change,status", [
    (dict(index=2), B.ERR_BAD_CONFIG), (dict(rows_dtype=2), B.ERR_BAD_CONFIG), (dict(table_dtype=-1), B.ERR_BAD_CONFIG),
    (dict(vocab=0), B.ERR_BAD_CONFIG), (dict(dim=0), B.ERR_BAD_CONFIG), (dict(rows_stride=7), B.ERR_BAD_CONFIG),
    (dict(table_stride=7), B.ERR_BAD_CONFIG), (dict(scale=float("inf")), B.ERR_BAD_CONFIG), (dict(tokens=None), B.ERR_NULL),
    (dict(rows=None), B.ERR_NULL), (dict(table=None), B.ERR_NULL), (dict(n=1 << 31), B.ERR_TOO_LARGE),
    (dict(tokens=PTR + 4), B.ERR_ALIGN), (dict(rows=PTR + 2), B.ERR_ALIGN), (dict(table=PTR + 1), B.ERR_ALIGN),
])
def test_embedding_refuses(omni, call, change, status):
    assert call(omni._h, **change) == status
    assert call(None) == B.ERR_NULL


def test_embedding_workspace(omni):
    size = C.c_uint64()
    sizes = []
    for n in (0, 1, 300, 70000):
        assert B.lib().omni_embed_workspace(n, 10, 8, C.byref(size)) == B.OK
        sizes.append(size.value)
        assert embed_backward(omni._h, n=n, size=size.value - 1) == B.ERR_TOO_LARGE
    assert sizes == sorted(sizes) and sizes[3] >= 2 * 8 * 70000
    assert embed_backward(omni._h, workspace=None) == B.ERR_NULL and embed_backward(omni._h, workspace=PTR + 8) == B.ERR_ALIGN
    assert B.lib().omni_embed_workspace(1 << 31, 1, 1, C.byref(size)) == B.ERR_TOO_LARGE
    assert B.lib().omni_embed_workspace(1, 0, 1, C.byref(size)) == B.ERR_BAD_CONFIG
    assert B.lib().omni_embed_workspace(1, 1, 1, None) == B.ERR_NULL


def attn(**kw):
    a = dict(batch=2, q_len=5, kv_len=7, heads=4, kv_heads=2, dim=64, causal=1, scale=0.1, q_lengths=None, kv_lengths=None)
    a.update(kw)
    return B.omni_attn(*a.values())


def attn_forward(ctx, a, lse=PTR, change=None, workspace=PTR, size=1 << 30):
    v = [B.omni_attn_view(PTR, 5 * 256, 256, 64), B.omni_attn_view(PTR, 7 * 128, 128, 64), B.omni_attn_view(PTR, 7 * 128, 128, 64),
         B.omni_attn_view(PTR, 5 * 256, 256, 64)]
    for i, view in (change or {}).items():
        v[i] = view
    return B.lib().omni_attn_forward(ctx, C.byref(a), *(None if x is None else C.byref(x) for x in v), lse, workspace, size, None)


@pytest.mark.parametrize("change,status", [
    (dict(heads=3), B.ERR_BAD_CONFIG), (dict(kv_heads=0), B.ERR_BAD_CONFIG), (dict(batch=-1), B.ERR_BAD_CONFIG),
    (dict(q_len=-1), B.ERR_BAD_CONFIG), (dict(dim=60), B.ERR_BAD_CONFIG), (dict(dim=0), B.ERR_BAD_CONFIG),
    (dict(scale=0.0), B.ERR_BAD_CONFIG), (dict(scale=float("nan")), B.ERR_BAD_CONFIG), (dict(dim=136), B.ERR_TOO_LARGE),
    (dict(batch=65536), B.ERR_TOO_LARGE), (dict(heads=131072), B.ERR_TOO_LARGE), (dict(kv_len=(1 << 30) + 1), B.ERR_TOO_LARGE),
    (dict(q_lengths=PTR + 2), B.ERR_ALIGN),
])
def test_attention_refuses_sizes(omni, change, status):
    size = C.c_uint64()
    assert attn_forward(omni._h, attn(**change)) == status
    assert B.lib().omni_attn_workspace(C.byref(attn(**change)), C.byref(size)) == status


@pytest.mark.parametrize("view,status", [
    (None, B.ERR_NULL), (B.omni_attn_view(None, 2048, 256, 64), B.ERR_NULL), (B.omni_attn_view(PTR + 8, 2048, 256, 64), B.ERR_ALIGN),
    (B.omni_attn_view(PTR, 2048, 260, 64), B.ERR_ALIGN), (B.omni_attn_view(PTR, 2048, 256, 56), B.ERR_BAD_CONFIG),
    (B.omni_attn_view(PTR, 1 << 38, 256, 64), B.ERR_TOO_LARGE),
])
def test_attention_refuses_operands(omni, view, status):
    for i in range(4):
        assert attn_forward(omni._h, attn(), change={i: view}) == status
    assert attn_forward(omni._h, attn(), lse=None) == B.ERR_NULL and attn_forward(omni._h, attn(), lse=PTR + 2) == B.ERR_ALIGN
    assert attn_forward(None, attn()) == B.ERR_NULL
    few = attn(batch=1, kv_len=5000)           # one pair of query tiles per head: the keys are split
    keys = B.omni_attn_view(PTR, 5000 * 128, 128, 64)
    size = C.c_uint64()
    assert B.lib().omni_attn_forward_workspace(C.byref(few), C.byref(size)) == B.OK and size.value > 5 * 4 * 64 * 4
    for workspace, n, status in ((None, size.value, B.ERR_NULL), (PTR + 8, size.value, B.ERR_ALIGN), (PTR, size.value - 1, B.ERR_TOO_LARGE)):
        assert attn_forward(omni._h, few, change={1: keys, 2: keys}, workspace=workspace, size=n) == status
    assert B.lib().omni_attn_forward_workspace(C.byref(attn(batch=100)), C.byref(size)) == B.OK and size.value == 0


def test_attention_backward_workspace(omni):
    size = C.c_uint64()
    assert B.lib().omni_attn_workspace(C.byref(attn()), C.byref(size)) == B.OK and size.value >= 2 * 2 * 4 * 128 * 4
    rows, keys = C.byref(B.omni_attn_view(PTR, 5 * 256, 256, 64)), C.byref(B.omni_attn_view(PTR, 7 * 128, 128, 64))

    def call(workspace, n, lse=PTR):
        return B.lib().omni_attn_backward(omni._h, C.byref(attn()), rows, keys, keys, rows, lse, rows, rows, keys, keys, workspace, n, None)

    assert call(PTR, size.value - 1) == B.ERR_TOO_LARGE and call(None, size.value) == B.ERR_NULL
    assert call(PTR, size.value, None) == B.ERR_NULL and call(PTR + 8, size.value) == B.ERR_ALIGN


def distill(**kw):
    d = dict(logits=PTR, rows=3, row_stride=50, vocab=50, dtype=B.F32, top_logits=PTR, top_index=PTR, top_stride=4, top=4,
             index_type=B.I64, temperature=1.0)
    d.update(kw)
    return C.byref(B.omni_distill(*d.values()))


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), B.ERR_BAD_CONFIG), (dict(index_type=2), B.ERR_BAD_CONFIG), (dict(vocab=0), B.ERR_BAD_CONFIG),
    (dict(top=0), B.ERR_BAD_CONFIG), (dict(temperature=0.0), B.ERR_BAD_CONFIG), (dict(temperature=float("nan")), B.ERR_BAD_CONFIG),
    (dict(row_stride=49), B.ERR_BAD_CONFIG), (dict(top_stride=3), B.ERR_BAD_CONFIG), (dict(top=257, top_stride=300), B.ERR_TOO_LARGE),
    (dict(rows=1 << 31), B.ERR_TOO_LARGE), (dict(logits=None), B.ERR_NULL), (dict(top_logits=None), B.ERR_NULL),
    (dict(logits=PTR + 2), B.ERR_ALIGN), (dict(top_index=PTR + 4), B.ERR_ALIGN),
])
def test_distillation_refuses(omni, change, status):
    lib = B.lib()
    assert lib.omni_distill_forward(omni._h, distill(**change), PTR, PTR, None) == status
    assert lib.omni_distill_backward(omni._h, distill(**change), PTR, PTR, PTR, 50, None) == status
    assert lib.omni_distill_step(omni._h, distill(**change), PTR, PTR, PTR, PTR, 50, None) == status


def test_distillation_refuses_outputs(omni):
    lib = B.lib()
    assert lib.omni_distill_forward(omni._h, distill(), None, PTR, None) == B.ERR_NULL
    assert lib.omni_distill_forward(omni._h, None, PTR, PTR, None) == B.ERR_NULL
    assert lib.omni_distill_forward(None, distill(), PTR, PTR, None) == B.ERR_NULL
    assert lib.omni_distill_backward(omni._h, distill(), None, PTR, PTR, 50, None) == B.ERR_NULL
    assert lib.omni_distill_backward(omni._h, distill(), PTR, PTR, PTR, 49, None) == B.ERR_BAD_CONFIG
    assert lib.omni_distill_step(omni._h, distill(), PTR, PTR + 2, PTR, PTR, 50, None) == B.ERR_ALIGN


def test_host_tensors_are_refused(omni):
    t, w = torch.zeros(3, dtype=torch.int64), torch.zeros(5, 8)
    with pytest.raises(ValueError):
        L.Embedding(omni, 5, 8).forward(t, w)
    with pytest.raises(ValueError):
        L.Embedding(omni, 5, 8).backward(t, torch.zeros(3, 8))
    q = torch.zeros(1, 3, 2, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        L.Attention(omni, 2, 2, 8).forward(q, q, q)
    with pytest.raises(ValueError):
        L.Distillation(omni).forward(w, torch.zeros(5, 2), torch.zeros(5, 2, dtype=torch.int64))
