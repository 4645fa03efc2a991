"""Ways through the language-model operators that depend on sizes, on the context and on capture: several rows a group in the
lookup, tables with gaps between their rows, a third pass of the sort, large tables, captured graphs, contexts without
dependent launches.  Tolerances are those of test_gpu_embedding.py; what has to be the same is compared bit by bit."""
import gc

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

from test_gpu_embedding import ROUND, check_grad, tokens_of

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


@pytest.mark.parametrize("table", [F32, BF16])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("n,dim", [
    (4737, 256), (5001, 255), (5001, 264), (19001, 256), (19003, 99), (18947, 1032), (160001, 8), (700001, 8), (700003, 1),
])
def test_lookup_of_many_rows(ctx, table, act, n, dim):
    """Two and four rows a group, two of them in flight, with remainders and tokens outside the vocabulary."""
    vocab = 3000
    gen = torch.Generator(device="cuda").manual_seed(n)
    w = torch.randn(vocab, dim, device="cuda", generator=gen).to(table)
    t = tokens_of(n, vocab, "wild", torch.int64 if n % 2 else torch.int32, gen)
    t[-3:] = torch.tensor([vocab, 5, -1], device="cuda").to(t.dtype)
    out = L.Embedding(ctx, vocab, dim, scale=1.7).forward(t, w, dtype=act)
    inside = (t >= 0) & (t < vocab)
    want = w[t.long().clamp(0, vocab - 1)].double() * float(torch.tensor(1.7, dtype=F32)) * inside[:, None]
    assert bool(((out.double() - want).abs() <= ROUND[act] * want.abs() * 1.0001 + 2.0 ** -24 * want.abs()).all())


@pytest.mark.parametrize("dst", [F32, BF16])
@pytest.mark.parametrize("n,vocab,dim,stride,shift", [
    (500, 3000, 40, 48, 0), (500, 3000, 40, 41, 0), (500, 3000, 40, 64, 1), (3000, 70, 99, 101, 3), (0, 300, 24, 32, 0), (1, 1, 8, 16, 0),
    (40000, 9000, 520, 528, 0),
])
def test_gradient_into_rows_with_gaps(ctx, dst, n, vocab, dim, stride, shift):
    gen = torch.Generator(device="cuda").manual_seed(n + stride)
    t = tokens_of(n, vocab, "zipf", torch.int64, gen)
    g = torch.randn(n, dim, device="cuda", generator=gen)
    store = torch.full((shift + vocab * stride + 9,), 5.0, device="cuda", dtype=dst)
    grad = store.as_strided((vocab, dim), (stride, 1), shift)
    e = L.Embedding(ctx, vocab, dim)
    assert e.backward(t, g, grad=grad) is grad
    check_grad(grad, t, g, vocab, 1.0, -1)
    assert torch.equal(grad, e.backward(t, g, dtype=dst))
    untouched = torch.ones_like(store, dtype=torch.bool)
    untouched.as_strided((vocab, dim), (stride, 1), shift).fill_(False)
    assert bool((store[untouched] == 5.0).all())


@pytest.mark.parametrize("kind", ["uniform", "zipf", "wild"])
@pytest.mark.parametrize("n,vocab,dim", [
    (20000, 300007, 8),                     # three passes
    (5, 300007, 24),                        # three passes, 28 MB to zero, one block
    (9000, 262144, 16),                     # two passes just hold it, 16 MB to zero
    (9000, 262145, 16),                     # and three
    (30000, 1 << 27, 1),                    # three passes just hold it
    (30000, (1 << 27) + 1, 1),              # four passes
    (20000, 70000, 65),                     # 18 MB, elements
    (2000, 70000, 59),                      # just below 16 MB
])
def test_gradient_of_large_vocabularies(ctx, n, vocab, dim, kind):
    gen = torch.Generator(device="cuda").manual_seed(n + vocab)
    t = tokens_of(n, vocab, kind, torch.int64, gen)
    t[:2] = torch.tensor([vocab - 1, 0], device="cuda")
    g = torch.randn(n, dim, device="cuda", generator=gen)
    e = L.Embedding(ctx, vocab, dim, padding=7)
    got = torch.full((vocab, dim), 3.0, device="cuda")
    e.backward(t, g, grad=got)
    rows, index = t.unique(return_inverse=True)
    keep = (rows >= 0) & (rows < vocab) & (rows != 7)
    # the rows that tokens name, as a table of their own; all others are zero
    check_grad(got[rows[keep]], torch.where(keep, keep.cumsum(0) - 1, -1)[index], g, int(keep.sum()), 1.0, -1)
    named = got[rows[keep]].clone()
    got[rows[keep]] = 0.0
    assert not bool(got.any())
    acc = torch.full_like(got, 2.0)
    e.backward(t, torch.zeros_like(g), grad=acc, accumulate=True)
    assert bool((acc == 2.0).all())
    assert bool(named.any())


def capture(f):
    f()
    torch.cuda.synchronize()
    gc.collect()                 # a context of another module that is freed during the capture would end it
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = f()
    return g, out


@pytest.mark.parametrize("n,vocab,dim", [(257, 500, 64), (5000, 40, 99), (9000, 70000, 64)])
def test_embedding_in_a_captured_graph(ctx, n, vocab, dim):
    """New tokens and gradients in the captured tensors, another result at each replay."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    t = tokens_of(n, vocab, "zipf", torch.int32, gen)
    w, dy = torch.randn(vocab, dim, device="cuda", generator=gen), torch.randn(n, dim, device="cuda", generator=gen)
    e = L.Embedding(ctx, vocab, dim, scale=0.5, padding=0)
    acc = torch.zeros(vocab, dim, device="cuda")
    g, (y, dw) = capture(lambda: (e.forward(t, w), e.backward(t, dy)))
    g2, _ = capture(lambda: e.backward(t, dy, grad=acc, accumulate=True))
    for seed in range(3):
        t.copy_(tokens_of(n, vocab, "wild", torch.int32, gen))
        dy.normal_(generator=gen)
        acc.fill_(1.0)
        g.replay()
        g2.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, e.forward(t, w)) and torch.equal(dw, e.backward(t, dy))
        assert torch.equal(acc, e.backward(t, dy, grad=torch.ones_like(acc), accumulate=True))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_loss_in_a_captured_graph(ctx, dtype):
    gen = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn(40, 1003, device="cuda", generator=gen).to(dtype)
    top, index = torch.topk(torch.randn(40, 1003, device="cuda", generator=gen), 9, dim=1)
    gl = torch.randn(40, device="cuda", generator=gen)
    d = L.Distillation(ctx, 2.0)

    def f():
        loss, lse = d.forward(z, top, index)
        return loss, lse, d.backward(z, top, index, lse, gl), *d.step(z, top, index, gl)

    g, got = capture(f)
    for seed in range(3):
        z.copy_(torch.randn(40, 1003, device="cuda", generator=gen))
        gl.normal_(generator=gen)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, f()))


def test_contexts_without_dependent_launches(ctx):
    """Kernels that wait for their predecessors altogether give the same bits."""
    plain = B.Omni(1, 1, 1, 1, flags=B.NO_BULK_COPY)
    gen = torch.Generator(device="cuda").manual_seed(3)
    results = []
    t = tokens_of(5000, 700, "zipf", torch.int64, gen)
    dy = torch.randn(5000, 72, device="cuda", generator=gen).to(BF16)
    q, k, v, do = (torch.randn(2, n, h, 64, device="cuda", generator=gen).to(BF16) for n, h in ((300, 4), (1500, 2), (1500, 2), (300, 4)))
    z = torch.randn(40, 1003, device="cuda", generator=gen)
    top, index = torch.topk(z, 9, dim=1)
    for c in (ctx, plain):
        e, a, d = L.Embedding(c, 700, 72), L.Attention(c, 4, 2, 64), L.Distillation(c)
        out, lse = a.forward(q, k, v)                               # 8 pairs of query tiles: the walks are dealt out and joined
        results.append((e.backward(t, dy), out, lse, *a.backward(q, k, v, out, lse, do), *d.step(z, top, index, z[:, 0].contiguous())))
        c.stats()
    assert all(torch.equal(x, y) for x, y in zip(*results))
