"""Results of the rotation that write an element twice are refused: heads, rows or sequences of one result, and the two results."""
import itertools

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

from test_rotary_host import KEYS, PTR, ROWS, backward, forward, rotary

AWAY = PTR + (1 << 20)
APART = B.omni_attn_view(AWAY, KEYS.batch, KEYS.row, KEYS.head)


@pytest.fixture(scope="module")
def omni():
    return B.Omni(1, 1, 1, 1)


def both(omni, q, k):
    """Statuses of both directions with these results, of 2 sequences of 5 rows of 4 and 2 heads of 64 bfloat16."""
    return forward(omni._h, rotary(), {2: q, 3: k}), backward(omni._h, rotary(), {4: q, 5: k})


# (batch, row, head) strides of four heads
@pytest.mark.parametrize("strides", [(1280, 64, 64), (1280, 255, 64), (1279, 256, 64), (256, 256, 64), (64, 256, 64), (320, 320, 64),
                                     (1280, 256, 100), (64, 128, 600), (400, 80, 783)])
def test_refuses_results_that_write_an_element_twice(omni, strides):
    assert both(omni, B.omni_attn_view(PTR, *strides), APART) == (B.ERR_BAD_CONFIG,) * 2


# element offset of the keys' result from the queries', and its strides
@pytest.mark.parametrize("offset,strides", [
    (0, (640, 128, 64)), (63, (1280, 256, 64)), (255, (1280, 256, 64)), (-63, (640, 128, 64)), (-639 - 640, (640, 128, 64)),
    (2559, (640, 128, 64)), (192, (1280, 256, 64)), (1500, (640, 128, 64)), (320 + 256 * 3, (1280, 256, 64)),
])
def test_refuses_results_that_overlap_each_other(omni, offset, strides):
    q = B.omni_attn_view(AWAY, 1280, 256, 64)
    assert both(omni, q, B.omni_attn_view(AWAY + 2 * offset, *strides)) == (B.ERR_BAD_CONFIG,) * 2


@pytest.mark.gpu
@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
def test_takes_results_that_lie_among_each_other(order):
    """Slices of one buffer whose batch, row and head axes lie in any order, the queries' heads beside the keys', with gaps or without; and
    one buffer with the queries' rows of a sequence before its keys'."""
    ctx = B.Omni(1, 1, 1, 1)
    b, n, h, hk, d = 3, 7, 4, 2, 32
    r = L.Rotary(ctx, h, hk, d, L.Rotary.geometric(16))
    q, k = torch.randn(b, n, h, d, device="cuda"), torch.randn(b, n, hk, d, device="cuda")
    at, w = torch.arange(n, device="cuda")[None].expand(b, -1), torch.ones(d, device="cuda")
    back = tuple(order.index(i) for i in range(3))

    def places(gap):
        sizes = (b + gap, n + gap, h + hk + gap)
        whole = torch.full((*(sizes[i] for i in order), d + gap), 5.0, device="cuda").permute(*back, 3)
        yield whole[:b, :n, :h, :d], whole[:b, :n, h:h + hk, :d]
        yield whole[:b, :n, hk:h + hk, :d], whole[:b, :n, :hk, :d]
        arena = torch.full((b, n * (h + hk) * d), 5.0, device="cuda")
        yield arena[:, :n * h * d].view(b, n, h, d), arena[:, n * h * d:].view(b, n, hk, d)

    for gap in (0, 1, 4):
        for out, other in zip(places(gap), places(gap)):
            # against the same strides in two buffers: the bits depend on the width of the accesses, which the strides decide
            apart = out[0], other[1]
            want = [t.clone() for t in r.forward(q, k, at, w, w, out=apart)]
            assert all(torch.equal(x, y) for x, y in zip(r.forward(q, k, at, w, w, out=out), want))
            grads = [t.clone() for t in r.backward(q, k, at, q, k, w, w, grads=apart)]
            assert all(torch.equal(x, y) for x, y in zip(r.backward(q, k, at, q, k, w, w, grads=out), grads))
    want = r.forward(q, k, at, w, w)
    one = r.forward(q[:1], k[:1], at[:1], w, w, out=(q[:1].expand(1, -1, -1, -1), k[:1]))       # the stride of a single sequence is not looked at
    assert torch.equal(one[0], want[0][:1])
