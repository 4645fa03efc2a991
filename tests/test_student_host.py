"""The student's parameters without a GPU: which of them are the norms' weights."""
import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import student as S


@pytest.mark.parametrize("vocab,dim,heads,kv_heads,head_dim", [(2, 16, 2, 1, 8), (30, 2, 1, 1, 4), (30, 16, 1, 1, 2), (2, 2, 1, 1, 2), (30, 16, 2, 1, 8)])
def test_norms_begin_at_one_and_nothing_else(vocab, dim, heads, kv_heads, head_dim):
    cfg = S.Config(vocab=vocab, dim=dim, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rotary=True)
    student = S.Student(B.Omni(1, 1, 1, 1), cfg, device="cpu")
    *others, norms = student.views(student.theta)
    assert norms.shape == (2, head_dim) and bool((norms == 1.0).all())
    for x in others:
        assert not bool((x == 1.0).any()) and float(x.std()) > 0
    plain = S.Student(B.Omni(1, 1, 1, 1), S.Config(**{**vars(cfg), "rotary": False}), device="cpu")
    assert all(torch.equal(a, b) for a, b in zip(others, plain.views(plain.theta)))


def test_momentum_is_the_other_optimizers():
    """AdamW has none: asked for, it is refused before any worker's pass; by default SGD has 0.9 as before."""
    student = S.Student(B.Omni(1, 1, 1, 1), S.Config(vocab=30, dim=16, heads=2, kv_heads=1, head_dim=8), device="cpu")
    student.gradient = lambda k, batch: torch.zeros(())
    got = []
    student.omni.step_bsp = lambda buckets, throughputs, lr, momentum: got.append(momentum)
    student.step([None], [1.0], 0.1)
    student.step([None], [1.0], 0.1, momentum=0.0)
    assert got == [0.9, 0.0]
    student.adamw = object()
    with pytest.raises(ValueError, match="momentum"):
        student.step([None], [1.0], 0.1, momentum=0.9)
