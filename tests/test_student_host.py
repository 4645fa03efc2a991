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
