"""AdamW with any eps: moments below float's normal range keep their root, and no quotient overflows that float can hold.  Bounds:
those of test_gpu_adamw.py; where eps is not between 2^-41 (1 - beta2)^(-1/2) and 2^100 every operation is rounded once, which 64 bits and
one more rounding show (but for a probability of 2^-29 a value)."""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B

from test_gpu_adamw import F32, Case, f32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


def sizes_of_all_kinds(c):
    """Gradients of either sign between 3e-20, whose square times 0.001 is a tenth of float's smallest normal number and below, and 30."""
    for gs in c.grads:
        for g in gs:
            size = 3 * 10.0 ** (torch.rand(g.shape, device="cuda", generator=c.gen) * 21 - 20)
            g.copy_(torch.where(torch.rand(g.shape, device="cuda", generator=c.gen) < 0.5, size, -size))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-30, 1e-20, 1e-12, 1e-8, 1.0, 1e30])
def test_small_moments(ctx, bits, shift, eps):
    c = Case(ctx, [3000, 257, 5], 1, F32, bits, copies=False, shift=shift, eps=eps)
    for _ in range(3):
        sizes_of_all_kinds(c)
        c.check_step()


@pytest.mark.parametrize("bits", [32, 8])
def test_small_moments_alone(ctx, bits):
    """Blocks in which nothing is larger, and a clock on the device."""
    c = Case(ctx, [3000], 1, F32, bits, copies=False, eps=0.0)
    c.grads[0][0].copy_(1e-19 * torch.where(torch.arange(3000, device="cuda") % 3 == 0, -1.0, 0.7))
    before, clock = c.params[0].double(), torch.ones(1, dtype=torch.int64, device="cuda")
    c.op.step(1e-3, clock=clock)
    # m / sqrt(v) is the gradient's sign but for v, a few steps of 2^-149 large, which is off by half a step of at least five
    want = before * (1 - 1e-5) - 1e-3 * torch.sign(c.grads[0][0].double())
    assert bool(((c.params[0].double() - want).abs() <= 1e-3 * 0.06 + 2.0 ** -22).all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-40, 1e-30, 1e-8])
def test_no_gradient_moves_nothing(ctx, bits, eps):
    c = Case(ctx, [700], 1, F32, bits, eps=eps)
    c.grads[0][0].zero_()
    before = c.params[0].clone()
    c.op.step(1e-3)
    assert torch.equal(c.params[0], before * f32(1 - 1e-5))


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-20, 1e-13, 1e31])
def test_parameters_bit_by_bit(ctx, shift, eps):
    c = Case(ctx, [3000, 257, 5], 1, F32, 32, shift=shift, eps=eps)
    for t in (1, 2):
        sizes_of_all_kinds(c)
        before = [p.clone() for p in c.params]
        c.op.step(1e-3)
        rate, spread, keep = f32(1e-3 / (1 - 0.9 ** t)), f32(1 / math.sqrt(1 - 0.999 ** t)), f32(1 - 1e-5)
        for p, p0, (m, v) in zip(c.params, before, c.op.state):
            below = (v.double().sqrt().float().double() * spread + f32(eps)).float()
            way = (m.double() / below.double()).float().double()
            assert torch.equal(p, ((p0.double() * keep).float().double() - rate * way).float())
