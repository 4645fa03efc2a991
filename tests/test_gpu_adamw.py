"""AdamW over many tensors against its formulas.

Moments are compared bit by bit: every operation of theirs is rounded once, and a product or fused operation of floats is
exact in 64 bits before that rounding (a second rounding from 64 bits to 32 differs from one with a probability of 2^-29 a value).  The
parameter: its quotient is off by 2^-21 of itself, the product and the sum are rounded:
  |error| <= rate |m / (sqrt(v) spread + eps)| 2^-20.5 + 2^-24 (|keep theta| + |theta'|).
"""
import math

import pytest
import torch

from paper_2503_17469_b200 import binding as B
from paper_2503_17469_b200 import language as L

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SIZES = [1, 2, 0, 255, 256, 257, 2047, 2048, 2049, 7, 30011]
BLOCK = B.ADAMW_BLOCK


@pytest.fixture(scope="module")
def ctx():
    return B.Omni(1, 1, 1, 1)


def f32(x):
    return float(torch.tensor(x, dtype=F32))


def random_bits(n, tensor, t):
    y = (torch.arange(n, device="cuda") * 0x9E3779B1 + t * 0x85EBCA77 + tensor * 0xC2B2AE3D) & 0xFFFFFFFF
    x = ((y ^ (y >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    return x ^ (x >> 15)


def decode(codes, tops, most):
    c = codes.long().view(-1)
    magnitude = c & most
    top = tops.long().repeat_interleave(BLOCK)[:c.numel()]
    x = torch.where(magnitude > 0, (magnitude + top - most) << 20, 0).int().view(F32)
    return torch.where(c > most, -x, x).view(codes.shape)


def encode(x, random, most):
    n = x.numel()
    bits = x.reshape(-1).view(torch.int32).long() & 0x7FFFFFFF
    r = ((bits + (random << 4)) >> 20).clamp(max=0x7FF)
    tops = torch.nn.functional.pad(r, (0, -n % BLOCK)).view(-1, BLOCK).amax(1) if n else r
    c = r - tops.repeat_interleave(BLOCK)[:n] + most
    if most == 255:
        c = torch.where(r > 0, c.clamp(min=1), 0)
    else:
        c = torch.where(c > 0, c + 128 * torch.signbit(x.reshape(-1)), 0)
    return c.to(torch.uint8).view(x.shape), tops.to(torch.int16)


def update(theta, grads, m, v, batches, t, lr, betas, eps, decay):
    """(m, v as floats, theta in double, its bound)."""
    b1, b2, c1, c2 = f32(betas[0]), f32(betas[1]), f32(1 - betas[0]), f32(1 - betas[1])
    g = torch.zeros_like(theta)
    for b, x in zip(batches, grads):
        g = (f32(b / sum(batches)) * x.double() + g.double()).float()
    m = (b1 * m.double() + (c1 * g).double()).float()
    v = ((c2 * g).double() * g.double() + (b2 * v).double()).float()
    rate, spread, keep = f32(lr / (1 - betas[0] ** t)), f32(1 / math.sqrt(1 - betas[1] ** t)), f32(1 - lr * decay)
    move = rate * m.double() / (v.double().sqrt() * spread + f32(eps))
    want = keep * theta.double() - move
    return m, v, want, move.abs() * 2.0 ** -20.5 + 2.0 ** -24 * (theta.abs() + want.abs()) + 1e-44


class Case:
    def __init__(self, ctx, sizes, K=1, dtype=F32, bits=32, copies=True, shift=0, seed=0, spread=1.0, **kw):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def flat(kind, std):
            """One buffer, each tensor on a boundary of 16 elements, or `shift` elements behind one."""
            store = (torch.randn(sum((n + 15) // 16 * 16 + 16 for n in sizes), device="cuda", generator=gen) * std).to(kind)
            at, out = shift, []
            for n in sizes:
                out.append(store[at:at + n])
                at += (n + 15) // 16 * 16 + 16 * (shift > 0)
            return store, out

        self.store, self.params = flat(F32, 0.05)
        size = [torch.exp(torch.randn(n, device="cuda", generator=gen) * spread) * 1e-3 for n in sizes]
        self.grads = [[] for _ in sizes]
        for _ in range(K):
            for into, g, s in zip(self.grads, flat(dtype, 1.0)[1], size):
                g.copy_(g.float() * s)
                into.append(g)
        self.copy_store, self.copies = flat(BF16, 1.0) if copies else (None, None)
        self.batches, self.gen, self.bits = [1 + 7 * k % 5 for k in range(K)], gen, bits
        self.op = L.AdamW(ctx, self.params, self.grads, self.copies, bits=bits, **kw)

    def new_gradients(self):
        for gs in self.grads:
            for g in gs:
                g.copy_(torch.randn(g.shape, device="cuda", generator=self.gen) * 1e-3)

    def check_step(self, lr=1e-3, **kw):
        op, bits = self.op, self.bits
        before = [p.clone() for p in self.params]
        states = [tuple(x.clone() for x in s) for s in op.state]
        t = op.steps + 1
        op.step(lr, self.batches, **kw)
        decay = self.decay if hasattr(self, "decay") else [0.01] * len(before)
        for i, (p0, s0, s1) in enumerate(zip(before, states, op.state)):
            m, v = s0 if bits == 32 else (decode(s0[0], s0[2][:, 0], 127), decode(s0[1], s0[2][:, 1], 255))
            m, v, want, bound = update(p0, self.grads[i], m, v, self.batches, t, lr, op.betas, op.eps, decay[i])
            if bits == 32:
                assert torch.equal(s1[0], m) and torch.equal(s1[1], v)
            else:
                x = random_bits(m.numel(), i, t)
                for j, (value, random, most) in enumerate(((m, x & 0xFFFF, 127), (v, x >> 16, 255))):
                    codes, tops = encode(value, random, most)
                    assert torch.equal(s1[j], codes) and torch.equal(s1[2][:, j], tops)
            err = (self.params[i].double() - want).abs()
            assert bool((err <= bound).all()), float((err - bound).max())
            if self.copies is not None:
                assert torch.equal(self.copies[i], self.params[i].bfloat16())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K,copies,shift", [(1, True, 0), (1, False, 0), (4, True, 0), (32, False, 0), (3, True, 1), (2, True, 4), (1, True, 8)])
def test_steps(ctx, bits, dtype, K, copies, shift):
    c = Case(ctx, SIZES, K, dtype, bits, copies, shift, seed=K + shift)
    rest = c.store.clone()
    for _ in range(3):
        c.check_step()
        c.new_gradients()
    untouched = torch.ones_like(rest, dtype=torch.bool)
    base = c.store.data_ptr()
    for p in c.params:
        a = (p.data_ptr() - base) // 4
        untouched[a:a + p.numel()] = False
    assert torch.equal(c.store[untouched], rest[untouched])


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(ctx, bits):
    """More than one launch of the moments, empty tensors among them, a decay for each."""
    sizes = [(37 * i) % 700 * (i % 11 > 0) for i in range(500)]
    decay = [0.1 * (i % 3) for i in range(500)]
    c = Case(ctx, sizes, 2, BF16, bits, weight_decay=decay, betas=(0.8, 0.95), eps=1e-6)
    c.decay = decay
    for _ in range(2):
        c.check_step(0.01)
    for s, (m, v) in zip(c.op.state, c.op.moments()):
        if bits == 32:
            assert m is s[0] and v is s[1]
        else:
            assert torch.equal(m, decode(s[0], s[2][:, 0], 127)) and torch.equal(v, decode(s[1], s[2][:, 1], 255))


def test_large_tensor_and_wide_values(ctx):
    """Gradients over many octaves inside a block: codes at both ends."""
    for bits in (32, 8):
        c = Case(ctx, [3_000_001, 5], 1, F32, bits, spread=6.0)
        for _ in range(2):
            c.check_step()


def test_against_the_definition_in_64_bits_over_steps(ctx):
    c = Case(ctx, [1000, 333], 3, F32, 32, copies=False, betas=(0.9, 0.99), weight_decay=0.1)
    theta = [p.double() for p in c.params]
    m, v = [torch.zeros_like(x) for x in theta], [torch.zeros_like(x) for x in theta]
    for t in range(1, 21):
        c.new_gradients()
        for i, gs in enumerate(c.grads):
            g = sum(b * x.double() for b, x in zip(c.batches, gs)) / sum(c.batches)
            m[i], v[i] = 0.9 * m[i] + 0.1 * g, 0.99 * v[i] + 0.01 * g * g
            theta[i] -= 1e-2 * (m[i] / (1 - 0.9 ** t) / ((v[i] / (1 - 0.99 ** t)).sqrt() + 1e-8) + 0.1 * theta[i])
        c.op.step(1e-2, c.batches)
    assert c.op.steps == 20
    for p, x in zip(c.params, theta):
        # twenty updates of at most 4 lr (|m| <= 4 sqrt(v) here), each off by a few 2^-22 of itself, and twenty roundings of theta
        assert float((p.double() - x).abs().max()) <= 20 * (4e-2 * 2.0 ** -19 + 2.0 ** -24 * float(x.abs().max()))


def test_8_bits_lose_nothing_on_average(ctx):
    """Rounding is off by less than an eighth of a value and by nothing on average: the mean of n roundings, each of a variance of at
    most 1/4 of the step's square, is within 5 deviations, 5 / 2 / sqrt(n) steps of an eighth."""
    n = 1 << 18
    c = Case(ctx, [n], 1, F32, 8, copies=False, spread=0.3)
    c.op.step(1e-3)
    g = c.grads[0][0].double()
    m, v = (x.double() for x in c.op.moments()[0])
    for got, want in ((m, f32(0.1) * g), (v, f32(1 - 0.999) * g * g)):
        large = want.abs() > want.abs().max() * 2.0 ** -12
        off = ((got - want) / want)[large]
        assert float(off.abs().max()) < 0.126 and abs(float(off.mean())) <= 5 / 2 / math.sqrt(int(large.sum())) / 8


def test_8_bits_decay(ctx):
    """Without gradients v falls by a thousandth a step, two hundred times, although a step of its codes is an eighth: the logarithm of
    the mean over n elements follows, each rounding adding at most (1/8)^2 / 4 variance an element."""
    n, steps = 1 << 16, 200
    c = Case(ctx, [n], 1, F32, 8, copies=False, spread=0.3)
    c.op.step(1e-3)
    start = c.op.moments()[0][1].double()
    c.grads[0][0].zero_()
    for _ in range(steps):
        c.op.step(1e-3)
    end = c.op.moments()[0][1].double()
    large = start > start.max() * 2.0 ** -12
    ratio = (end / start)[large]
    expect = 0.999 ** steps
    assert abs(float(ratio.mean()) / expect - 1) <= 5 * math.sqrt(steps / 4) / 8 / math.sqrt(int(large.sum()))
    assert bool((end[start > 0] > 0).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_zeros_and_what_is_not_finite(ctx, bits):
    c = Case(ctx, [3000, 700], 1, F32, bits)
    for g in c.grads[0] + c.grads[1]:
        g.zero_()
    before = [p.clone() for p in c.params]
    c.op.step(1e-3)
    for p, b, (m, v) in zip(c.params, before, c.op.moments()):
        assert not bool(m.any()) and not bool(v.any())
        assert torch.equal(p, (b * f32(1 - 1e-5)))
    c.new_gradients()
    c.check_step()
    c.grads[0][0][300] = math.nan
    c.grads[0][0][1300] = math.inf
    c.op.step(1e-3)
    bad = torch.zeros(3000, device="cuda", dtype=torch.bool)
    bad[[300, 1300]] = True
    assert torch.equal(c.params[0].isfinite(), ~bad) and bool(c.params[1].isfinite().all())
    m, v = c.op.moments()[0]
    assert math.isnan(m[300]) and math.isnan(v[300]) and math.isinf(v[1300])
    blocks = torch.arange(3000, device="cuda") // BLOCK
    sound = (blocks != 300 // BLOCK) & (blocks != 1300 // BLOCK) if bits == 8 else ~bad
    assert bool(m[sound].isfinite().all()) and bool(v[sound].isfinite().all())
    tiny = Case(ctx, [600], 1, F32, bits)
    tiny.grads[0][0].mul_(1e-20)                                      # v underflows in float
    tiny.check_step()


@pytest.mark.parametrize("bits", [32, 8])
def test_going_on_from_a_state(ctx, bits):
    a = Case(ctx, SIZES, 2, BF16, bits, seed=5)
    for _ in range(3):
        a.op.step(1e-3, a.batches)
    state = [tuple(x.clone() for x in s) for s in a.op.state]
    params = [p.clone() for p in a.params]
    other = L.AdamW(ctx, params, a.grads, None, bits=bits, state=state, steps=a.op.steps)
    for _ in range(2):
        a.op.step(1e-3, a.batches)
        other.step(1e-3, a.batches)
    assert other.steps == 5 and all(torch.equal(x, y) for x, y in zip(a.params, params))
    assert all(torch.equal(x, y) for s, u in zip(a.op.state, state) for x, y in zip(s, u))


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_and_streams(ctx, bits):
    a, b, d = (Case(ctx, SIZES, 2, BF16, bits, seed=6) for _ in range(3))
    clock = torch.zeros(1, dtype=torch.int64, device="cuda")
    L.AdamW(ctx, [torch.zeros(3, device="cuda")], [[torch.zeros(3, device="cuda")]]).step(1e-3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clock.add_(1)
        a.op.step(1e-3, a.batches, clock=clock)
    clock.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for x in (a, b, d):
            x.new_gradients()
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        b.op.step(1e-3, b.batches)
        d.op.step(1e-3, d.batches, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert int(clock) == 4 and a.op.steps == 0 and b.op.steps == 4
    for other in (a, d):
        assert all(torch.equal(x, y) for x, y in zip(other.params, b.params))
        assert all(torch.equal(x, y) for s, u in zip(other.op.state, b.op.state) for x, y in zip(s, u))
        assert all(torch.equal(x, y) for x, y in zip(other.copies, b.copies))
    ctx.stats()


def test_the_weighted_mean_is_that_of_the_synchronous_step(ctx):
    """The same chain of fused operations: with b1 = 0 and a first step m is the aggregated gradient, as momentum 0 leaves it in v."""
    K, n = 5, 10_007
    c = Case(ctx, [n], K, BF16, 32, copies=False, betas=(0.0, 0.5))
    omni = B.Omni(K, sum(c.batches), 1, 100)
    theta, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    omni.aggregate_bsp(B.BucketSet([theta], [c.grads[0]], [v]), c.batches, 1.0, 0.0)
    c.op.step(1e-3, c.batches)
    assert torch.equal(c.op.state[0][0], -theta)


def test_nothing(ctx):
    L.AdamW(ctx, [], []).step(1e-3)
    op = L.AdamW(ctx, [torch.zeros(0, device="cuda")], [[torch.zeros(0, device="cuda")]], bits=8)
    op.step(1e-3)
    assert op.steps == 1 and op.moments()[0][0].numel() == 0


def test_refusals(ctx):
    p, g = torch.zeros(40, device="cuda"), torch.zeros(40, device="cuda")
    make = lambda **kw: L.AdamW(ctx, **{**dict(params=[p], grads=[[g]]), **kw})  # noqa: E731
    op = make()
    two = make(grads=[[g, g]])
    for bad in (lambda: make(bits=16), lambda: make(grads=[]), lambda: make(grads=[[]]), lambda: make(grads=[[g] * 33]),
                lambda: make(grads=[[g[:39]]]), lambda: make(grads=[[torch.zeros(80, device="cuda")[::2]]]), lambda: make(copies=[]),
                lambda: make(weight_decay=[0.1, 0.1]), lambda: make(betas=(1.0, 0.9)), lambda: make(eps=-1.0), lambda: make(steps=-1),
                lambda: make(state=[]), lambda: make(state=[(g,)]), lambda: make(state=[(g, p.cpu())]), lambda: make(grads=[[g.cpu()]]),
                lambda: make(bits=8, state=[(p.byte(), g.byte(), torch.zeros(2, 2, dtype=torch.int16, device="cuda"))]),
                lambda: op.step(1e-3, [1, 2]), lambda: two.step(1e-3), lambda: op.step(1e-3, clock=torch.ones(1, dtype=torch.int64)),
                lambda: op.step(1e-3, clock=torch.ones(2, dtype=torch.int64, device="cuda")), lambda: op.moments(out=[(p, g)]),
                lambda: make(bits=8).moments(out=[]), lambda: make(bits=8).moments(out=[(p, g[:3])])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: make(params=[p.double()]), lambda: make(grads=[[g.half()]]), lambda: make(copies=[g]),
                lambda: make(bits=8, state=[(p, g, p)]), lambda: make(grads=[[g, g.bfloat16()]])):
        with pytest.raises(TypeError):
            bad()
    for bad, status in ((lambda: op.step(math.nan), B.ERR_BAD_CONFIG), (lambda: two.step(1e-3, [1, 0]), B.ERR_BAD_BATCH),
                        (lambda: make(params=[p, p], grads=[[g], [g]]), B.ERR_BAD_CONFIG),
                        (lambda: make(params=[p[:30], p[29:]], grads=[[g[:30]], [g[29:]]]), B.ERR_BAD_CONFIG),
                        (lambda: make(state=[(p, g)]), B.ERR_BAD_CONFIG), (lambda: make(weight_decay=math.inf), B.ERR_BAD_CONFIG)):
        with pytest.raises(B.OmniError) as err:
            bad()
        assert err.value.status == status
    assert op.steps == 0 and two.steps == 0
