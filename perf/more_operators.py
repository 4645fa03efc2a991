"""Cases of the operators of a language model's policy training, their inputs, and the operators in plain form.

Beside the embedding, the attention and the distillation loss a worker's pass needs positions (norms
of the query and key heads with the rotation, before attention), an objective on sampled tokens (the
clipped policy loss with its divergence from a reference), and the step that takes the K workers'
gradients has an AdamW form over many tensors, with states of 32 or 8 bits.

``own`` false: elementary torch operations in float32 (64 bits for angles, long sums and what is
rounded to codes), rounded once at the end.  ``own`` true: the calls of ``paper_2503_17469_b200.language``.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
BLOCK = 256              # elements that share the offsets of their 8-bit codes


def listed():
    return [
        # decoding: one token each of 16 running sequences at far positions; a latency-bound call
        dict(name="rotary_decode", op="rotary", way="forward", batch=16, length=1, heads=16, kv_heads=4, dim=128, rotated=128, axes=1,
             act="bf16", norm=True, interleaved=False, ragged=False),
        # the prompt pass or the forward half of a training step on long sequences with shared key heads
        dict(name="rotary_fwd_long", op="rotary", way="forward", batch=4, length=4096, heads=32, kv_heads=8, dim=128, rotated=128, axes=1,
             act="bf16", norm=True, interleaved=False, ragged=False),
        # patches of videos (time, height, width) of different lengths, one of them empty; part of a head of 80 is rotated
        dict(name="rotary_bwd_video", op="rotary", way="backward", batch=6, length=1777, heads=12, kv_heads=12, dim=80, rotated=48, axes=3,
             act="f32", norm=True, interleaved=True, ragged=True),
        # the longest training context
        dict(name="rotary_bwd_long", op="rotary", way="backward", batch=2, length=8192, heads=16, kv_heads=8, dim=128, rotated=128, axes=1,
             act="bf16", norm=True, interleaved=False, ragged=False),
        # a small model's loss with its gradient: a latency-bound call
        dict(name="policy_step_small", op="policy", way="step", rows=48, vocab=1000, act="f32", index="i64", temperature=1.0, kl=0.05),
        # one worker's batch of sampled answers: loss and gradient in one pass, rows 2-byte aligned only
        dict(name="policy_step_batch", op="policy", way="step", rows=8192, vocab=50257, act="bf16", index="i64", temperature=1.0, kl=0.02),
        # log-probabilities under a frozen model, before the training steps
        dict(name="policy_logprob_wide", op="policy", way="logprob", rows=3000, vocab=131072, act="bf16", index="i32", temperature=1.0, kl=0.0),
        # the gradient alone, from the kept log-sum-exp, as an autograd backward asks for it
        dict(name="policy_bwd", op="policy", way="backward", rows=4096, vocab=32000, act="f32", index="i32", temperature=0.7, kl=0.1),
        # a small model's three tensors, gradients of four workers of different batch sizes; a latency-bound call
        dict(name="adamw_small", op="adamw", bits=32, K=4, kind="model", vocab=1000, dim=128, layers=1, tensors=0, act="bf16", copy=True),
        # a model of 140 million parameters, float states
        dict(name="adamw_model", op="adamw", bits=32, K=1, kind="model", vocab=50257, dim=1024, layers=8, tensors=0, act="bf16", copy=True),
        # the same with states of 8 bits
        dict(name="adamw8_model", op="adamw", bits=8, K=1, kind="model", vocab=50257, dim=1024, layers=8, tensors=0, act="bf16", copy=True),
        # many small tensors of odd sizes (adapters, norms, biases), float gradients of two workers, states of 8 bits
        dict(name="adamw8_many", op="adamw", bits=8, K=2, kind="many", vocab=0, dim=0, layers=0, tensors=400, act="f32", copy=False),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm; odd ones as they fall."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotary", "policy", "adamw"))
    act = rng.choice(("f32", "bf16"))
    if op == "rotary":
        dim = rng.choice((64, 128, 16 * rng.randint(1, 16), 2 * rng.randint(1, 128)))
        kv_heads = rng.choice((1, 2, 4, 8))
        heads = kv_heads * rng.choice((1, 2, 3, 4))
        batch = rng.choice((1, 2, 3, 5, 16))
        most = max(1, min(32768, (1 << 26) // (batch * (heads + kv_heads) * dim)))
        return dict(op=op, way=rng.choice(("forward", "backward")), batch=batch, length=_log(rng, 1, most), heads=heads, kv_heads=kv_heads,
                    dim=dim, rotated=dim if rng.random() < 0.6 else 2 * rng.randint(1, dim // 2), axes=rng.choice((1, 1, 2, 3)), act=act,
                    norm=rng.random() < 0.75, interleaved=rng.random() < 0.4, ragged=rng.random() < 0.4)
    if op == "policy":
        vocab = _log(rng, 100, 200000)
        return dict(op=op, way=rng.choice(("logprob", "forward", "backward", "step", "step")), vocab=vocab,
                    rows=_log(rng, 1, max(1, min(16384, 800_000_000 // (vocab * SIZE[act])))), act=act, index=rng.choice(("i32", "i64")),
                    temperature=rng.choice((1.0, 1.0, 0.7, 2.0)), kl=rng.choice((0.0, 0.02, 0.1)))
    common = dict(op=op, bits=rng.choice((32, 8, 8)), K=rng.choice((1, 1, 2, 4, 7)), act=act, copy=rng.random() < 0.5)
    if rng.random() < 0.4:
        return dict(common, kind="many", vocab=0, dim=0, layers=0, tensors=_log(rng, 1, 1000))
    dim = _log(rng, 8, 1000)
    return dict(common, kind="model", vocab=_log(rng, 50, 24_000_000 // dim), dim=dim, layers=rng.randint(1, 2), tensors=0)


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------

def _normal(gen, shape, std, dtype=torch.float32):
    return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0.0, std, generator=gen).to(dtype)


def _frequencies(c):
    """Of each pair in radians per position, base 10000; the pairs take turns by runs between the axes."""
    pairs = c["rotated"] // 2
    frequencies = [10000.0 ** (-i / pairs) for i in range(pairs)]
    return frequencies, [i * c["axes"] // pairs for i in range(pairs)]


def _positions(c, gen):
    """[axes, batch, length]: far along for single tokens, a frame's patches (8 high, 13 wide) for several axes."""
    b, n = c["batch"], c["length"]
    at = torch.arange(n, device="cuda")
    if c["axes"] == 1:
        if n == 1:
            return torch.randint(0, 131072, (1, b, 1), device="cuda", generator=gen)
        return (at + torch.randint(0, 1000, (b, 1), device="cuda", generator=gen))[None].contiguous()
    parts = [at // 104, at % 104 // 13, at % 13][:c["axes"]]
    return torch.stack(parts)[:, None].expand(-1, b, -1).contiguous()


def _prepare_rotary(c, gen):
    """Queries and keys as slices of one projection's output, as attention takes them."""
    b, n, h, hk, d = c["batch"], c["length"], c["heads"], c["kv_heads"], c["dim"]
    dtype = DTYPES[c["act"]]
    packed = _normal(gen, (b, n, h + 2 * hk, d), 1.5, dtype)
    s = dict(c, q=packed[:, :, :h], k=packed[:, :, h:h + hk], positions=_positions(c, gen), lengths=None, q_weight=None, k_weight=None)
    s["frequencies"], s["axis"] = _frequencies(c)
    if c["norm"]:
        s["q_weight"], s["k_weight"] = ((1.0 + _normal(gen, (d,), 0.2)).to(dtype) for _ in range(2))
    if c["ragged"]:
        u = torch.rand(b, device="cuda", generator=gen)
        u[0] = 1.0
        if b > 2:
            u[-1] = 0.0
        s["lengths"] = torch.ceil(u * n).int()
    if c["way"] == "backward":
        s["grad_q"], s["grad_k"] = (_normal(gen, (b, n, x, d), 1e-2, dtype) for x in (h, hk))
    return s


CLIP = (0.2, 0.28)


def _prepare_policy(c, gen):
    """A policy's logits (the last columns are the padding of the vocabulary: -inf), sampled tokens, rows without one (prompt and
    padding), the log-probabilities when the tokens were sampled and under the reference, advantages."""
    rows, vocab, temp = c["rows"], c["vocab"], c["temperature"]
    logits = _normal(gen, (rows, vocab), 2.0)
    logits[:, vocab - vocab // 64:] = -math.inf
    logits = logits.to(DTYPES[c["act"]])
    lse, tokens = [], []
    step = max(1, (1 << 27) // vocab)
    for a in range(0, rows, step):
        z = logits[a:a + step].double() / temp
        lse.append(torch.logsumexp(z, 1))
        noise = torch.empty_like(z, dtype=torch.float32).exponential_(generator=gen)
        tokens.append((z - noise.log()).argmax(1))
    lse, tokens = torch.cat(lse), torch.cat(tokens)
    logp = logits.gather(1, tokens[:, None])[:, 0].double() / temp - lse
    # how far the policy has moved since; no row stands within rounding of a clipping border, where either side would be right
    moved = _normal(gen, (rows,), 0.2).double()
    for border in (math.log(1 - CLIP[0]), math.log(1 + CLIP[1])):
        moved += 2e-4 * ((moved - border).abs() < 1e-4)
    s = dict(c, logits=logits, old=(logp - moved).float(), reference=(logp + _normal(gen, (rows,), 0.3)).float(),
             advantage=_normal(gen, (rows,), 1.0), grad_loss=torch.full((rows,), 1.0 / rows, device="cuda"), lse=lse.float())
    tokens[torch.rand(rows, device="cuda", generator=gen) < 0.1] = -1
    s["tokens"] = tokens.int() if c["index"] == "i32" else tokens
    return s


BETAS, EPS, DECAY, RATE = (0.9, 0.95), 1e-8, 0.1, 1e-3


def _sizes(c):
    """Elements of each tensor."""
    if c["kind"] == "many":
        return [(7919 * (i + 1)) % 60013 + 1 for i in range(c["tensors"])]
    d = c["dim"]
    return [c["vocab"] * d] + [n for _ in range(c["layers"]) for n in (d, d * d * 3 // 2, d * d, d, 4 * d * d, 4 * d * d)]


def _nearest_codes(x, most):
    """The state a checkpoint holds: magnitudes as the top 12 bits of the float, nearest, counted from the block's largest."""
    n = x.numel()
    r = ((x.abs().view(torch.int32).long() + (1 << 19)) >> 20)
    r = torch.nn.functional.pad(r, (0, -n % BLOCK)).view(-1, BLOCK)
    top = r.amax(1)
    code = (r - top[:, None] + most).clamp(min=0).view(-1)[:n]
    return torch.where(x.abs() > 0, code, 0), top


def _views(flat, sizes):
    """The tensors of one flat buffer, each on a boundary of 64 elements."""
    at, out = 0, []
    for n in sizes:
        out.append(flat[at:at + n])
        at += (n + 63) // 64 * 64
    return out


def _prepare_adamw(c, gen):
    """Parameters, gradients and states in the middle of a training run, as views of flat buffers."""
    sizes, K = _sizes(c), c["K"]
    total = sum((n + 63) // 64 * 64 for n in sizes)
    there = torch.zeros(total, device="cuda", dtype=torch.bool)
    for x in _views(there, sizes):
        x.fill_(True)

    def flat(std, dtype=torch.float32):
        return _normal(gen, (total,), std, dtype).masked_fill_(~there, 0.0)

    s = dict(c, sizes=sizes, flat=flat(0.02), batches=[3 + 5 * k % 11 for k in range(K)], steps=100)
    s["params"] = _views(s["flat"], sizes)
    per_worker = [_views(flat(1e-3, DTYPES[c["act"]]), sizes) for _ in range(K)]
    s["grads"] = [[g[i] for g in per_worker] for i in range(len(sizes))]
    s["flat_copy"] = s["flat"].bfloat16() if c["copy"] else None
    s["copies"] = _views(s["flat_copy"], sizes) if c["copy"] else None
    s["m"], s["v"] = flat(2e-4), flat(1e-3).square_()
    s["moments"] = list(zip(_views(s["m"], sizes), _views(s["v"], sizes)))
    if c["bits"] == 32:
        s["state"] = s["moments"]
        return s
    s["state"] = []
    for m, v in s["moments"]:
        codes, tops = zip(_nearest_codes(m, 127), _nearest_codes(v, 255))
        signed = torch.where(codes[0] > 0, codes[0] + 128 * (m < 0), 0)
        s["state"].append((signed.to(torch.uint8), codes[1].to(torch.uint8), torch.stack(tops, 1).to(torch.int16)))
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"rotary": _prepare_rotary, "policy": _prepare_policy, "adamw": _prepare_adamw}[case["op"]](case, gen)


# ------------------------------------------------------------------------------------------------
# The plain forms
# ------------------------------------------------------------------------------------------------

def _pairs(x, s):
    """First and second elements of the rotated pairs, and the rest of the head."""
    r = s["rotated"]
    if s["interleaved"]:
        return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]
    return x[..., :r // 2], x[..., r // 2:r], x[..., r:]


def _joined(a, b, rest, s):
    turned = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, rest], -1)


def _turns(s):
    """Cosines and sines [batch, length, 1, pairs]: the angles in 64 bits, which float positions would spoil."""
    axis = torch.tensor(s["axis"], device="cuda")
    angle = s["positions"].permute(1, 2, 0)[:, :, axis].double() * torch.tensor(s["frequencies"], device="cuda", dtype=torch.float64)
    return torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]


def _there(s):
    """[batch, length, 1, 1]: rows before the lengths."""
    return (torch.arange(s["length"], device="cuda")[None] < s["lengths"][:, None])[:, :, None, None]


def _plain_rotary(s):
    cos, sin = _turns(s)
    out, weights = [], []
    for name in ("q", "k"):
        x, w = s[name].float(), s[name + "_weight"]
        if s["lengths"] is not None:
            x = x.masked_fill(~_there(s), 0.0)
        scale = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) if s["norm"] else 1.0
        if s["way"] == "forward":
            a, b, rest = _pairs(x * scale * w.float() if s["norm"] else x, s)
            y = _joined(a * cos - b * sin, b * cos + a * sin, rest, s)
        else:
            g = s["grad_" + name].float()
            if s["lengths"] is not None:
                g = g.masked_fill(~_there(s), 0.0)
            a, b, rest = _pairs(g, s)
            y = _joined(a * cos + b * sin, b * cos - a * sin, rest, s)
            if s["norm"]:
                n = x * scale
                weights.append((y * n).double().sum((0, 1, 2)).float())
                y = y * w.float()
                y = scale * (y - n * (y * n).mean(-1, keepdim=True))
        out.append(y.to(s[name].dtype))
    return tuple(out + weights)


def _policy_terms(s, logp):
    """(loss, its derivative by the log-probability) of rows with a token, from their log-probabilities."""
    a, low, high = s["advantage"].to(logp.dtype), 1.0 - CLIP[0], 1.0 + CLIP[1]
    ratio = torch.exp(logp - s["old"])
    gain, clipped = ratio * a, ratio.clamp(low, high) * a
    gap = s["reference"] - logp
    loss = -torch.minimum(gain, clipped) + s["kl"] * (torch.expm1(gap) - gap)
    return loss, -torch.where(gain <= clipped, gain, 0.0) - s["kl"] * torch.expm1(gap)


def _plain_policy(s):
    z = s["logits"].float() / s["temperature"]
    tokens = s["tokens"].long()
    there = tokens >= 0
    if s["way"] == "backward":
        lse = s["lse"]
    else:
        top = z.amax(1, keepdim=True)
        lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))[:, 0]
    logp = torch.where(there, z.gather(1, tokens.clamp(min=0)[:, None])[:, 0] - lse, 0.0)
    if s["way"] == "logprob":
        return logp, lse
    loss, slope = _policy_terms(s, logp)
    loss = torch.where(there, loss, 0.0)
    if s["way"] == "forward":
        return loss, logp, lse
    gain = torch.where(there, slope * s["grad_loss"] / s["temperature"], 0.0)[:, None]
    grad = torch.exp(z - lse[:, None]).mul_(-gain).scatter_add_(1, tokens.clamp(min=0)[:, None], gain).to(s["logits"].dtype)
    return grad if s["way"] == "backward" else (loss, logp, lse, grad)


def _fma(a, b, c):
    """a * b + c of floats, rounded once: the product is exact in 64 bits."""
    return (torch.as_tensor(a).double() * torch.as_tensor(b).double() + c.double()).float()


def _float(x):
    """A Python number rounded to 32 bits."""
    return float(torch.tensor(x, dtype=torch.float32))


def _random_bits(n, tensor, step):
    """32 bits for each element of a tensor, by multiplications and shifts of its number, the tensor's and the step's."""
    mask = 0xFFFFFFFF
    start = (step * 0x85EBCA77 + tensor * 0xC2B2AE3D) & mask
    x = (torch.arange(n, device="cuda") * 0x9E3779B1 + start) & mask
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & mask
    return x ^ (x >> 15)


def _values(codes, top, most):
    """What codes stand for: the float whose top 12 bits are the code, counted from the block's largest."""
    c = codes.long() & most
    bits = (c + top.long().repeat_interleave(BLOCK)[:c.numel()] - most) << 20
    x = torch.where(c > 0, bits, 0).int().view(torch.float32)
    return torch.where(codes > most, -x, x)


def _codes(x, random, most):
    """Stochastic rounding to the top 12 bits, and the blocks' largest.  What is positive throughout keeps code 1 at least."""
    n = x.numel()
    r = ((x.abs().view(torch.int32).long() + (random << 4)) >> 20).clamp(max=0x7FF)
    top = torch.nn.functional.pad(r, (0, -n % BLOCK)).view(-1, BLOCK).amax(1)
    code = r - top.repeat_interleave(BLOCK)[:n] + most
    if most == 255:
        return torch.where(r > 0, code.clamp(min=1), 0).to(torch.uint8), top
    code = code.clamp(min=0)
    return torch.where(code > 0, code + 128 * (x < 0), 0).to(torch.uint8), top


def _adamw_results(s):
    """Whole buffers: parameters, their copy, first and second moments."""
    return (s["flat"], *([s["flat_copy"]] if s["copy"] else []), s["m"], s["v"])


def _plain_adamw(s):
    s["steps"] += 1
    t, total = s["steps"], sum(s["batches"])
    b1, b2 = _float(BETAS[0]), _float(BETAS[1])
    c1, c2 = _float(1 - BETAS[0]), _float(1 - BETAS[1])
    rate, spread = _float(RATE / (1 - BETAS[0] ** t)), _float(1 / math.sqrt(1 - BETAS[1] ** t))
    keep = _float(1 - RATE * DECAY)
    for i, p in enumerate(s["params"]):
        g = torch.zeros_like(p)
        for b, part in zip(s["batches"], s["grads"][i]):
            g = _fma(_float(b / total), part, g)
        m, v = s["moments"][i]
        if s["bits"] == 8:
            cm, cv, top = s["state"][i]
            m.copy_(_values(cm, top[:, 0], 127))
            v.copy_(_values(cv, top[:, 1], 255))
        m.copy_(_fma(b1, m, c1 * g))
        v.copy_(_fma(c2 * g, g, b2 * v))
        p.copy_(_fma(-rate, m / _fma(torch.sqrt(v), spread, torch.tensor(_float(EPS))), keep * p))
        if s["copy"]:
            s["copies"][i].copy_(p)
        if s["bits"] == 8:
            random = _random_bits(p.numel(), i, t)
            for x, codes, axis, most, bits in ((m, cm, 0, 127, random & 0xFFFF), (v, cv, 1, 255, random >> 16)):
                new, largest = _codes(x, bits, most)
                codes.copy_(new)
                top[:, axis] = largest
                x.copy_(_values(codes, top[:, axis], most))
    return _adamw_results(s)


def _plain(s):
    return {"rotary": _plain_rotary, "policy": _plain_policy, "adamw": _plain_adamw}[s["op"]](s)


# ------------------------------------------------------------------------------------------------
# The framework's operators
# ------------------------------------------------------------------------------------------------

_context = []


def _operator(s):
    """The operator object of this state, on the process's one context."""
    from paper_2503_17469_b200 import binding, language

    if not _context:
        _context.append(binding.Omni(1, 1, 1, 1))
    if s["op"] == "rotary":
        return language.Rotary(_context[0], s["heads"], s["kv_heads"], s["dim"], s["frequencies"], axes=s["axis"],
                               interleaved=s["interleaved"], eps=1e-6)
    if s["op"] == "policy":
        return language.Policy(_context[0], clip=CLIP[0], clip_high=CLIP[1], kl=s["kl"], temperature=s["temperature"])
    return language.AdamW(_context[0], s["params"], s["grads"], copies=s["copies"], betas=BETAS, eps=EPS, weight_decay=DECAY,
                          bits=s["bits"], state=s["state"], steps=s["steps"])


def _own(s):
    f = s.get("operator")
    if f is None:
        f = s["operator"] = _operator(s)
    if s["op"] == "rotary":
        given = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], lengths=s["lengths"])
        if s["way"] == "forward":
            return f.forward(s["q"], s["k"], s["positions"], **given)
        out = f.backward(s["q"], s["k"], s["positions"], s["grad_q"], s["grad_k"], **given)
        return out if s["norm"] else out[:2]
    if s["op"] == "adamw":
        f.step(RATE, s["batches"])
        if s["bits"] == 8:
            f.moments(out=s["moments"])
        return _adamw_results(s)
    if s["way"] == "logprob":
        return f.logprob(s["logits"], s["tokens"])
    reference = s["reference"] if s["kl"] else None
    if s["way"] == "forward":
        return f.forward(s["logits"], s["tokens"], s["old"], s["advantage"], reference)
    if s["way"] == "backward":
        return f.backward(s["logits"], s["tokens"], s["lse"], s["old"], s["advantage"], s["grad_loss"], reference)
    return f.step(s["logits"], s["tokens"], s["old"], s["advantage"], s["grad_loss"], reference)


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "rotary":
        rows = c["batch"] * c["length"]
        elements = rows * (c["heads"] + c["kv_heads"]) * c["dim"]
        read = 0.5 if c["ragged"] else 1.0             # of a ragged batch about half the rows are there
        moved = (read + 1 if c["way"] == "forward" else 2 * read + 1) * elements * SIZE[c["act"]]
        weights = 2 * c["dim"] * (SIZE[c["act"]] if c["way"] == "forward" else SIZE[c["act"]] + 4) if c["norm"] else 0
        return {"bytes": moved + weights + 8 * c["axes"] * rows, "flops": read * elements * (8 if c["way"] == "forward" else 16)}
    if c["op"] == "policy":
        act, index = SIZE[c["act"]], 8 if c["index"] == "i64" else 4
        values = {"logprob": 2, "forward": 6, "backward": 5, "step": 7}[c["way"]] - (0 if c["kl"] or c["way"] == "logprob" else 1)
        row = c["vocab"] * act * (2 if c["way"] in ("backward", "step") else 1) + index + 4 * values
        return {"bytes": c["rows"] * row, "flops": c["rows"] * c["vocab"] * (6 if c["way"] == "step" else 4 if c["way"] == "backward" else 3)}
    # codes of 8 bits are read and written, and written once more as the floats that they stand for
    n = sum(_sizes(c))
    states = 16 if c["bits"] == 32 else 4 + 8 + 8 / BLOCK
    return {"bytes": n * (c["K"] * SIZE[c["act"]] + 8 + (2 if c["copy"] else 0) + states), "flops": n * (2 * c["K"] + 14)}


# ------------------------------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# ------------------------------------------------------------------------------------------------

def _exact_rotary(s):
    """Rotations as products of complex numbers; the norm's gradient as that of x / |x|."""
    r, d, n = s["rotated"], s["dim"], s["length"]
    axis = torch.tensor(s["axis"], device="cuda")
    frequency = torch.tensor(s["frequencies"], device="cuda", dtype=torch.float64)
    results, weights = [], []
    for name in ("q", "k"):
        x = s[name].double()
        w = s[name + "_weight"].double() if s["norm"] else None
        y = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        dw = torch.zeros(d, dtype=torch.float64, device="cuda")
        for b in range(s["batch"]):
            m = n if s["lengths"] is None else int(s["lengths"][b])
            if m == 0:
                continue
            angle = s["positions"][:, b, :m].double()[axis].T * frequency
            turn = torch.polar(torch.ones_like(angle), angle if s["way"] == "forward" else -angle)[:, None]

            def rotate(v):
                first, rest = v[..., :r], v[..., r:]
                pair = first.unflatten(-1, (r // 2, 2)) if s["interleaved"] else first.unflatten(-1, (2, r // 2)).transpose(-1, -2)
                z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
                z = z if s["interleaved"] else z.transpose(-1, -2)
                return torch.cat([z.flatten(-2), rest], -1)

            xb = x[b, :m]
            length = torch.sqrt(xb.square().sum(-1, keepdim=True) + d * 1e-6) / math.sqrt(d)
            if s["way"] == "forward":
                y[b, :m] = rotate(xb / length * w if s["norm"] else xb)
                continue
            g = rotate(s["grad_" + name][b, :m].double())
            if s["norm"]:
                dw += (g * xb / length).sum((0, 1))
                g = g * w
                g = g / length - xb * (g * xb).sum(-1, keepdim=True) / (d * length ** 3)
            y[b, :m] = g
        results.append(y)
        weights.append(dw)
    return tuple(results + (weights if s["way"] == "backward" and s["norm"] else []))


def _exact_policy(s):
    """Blocks of rows; the surrogate by the sign of its advantage."""
    temp, low, high = s["temperature"], 1.0 - CLIP[0], 1.0 + CLIP[1]
    parts = [[], [], [], []]
    step = max(1, (1 << 26) // s["vocab"])
    for i in range(0, s["rows"], step):
        cut = slice(i, i + step)
        z = s["logits"][cut].double() / temp
        tokens = s["tokens"][cut].long()
        there, at = tokens >= 0, tokens.clamp(min=0)[:, None]
        lse = s["lse"][cut].double() if s["way"] == "backward" else torch.logsumexp(z, 1)
        logp = z.gather(1, at)[:, 0] - lse
        a, gap = s["advantage"][cut].double(), s["reference"][cut].double() - logp
        ratio = torch.exp(logp - s["old"][cut].double())
        active = torch.where(a > 0, ratio <= high, ratio >= low)
        surrogate = torch.where(active, ratio, torch.where(a > 0, high, low)) * a
        loss = s["kl"] * (torch.exp(gap) - gap - 1.0) - surrogate
        parts[0].append(torch.where(there, loss, 0.0))
        parts[1].append(torch.where(there, logp, 0.0))
        parts[2].append(lse)
        if s["way"] in ("backward", "step"):
            slope = s["kl"] * (1.0 - torch.exp(gap)) - active * ratio * a
            one = torch.zeros_like(z).scatter_(1, at, 1.0)
            parts[3].append((one - torch.exp(z - lse[:, None])) * (there * slope * s["grad_loss"][cut].double() / temp)[:, None])
    loss, logp, lse, grad = (torch.cat(x) if x else None for x in parts)
    return {"logprob": (logp, lse), "forward": (loss, logp, lse), "backward": grad, "step": (loss, logp, lse, grad)}[s["way"]]


def _exact_adamw(s):
    """What is kept in 8 bits has no such value: rounded by random bits, a moment next to a border of its codes goes either way
    with the last bit of the float that it is rounded from, by the whole step of an eighth of an octave."""
    t, total = s["steps"] + 1, sum(s["batches"])
    p_all, m_all, v_all = (torch.zeros(s["flat"].numel(), dtype=torch.float64, device="cuda") for _ in range(3))
    for i, (p, p1, m1, v1) in enumerate(zip(s["params"], *(_views(x, s["sizes"]) for x in (p_all, m_all, v_all)))):
        g = sum(part.double() * (b / total) for b, part in zip(s["batches"], s["grads"][i]))
        m, v = (x.double() for x in s["moments"][i])
        if s["bits"] == 8:
            cm, cv, top = s["state"][i]
            m, v = _values(cm, top[:, 0], 127).double(), _values(cv, top[:, 1], 255).double()
        m1.copy_(BETAS[0] * m + (1 - BETAS[0]) * g)
        v1.copy_(BETAS[1] * v + (1 - BETAS[1]) * g * g)
        step = m1 / (1 - BETAS[0] ** t) / (torch.sqrt(v1 / (1 - BETAS[1] ** t)) + EPS)
        p1.copy_(p.double() - RATE * (step + DECAY * p.double()))
    moments = (m_all, v_all) if s["bits"] == 32 else (None, None)
    return (p_all, *([p_all] if s["copy"] else []), *moments)


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "policy": _exact_policy, "adamw": _exact_adamw}[case["op"]](s)
