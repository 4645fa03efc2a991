"""What the language-model operators are measured on: cases, their inputs, and the operators in plain form.

A worker of the data-parallel step computes a language model's gradients between three operators:
the embedding at the bottom (lookup, and its dense gradient that goes into a gradient bucket),
attention in the blocks (forward, and backward from the kept log-sum-exp), and a distillation loss
on top (forward, backward, or both in one pass).  A case names an operator and a direction.

``own`` false: elementary torch operations in float32, rounded once at the end.  ``own`` true: the
calls of ``paper_2503_17469_b200.language``.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # a short prompt's lookup in a float table: a latency-bound call
        dict(name="embed_fwd_short", op="embed", way="forward", n=257, vocab=8192, dim=512, table="f32", act="f32", index="i64"),
        # one worker's large batch, from the bfloat16 copy of the parameters
        dict(name="embed_fwd_batch", op="embed", way="forward", n=65536, vocab=50257, dim=1024, table="bf16", act="bf16", index="i64"),
        # a small character-level model: odd vocabulary and width, rows that no 16-byte access fits
        dict(name="embed_grad_odd", op="embed", way="backward", n=1500, vocab=331, dim=99, table="f32", act="f32", index="i32"),
        # the dense gradient of a large table into a float gradient bucket
        dict(name="embed_grad_batch", op="embed", way="backward", n=32768, vocab=50257, dim=768, table="f32", act="bf16", index="i64"),
        # short sequences: a few tiles for the whole GPU
        dict(name="attn_fwd_short", op="attn", way="forward", batch=4, q_len=128, kv_len=128, heads=8, kv_heads=8, dim=64, causal=True, ragged=False),
        # long causal context with shared key/value heads
        dict(name="attn_fwd_long", op="attn", way="forward", batch=2, q_len=4096, kv_len=4096, heads=16, kv_heads=4, dim=128, causal=True, ragged=False),
        # a padded batch of sequences of different lengths, one of them empty; odd length, a head of 80
        dict(name="attn_bwd_ragged", op="attn", way="backward", batch=6, q_len=777, kv_len=777, heads=12, kv_heads=4, dim=80, causal=True, ragged=True),
        # the longest training context
        dict(name="attn_bwd_long", op="attn", way="backward", batch=1, q_len=8192, kv_len=8192, heads=16, kv_heads=8, dim=128, causal=True, ragged=False),
        # a small model's loss with its gradient: a latency-bound call
        dict(name="distill_step_small", op="distill", way="step", rows=48, vocab=1000, top=8, act="f32", index="i64", temperature=1.0),
        # one worker's batch: loss and gradient in one pass over logits whose rows are 2-byte aligned only
        dict(name="distill_step_batch", op="distill", way="step", rows=8192, vocab=50257, top=64, act="bf16", index="i32", temperature=2.0),
        # evaluation on a large vocabulary: the loss alone
        dict(name="distill_fwd_wide", op="distill", way="forward", rows=3000, vocab=131072, top=32, act="bf16", index="i32", temperature=1.0),
        # the gradient alone, from the kept log-sum-exp, as an autograd backward asks for it
        dict(name="distill_bwd", op="distill", way="backward", rows=4096, vocab=32000, top=20, act="f32", index="i64", temperature=4.0),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm; odd ones as they fall.
    Multiples of 1024 move off by one: the listed cases have such sizes."""
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return x - 1 if x % 1024 == 0 else x


def draw(rng):
    op = rng.choice(("embed", "attn", "distill"))
    index = rng.choice(("i32", "i64"))
    if op == "embed":
        dim = rng.choice((_log(rng, 16, 2048), 8 * _log(rng, 4, 256)))
        vocab = _log(rng, 100, 131072)
        n = _log(rng, 1, min(131072, (1 << 27) // dim))
        vocab = min(vocab, (1 << 27) // dim)
        return dict(op=op, way=rng.choice(("forward", "backward", "backward")), n=n, vocab=vocab, dim=dim,
                    table=rng.choice(("f32", "bf16")), act=rng.choice(("f32", "bf16")), index=index)
    if op == "attn":
        kv_heads = rng.choice((1, 2, 4, 8))
        heads = kv_heads * rng.choice((1, 2, 3, 4))
        dim = rng.choice((64, 128, 8 * rng.randint(2, 16)))
        batch = rng.choice((1, 2, 3, 5, 8))
        causal = rng.random() < 0.7
        most = min(8192, int(math.sqrt((1 << (30 if causal else 29)) / (batch * heads))))
        q_len = _log(rng, 1, most)
        kv_len = q_len if rng.random() < 0.7 else _log(rng, 1, most)
        return dict(op=op, way=rng.choice(("forward", "backward")), batch=batch, q_len=q_len, kv_len=kv_len, heads=heads,
                    kv_heads=kv_heads, dim=dim, causal=causal, ragged=rng.random() < 0.4)
    vocab = _log(rng, 100, 200000)
    act = rng.choice(("f32", "bf16"))
    rows = _log(rng, 1, min(16384, 800_000_000 // (vocab * SIZE[act])))
    return dict(op=op, way=rng.choice(("forward", "backward", "step", "step")), rows=rows, vocab=vocab,
                top=min(vocab // 2, _log(rng, 1, 256)), act=act, index=index, temperature=rng.choice((1.0, 2.0, 4.0)))


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------

def _normal(gen, shape, std, dtype):
    return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0.0, std, generator=gen).to(dtype)


def _prepare_embed(c, gen):
    """Tokens by a Zipf law (rank and id alike, as tokenizers number them), one in 64 of them padding."""
    u = torch.rand(c["n"], device="cuda", generator=gen)
    tokens = (torch.exp(u * math.log(c["vocab"] + 1.0)) - 1.0).long().clamp_(0, c["vocab"] - 1)
    tokens[torch.rand(c["n"], device="cuda", generator=gen) < 1 / 64] = 0
    s = dict(c, tokens=tokens.int() if c["index"] == "i32" else tokens, scale=math.sqrt(c["dim"]))
    if c["way"] == "forward":
        s["weight"] = _normal(gen, (c["vocab"], c["dim"]), 0.05, DTYPES[c["table"]])
    else:
        s["dout"] = _normal(gen, (c["n"], c["dim"]), 1e-3, DTYPES[c["act"]])
    return s


def _lengths(c, gen):
    """Lengths of a padded batch: the first full, the last empty where there are more than two.
    Queries and keys of one sequence where the padded lengths agree, of two where they do not."""
    if not c["ragged"]:
        return None, None
    u = torch.rand(2, c["batch"], device="cuda", generator=gen)
    u[:, 0] = 1.0
    if c["batch"] > 2:
        u[:, -1] = 0.0
    kv = 0 if c["q_len"] == c["kv_len"] else 1
    return torch.ceil(u[0] * c["q_len"]).int(), torch.ceil(u[kv] * c["kv_len"]).int()


def _prepare_attn(c, gen):
    """Queries, keys and values as slices of one projection's output where the lengths agree."""
    b, h, hk, d = c["batch"], c["heads"], c["kv_heads"], c["dim"]
    if c["q_len"] == c["kv_len"]:
        packed = _normal(gen, (b, c["q_len"], h + 2 * hk, d), 1.0, torch.bfloat16)
        q, k, v = packed[:, :, :h], packed[:, :, h:h + hk], packed[:, :, h + hk:]
    else:
        q = _normal(gen, (b, c["q_len"], h, d), 1.0, torch.bfloat16)
        k = _normal(gen, (b, c["kv_len"], hk, d), 1.0, torch.bfloat16)
        v = _normal(gen, (b, c["kv_len"], hk, d), 1.0, torch.bfloat16)
    q_lengths, kv_lengths = _lengths(c, gen)
    s = dict(c, q=q, k=k, v=v, q_lengths=q_lengths, kv_lengths=kv_lengths, scale=1.0 / math.sqrt(d))
    if c["way"] == "backward":
        s["out"], s["lse"] = _plain_attn_forward(s)
        s["dout"] = _normal(gen, (b, c["q_len"], h, d), 1.0, torch.bfloat16)
    return s


def _prepare_distill(c, gen):
    """A student's logits, the top logits of a teacher near it, and rows without a target (prompt
    tokens).  The last columns are the padding of the vocabulary: -inf for the student."""
    rows, vocab, top = c["rows"], c["vocab"], c["top"]
    logits = _normal(gen, (rows, vocab), 2.0, torch.float32)
    logits[:, vocab - vocab // 64:] = -math.inf
    logits = logits.to(DTYPES[c["act"]])
    teacher = logits.float() + _normal(gen, (rows, vocab), 1.0, torch.float32)
    top_logits, top_index = torch.topk(teacher, top, dim=1)
    del teacher
    top_index[torch.rand(rows, device="cuda", generator=gen) < 0.1] = -1
    s = dict(c, logits=logits, top_logits=top_logits, top_index=top_index.int() if c["index"] == "i32" else top_index)
    if c["way"] != "forward":
        s["dloss"] = torch.full((rows,), 1.0 / rows, device="cuda")
    if c["way"] == "backward":
        s["lse"] = torch.logsumexp(logits.double() / c["temperature"], dim=1).float()
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"embed": _prepare_embed, "attn": _prepare_attn, "distill": _prepare_distill}[case["op"]](case, gen)


# ------------------------------------------------------------------------------------------------
# The plain forms
# ------------------------------------------------------------------------------------------------

def _plain_embed(s):
    tokens = s["tokens"].long()
    if s["way"] == "forward":
        return (s["weight"][tokens].float() * s["scale"]).to(DTYPES[s["act"]])
    rows = s["dout"].float() * s["scale"] * (tokens != 0)[:, None]      # token 0 is the padding: no gradient
    grad = torch.zeros(s["vocab"], s["dim"], device="cuda").index_add_(0, tokens, rows)
    return grad.to(DTYPES[s["table"]])


def _heads_first(x):
    return x.transpose(1, 2).float()


def _shared(x, group):
    """[batch, kv_heads, len, dim] seen by every query head of its group."""
    return x[:, :, None].expand(-1, -1, group, -1, -1).flatten(1, 2)


def _allowed(s):
    """[batch, 1, q_len, kv_len]: which keys a query sees.  Causal is aligned at the sequences' ends."""
    q_len, kv_len = s["q_len"], s["kv_len"]
    i = torch.arange(q_len, device="cuda")[None, :, None]
    j = torch.arange(kv_len, device="cuda")[None, None, :]
    ql = s["q_lengths"][:, None, None] if s["ragged"] else q_len
    kl = s["kv_lengths"][:, None, None] if s["ragged"] else kv_len
    ok = (i < ql) & (j < kl)
    if s["causal"]:
        ok = ok & (j <= i + (kl - ql))
    return ok[:, None]


def _scores(s):
    q, k = _heads_first(s["q"]), _shared(_heads_first(s["k"]), s["heads"] // s["kv_heads"])
    return torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).masked_fill_(~_allowed(s), -math.inf)


def _plain_attn_forward(s):
    x = _scores(s)
    top = x.amax(3, keepdim=True)
    p = torch.exp(x.sub_(top.masked_fill(top == -math.inf, 0.0)))
    total = p.sum(3, keepdim=True)
    v = _shared(_heads_first(s["v"]), s["heads"] // s["kv_heads"])
    out = torch.matmul(p, v) / total.masked_fill(total == 0.0, 1.0)      # a row that sees nothing: zeros
    return out.transpose(1, 2).contiguous().to(torch.bfloat16), (top + torch.log(total))[..., 0]


def _plain_attn_backward(s):
    group = s["heads"] // s["kv_heads"]
    lse = s["lse"][..., None]
    p = torch.exp(_scores(s).sub_(lse.masked_fill(lse == -math.inf, 0.0)))
    do, v = _heads_first(s["dout"]), _shared(_heads_first(s["v"]), group)
    dv = torch.matmul(p.transpose(2, 3), do)
    delta = (do * _heads_first(s["out"])).sum(3, keepdim=True)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_(delta).mul_(p).mul_(s["scale"])
    dq = torch.matmul(ds, _shared(_heads_first(s["k"]), group))
    dk = torch.matmul(ds.transpose(2, 3), _heads_first(s["q"]))
    dk, dv = (x.unflatten(1, (s["kv_heads"], group)).sum(2) for x in (dk, dv))
    return tuple(x.transpose(1, 2).contiguous().to(torch.bfloat16) for x in (dq, dk, dv))


def _teacher(s):
    """Probabilities over the teacher's entries, and where they stand; an entry of index -1 is none."""
    index = s["top_index"].long()
    there = index >= 0
    t = (s["top_logits"] / s["temperature"]).masked_fill(~there, -math.inf)
    e = torch.exp(t - t.amax(1, keepdim=True).clamp(min=-3e38))
    total = e.sum(1, keepdim=True)
    return e / total.masked_fill(total == 0.0, 1.0), index.clamp(min=0)


def _plain_distill(s):
    p, index = _teacher(s)
    temp = s["temperature"]
    z = s["logits"].float() / temp
    if s["way"] == "backward":
        lse = s["lse"]
    else:
        top = z.amax(1, keepdim=True)
        lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))[:, 0]
        gap = torch.log(p.clamp(min=1e-38)) - (torch.gather(z, 1, index) - lse[:, None])
        loss = temp * temp * (p * gap).sum(1)
        if s["way"] == "forward":
            return loss, lse
    q = torch.exp(z - lse[:, None]) * (p.sum(1, keepdim=True) > 0.5)       # a row without a target: no gradient
    dlogits = (q.scatter_add_(1, index, -p) * (s["dloss"][:, None] * temp)).to(s["logits"].dtype)
    return dlogits if s["way"] == "backward" else (loss, lse, dlogits)


def _plain(s):
    if s["op"] == "embed":
        return _plain_embed(s)
    if s["op"] == "distill":
        return _plain_distill(s)
    return _plain_attn_forward(s) if s["way"] == "forward" else _plain_attn_backward(s)


# ------------------------------------------------------------------------------------------------
# The framework's operators
# ------------------------------------------------------------------------------------------------

_context = []


def _operator(s):
    """The operator object of this state, on the process's one context."""
    from paper_2503_17469_b200 import binding, language

    if not _context:
        _context.append(binding.Omni(1, 1, 1, 1))
    if s["op"] == "embed":
        return language.Embedding(_context[0], s["vocab"], s["dim"], scale=s["scale"], padding=0)
    if s["op"] == "attn":
        return language.Attention(_context[0], s["heads"], s["kv_heads"], s["dim"], causal=s["causal"], scale=s["scale"])
    return language.Distillation(_context[0], s["temperature"])


def _own(s):
    f = s.get("operator")
    if f is None:
        f = s["operator"] = _operator(s)
    if s["op"] == "embed":
        if s["way"] == "forward":
            return f.forward(s["tokens"], s["weight"], dtype=DTYPES[s["act"]])
        return f.backward(s["tokens"], s["dout"], dtype=DTYPES[s["table"]])
    if s["op"] == "attn":
        if s["way"] == "forward":
            return f.forward(s["q"], s["k"], s["v"], s["q_lengths"], s["kv_lengths"])
        return f.backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["q_lengths"], s["kv_lengths"])
    if s["way"] == "forward":
        return f.forward(s["logits"], s["top_logits"], s["top_index"])
    if s["way"] == "backward":
        return f.backward(s["logits"], s["top_logits"], s["top_index"], s["lse"], s["dloss"])
    return f.step(s["logits"], s["top_logits"], s["top_index"], s["dloss"])


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------------

def _distinct(n, vocab):
    """How many different tokens n draws of the Zipf law name, on average."""
    rank = torch.arange(1, vocab + 1, dtype=torch.float64)
    return float((1 - (1 - torch.log1p(1 / rank) / math.log(vocab + 1.0)) ** n).sum())


def work(case):
    c = case
    if c["op"] == "embed":
        act, table, index = SIZE[c["act"]], SIZE[c["table"]], 8 if c["index"] == "i64" else 4
        if c["way"] == "forward":
            rows = _distinct(c["n"], c["vocab"])
            return {"bytes": c["n"] * (index + act * c["dim"]) + rows * table * c["dim"], "flops": c["n"] * c["dim"]}
        return {"bytes": c["n"] * (index + act * c["dim"]) + c["vocab"] * c["dim"] * table, "flops": 2 * c["n"] * c["dim"]}
    if c["op"] == "attn":
        # pairs of a query and a key that it sees; of a ragged batch about two fifths
        ql, kl = c["q_len"], c["kv_len"]
        pairs = ql * kl
        if c["causal"]:
            first = kl - ql                       # keys before the first query's own
            pairs = ql * kl - ql * (ql - 1) // 2 if first >= 0 else kl * (kl + 1) // 2
        if c["ragged"]:
            pairs = pairs * 0.4
        products = 2 if c["way"] == "forward" else 5
        q_bytes, kv_bytes = 2 * c["batch"] * ql * c["heads"] * c["dim"], 2 * c["batch"] * kl * c["kv_heads"] * c["dim"]
        lse = 4 * c["batch"] * c["heads"] * ql
        moved = 2 * q_bytes + 2 * kv_bytes + lse if c["way"] == "forward" else 4 * q_bytes + 4 * kv_bytes + lse
        return {"bytes": moved, "flops": 2 * products * c["batch"] * c["heads"] * pairs * c["dim"]}
    act, index = SIZE[c["act"]], 8 if c["index"] == "i64" else 4
    row = c["vocab"] * act * (1 if c["way"] == "forward" else 2) + c["top"] * (4 + index) + 12
    return {"bytes": c["rows"] * row, "flops": c["rows"] * c["vocab"] * (4 if c["way"] == "backward" else 3 if c["way"] == "forward" else 6)}


# ------------------------------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# ------------------------------------------------------------------------------------------------

def _exact_embed(s):
    scale = float(s["scale"])
    if s["way"] == "forward":
        return torch.index_select(s["weight"].double(), 0, s["tokens"].long()) * scale
    order = torch.sort(s["tokens"].long()).indices
    ids, counts = torch.unique_consecutive(s["tokens"].long()[order], return_counts=True)
    at = torch.repeat_interleave(torch.arange(len(ids), device="cuda"), counts)
    sums = torch.zeros(len(ids), s["dim"], dtype=torch.float64, device="cuda")
    sums.index_add_(0, at, s["dout"][order].double())
    grad = torch.zeros(s["vocab"], s["dim"], dtype=torch.float64, device="cuda")
    grad[ids] = sums * scale
    grad[0] = 0.0
    return grad


def _exact_attn(s):
    """One sequence and one head after the other, on the keys and queries that are there."""
    group = s["heads"] // s["kv_heads"]
    new = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, dq, dk, dv = new(s["q"]), new(s["q"]), new(s["k"]), new(s["v"])
    lse = torch.full((s["batch"], s["heads"], s["q_len"]), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(s["batch"]):
        ql = int(s["q_lengths"][b]) if s["ragged"] else s["q_len"]
        kl = int(s["kv_lengths"][b]) if s["ragged"] else s["kv_len"]
        first = max(0, ql - kl) if s["causal"] else 0 if kl else ql          # queries before this one see nothing
        if first >= ql or kl == 0:
            continue
        for h in range(s["heads"]):
            q, k, v = s["q"][b, first:ql, h].double(), s["k"][b, :kl, h // group].double(), s["v"][b, :kl, h // group].double()
            x = (q @ k.T) * s["scale"]
            if s["causal"]:
                x += torch.triu(torch.full_like(x, -math.inf), diagonal=kl - ql + first + 1)
            if s["way"] == "forward":
                lse[b, h, first:ql] = torch.logsumexp(x, 1)
                out[b, first:ql, h] = torch.softmax(x, 1) @ v
                continue
            p = torch.exp(x - s["lse"][b, h, first:ql].double()[:, None])
            do, o = s["dout"][b, first:ql, h].double(), s["out"][b, first:ql, h].double()
            ds = p * (do @ v.T - (do * o).sum(1, keepdim=True)) * s["scale"]
            dq[b, first:ql, h] = ds @ k
            dk[b, :kl, h // group] += ds.T @ q
            dv[b, :kl, h // group] += p.T @ do
    return (out, lse) if s["way"] == "forward" else (dq, dk, dv)


def _exact_distill(s):
    """Blocks of rows; the sum over the teacher's entries that are there."""
    loss, lse, grad = [], [], []
    temp = s["temperature"]
    step = max(1, (1 << 26) // s["vocab"])
    for a in range(0, s["rows"], step):
        z = s["logits"][a:a + step].double() / temp
        index = s["top_index"][a:a + step].long()
        t = torch.where(index >= 0, s["top_logits"][a:a + step].double() / temp, -math.inf)
        target = index[:, :1] >= 0
        p = torch.where(target, torch.softmax(t, 1), 0.0).nan_to_num(0.0)
        l = s["lse"][a:a + step].double() if s["way"] == "backward" else torch.logsumexp(z, 1)
        if s["way"] != "backward":
            loss.append(temp * temp * torch.where(p > 0, p * (torch.log(p) - z.gather(1, index.clamp(min=0)) + l[:, None]), 0.0).sum(1))
            lse.append(l)
        if s["way"] != "forward":
            dense = torch.zeros_like(z).scatter_add_(1, index.clamp(min=0), p)
            grad.append(torch.where(target, torch.exp(z - l[:, None]) - dense, 0.0) * (temp * s["dloss"][a:a + step].double()[:, None]))
    loss, lse, grad = (torch.cat(x) if x else None for x in (loss, lse, grad))
    return {"forward": (loss, lse), "backward": grad, "step": (loss, lse, grad)}[s["way"]]


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "attn": _exact_attn, "distill": _exact_distill}[case["op"]](s)
