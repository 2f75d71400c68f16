"""Timed cases of the 4-bit state store, the attention that reads it, the weights that attention gives its keys, and eviction by them.

A state store keeps the keys and values of tokens in pages.  In 8 bits (`States`) a row (one token and head) has one step; in 4 bits (`States4`) it has a step a / 6, a its
largest magnitude, and for each 32 values a factor r: codes are of the eight magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a sign, nearest to 6 x / (r a), ties to the even code,
r the smallest of the numbers (1 + m / 8) 2^e from 2^-13 to 1 with which no code is cut off.  A case is one pass of one operator:

  op        "write"     a call that quantises new tokens' keys and values into their slots, and one that reads them back (4 bits)
            "chunk"     attention of every sequence's newest tokens over its own pages, causal (4 bits)
            "passages"  attention over the states of the passages that a search returned for each sequence (4 bits)
            "weights"   the attention weight that each key gets from a sequence's newest tokens, added to what it had before (8 or 4 bits)
            "evict"     the keys with the largest sums of weights and the newest ones of each sequence and head are moved to other pages, and read back (8 or 4 bits)
  type      "bf16", "f16" or "f32": what is written, read, asked and answered
  heads, group, dim, page   heads of the store, query heads for each of them, values a head, tokens a page
  bits      of the store, where both are offered

and the lengths, which follow from the case alone (content, page numbers and passages follow from the seed):

  write            tokens; run (tokens of one sequence that lie one after the other); sliced (keys and values are parts of one fused projection)
  chunk, weights   sequences, new (most new tokens of a sequence), context (most tokens before them), ragged
  passages         sequences, new, k (passages of a sequence), length (most tokens of a passage), stock (passages in the store), ragged, weighted
  evict            sequences, context (most tokens of a sequence), budget (tokens kept of each), recent (of them the newest), ragged
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
FACTORS = [(1 + m / 8) * 2.0 ** e for e in range(-13, 1) for m in range(8)][:105]          # of bytes 0x10 (2^-13) to 0x78 (1): a binary16 number without its sign and last seven bits


def _write(name, tokens, heads, dim, page, run, type="bf16", sliced=False):
    return dict(name=name, op="write", tokens=tokens, heads=heads, dim=dim, page=page, run=run, type=type, sliced=sliced)


def _chunk(name, sequences, new, context, heads, group, dim, page, type="bf16", ragged=True):
    return dict(name=name, op="chunk", sequences=sequences, new=new, context=context, heads=heads, group=group, dim=dim, page=page, type=type, ragged=ragged)


def _passages(name, sequences, new, k, length, stock, heads, group, dim, page, type="bf16", ragged=True, weighted=False):
    return dict(name=name, op="passages", sequences=sequences, new=new, k=k, length=length, stock=stock, heads=heads, group=group, dim=dim, page=page, type=type,
                ragged=ragged, weighted=weighted)


def _weights(name, sequences, new, context, heads, group, dim, page, bits, type="bf16", ragged=True):
    return dict(name=name, op="weights", sequences=sequences, new=new, context=context, heads=heads, group=group, dim=dim, page=page, bits=bits, type=type, ragged=ragged)


def _evict(name, sequences, context, budget, recent, heads, dim, page, bits, type="bf16", ragged=True):
    return dict(name=name, op="evict", sequences=sequences, context=context, budget=budget, recent=recent, heads=heads, dim=dim, page=page, bits=bits, type=type, ragged=ragged)


def listed():
    return [
        # one decoding step of a small batch: a token each, latency counts
        _write("write4-step", 8, 8, 128, 64, 1),
        # passages taken into the store after an encoder has run over them, in bulk, from slices of its fused projection
        _write("write4-passages", 50_000, 8, 128, 64, 411, sliced=True),
        # the next token of one conversation: latency counts
        _chunk("token4-one", 1, 1, 4000, 8, 4, 128, 64, ragged=False),
        # the next token of a serving batch, every conversation of another length
        _chunk("token4-batch", 64, 1, 8192, 8, 4, 128, 64),
        # a large piece of a long prompt
        _chunk("chunk4-long", 1, 4096, 28_672, 8, 4, 128, 64, ragged=False),
        # a serving batch of single tokens, passages shared between sequences, weighted by the search's scores
        _passages("found4-batch", 48, 1, 10, 400, 1500, 8, 4, 128, 32, weighted=True),
        # questions read in full against their passages, one key head for each query head
        _passages("found4-questions", 24, 96, 10, 512, 1200, 16, 1, 64, 16, type="f16", weighted=True),
        # what every key of a serving batch was worth to the newest token
        _weights("weights-token", 64, 1, 8192, 8, 4, 128, 64, 8),
        # what the keys of long prompts were worth to their last 32 tokens: asked once, before most of them are dropped
        _weights("weights4-window", 4, 32, 16_000, 8, 4, 128, 64, 4, ragged=False),
        # a few heads of odd sizes, more rows than a tile
        _weights("weights-odd", 3, 100, 1000, 5, 3, 96, 16, 8, type="f16"),
        # conversations cut back to a budget
        _evict("evict4-batch", 32, 6000, 2048, 256, 8, 128, 64, 4),
        # one long document cut down once
        _evict("evict-long", 1, 100_000, 12_000, 500, 8, 128, 128, 8, ragged=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "chunk", "chunk", "passages", "weights", "weights", "evict", "evict"])
    base = dict(op=op, heads=rng.choice([1, 2, 3, 4, 8, 8, 16]), dim=rng.choice([32, 64, 96, 128, 128]), page=rng.choice([16, 32, 64, 128]))
    if op == "write":
        tokens = _log_int(rng, 1, 60_000)
        c = dict(base, tokens=tokens, run=min(tokens, _log_int(rng, 1, 5000)), type=rng.choice(["bf16", "f16", "f32"]), sliced=rng.random() < 0.4)
        while work(c)["bytes"] > 3e8:
            c["tokens"] = c["tokens"] // 2 + 1
            c["run"] = min(c["run"], c["tokens"])
        return c
    base.update(type=rng.choice(["bf16", "bf16", "f16"]), ragged=rng.random() < 0.8)
    if op == "evict":
        c = dict(base, sequences=_log_int(rng, 1, 64), context=_log_int(rng, 1, 100_000), bits=rng.choice([8, 4]))
        while work(dict(c, budget=c["context"], recent=0))["bytes"] > 1e9:
            at = "sequences" if c["sequences"] > 1 and rng.random() < 0.7 else "context"
            c[at] = c[at] // 2 + 1 if c[at] > 2 else 1
        budget = min(c["context"], _log_int(rng, 1, 20_000))
        return dict(c, budget=budget, recent=rng.choice([0, min(budget, 16), budget // 4, budget]))
    base.update(group=rng.choice([1, 2, 4, 4, 6, 8]))
    new = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 64, 2048)])
    if op == "passages":
        stock = _log_int(rng, 20, 1500)
        c = dict(base, sequences=_log_int(rng, 1, 64), new=min(new, 300), k=min(stock, rng.choice([1, 3, 5, 10, 10, 20])), length=_log_int(rng, 4, 700), stock=stock, weighted=rng.random() < 0.5)
        shrink = ("sequences", "stock")
    else:
        c = dict(base, sequences=_log_int(rng, 1, 64), new=new, context=_log_int(rng, 1, 60_000))
        if op == "weights":
            c.update(bits=rng.choice([8, 4]), new=min(new, 300))
        shrink = ("sequences", "context")
    # no case costs more than the largest listed ones: products, states held, and the matrix of scores that the plain form makes
    while True:
        keys = c["k"] * (c["length"] + c["page"]) if op == "passages" else c["context"] + c["new"] + c["page"]
        held = 8 * c["heads"] * c["dim"] * max(keys * c["sequences"], c["stock"] * (c["length"] + c["page"]) if op == "passages" else 0)
        if work(c)["flops"] < 1e12 and held < 6e9 and 4 * c["sequences"] * c["new"] * c["group"] * c["heads"] * keys < 8e9:
            return c
        at = shrink[0] if c[shrink[0]] > 1 and rng.random() < 0.7 else shrink[1]
        c[at] = c[at] // 2 + 1 if c[at] > 2 else 1
        if op == "passages":
            c["k"] = min(c["k"], c["stock"])
        if all(c[s] <= 2 for s in shrink):
            c["new"] = c["new"] // 2 + 1


# ---------------------------------------------------------------------------------------------------------------
# Lengths: from the case alone.

def _spread(n, most, ragged, at=0.0):
    """n lengths between a quarter of `most` and `most`, spread evenly over the range in an order without a pattern; the first is `most`."""
    return [most if not ragged or i == 0 else max(1, int(most * (0.25 + 0.75 * ((i * 0.6180339887 + at) % 1.0)))) for i in range(n)]


def _lengths(case):
    """(new tokens of each sequence, tokens before them)"""
    return _spread(case["sequences"], case["new"], case["ragged"], 0.3), _spread(case["sequences"], case["context"], case["ragged"])


def _stock(case):
    return _spread(case["stock"], case["length"], case["ragged"])


def work(case):
    """Bytes and operations of one pass.  What a passages case reads depends on which passages are named: every sequence's are counted, but no more
    than the whole stock once."""
    H, D, e = case["heads"], case["dim"], 4 if case["type"] == "f32" else 2
    side = D + 4 if case.get("bits") == 8 else D // 2 + 8           # bytes of a row of keys, or of values
    if case["op"] == "write":
        T = case["tokens"]
        return {"bytes": 2 * (2 * T * H * D * e + 2 * T * H * side + 8 * T), "flops": 0}
    if case["op"] == "evict":
        lens = _spread(case["sequences"], case["context"], case["ragged"])
        kept = sum(min(n, case["budget"]) for n in lens)
        # sums read; rows read and written, their numbers and sums written; rows read back, the values written
        return {"bytes": H * (4 * sum(lens) + kept * (4 * side + 8) + kept * (2 * side + 2 * D * e)), "flops": 0}
    G, D2 = case["group"], 2 * D
    if case["op"] == "passages":
        new, lens = _spread(case["sequences"], case["new"], case["ragged"], 0.3), _stock(case)
        mean = sum(lens) / len(lens)
        pairs, keys = sum(new) * case["k"] * mean, mean * min(case["stock"], case["sequences"] * case["k"])
    else:
        new, before = _lengths(case)
        pairs = sum(n * b + n * (n + 1) // 2 for n, b in zip(new, before))
        keys = sum(n + b for n, b in zip(new, before))
    N = sum(new)
    if case["op"] == "weights":
        return {"bytes": N * H * G * D * e + keys * H * (side + 8), "flops": D2 * H * G * pairs}
    return {"bytes": 2 * N * H * G * D * e + 2 * keys * H * side, "flops": 2 * D2 * H * G * pairs}


# ---------------------------------------------------------------------------------------------------------------
# Inputs.

def _quantise8(x):
    """Codes and steps of rows along the last axis, as the 8-bit store holds them."""
    top = x.abs().amax(-1)
    return torch.round(x * 127 / top.clamp_min(2.0 ** -100)[..., None]).to(torch.int8), top / 127


def _quantise4(x):
    """Codes 0 .. 15 (bit 3: the sign), bytes of the factors of each 32 values and steps of rows [..., dim].  In 64 bits, where every product with a level and a factor is exact."""
    size = x.abs().double().unflatten(-1, (-1, 32))
    group = size.amax(-1)
    top = group.amax(-1)
    use = top.clamp_min(2.0 ** -100)
    factors = torch.tensor(FACTORS, dtype=torch.float64, device=x.device)
    index = torch.searchsorted(factors, (group / use[..., None]).contiguous())
    y = size * 6 / (factors[index] * use[..., None])[..., None]
    code = (y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)
    code = code.flatten(-2) + 8 * torch.signbit(x).to(torch.uint8)
    return code, (index + 0x10).to(torch.uint8), top.float() / 6


def _pack_keys(code):
    """[..., dim] -> [..., dim / 2]: components 2 i and 2 i + 1 in byte i"""
    return code[..., 0::2] | code[..., 1::2] << 4


def _pack_values(code):
    """[..., dim] -> [..., dim / 2]: components 32 g + n and 32 g + 16 + n in byte 16 g + n"""
    c = code.unflatten(-1, (-1, 2, 16))
    return (c[..., 0, :] | c[..., 1, :] << 4).flatten(-2)


def _four_bytes(factor):
    """The bytes of a row's factors, four whatever the dimension is."""
    return torch.nn.functional.pad(factor, (0, 4 - factor.shape[-1]))


def _states(shape, g, spread):
    """Rows of encoder or decoder states: components of different sizes with a mean of their own, rows of different lengths."""
    d = shape[-1]
    size = torch.exp(spread * torch.randn(d, generator=g, device="cuda"))
    mean = 0.5 * size * torch.randn(d, generator=g, device="cuda")
    x = torch.randn(shape, generator=g, device="cuda").mul_(size).add_(mean)
    return x.mul_(torch.exp(0.2 * torch.randn(shape[:-1], generator=g, device="cuda"))[..., None])


def _pool(pages, case, g, bits):
    """A store of `pages` pages in use: every slot holds the states of some token."""
    H, P, D = case["heads"], case["page"], case["dim"]
    if bits == 8:
        kc, ks = _quantise8(_states((pages, H, P, D), g, 0.6))
        vc, vs = _quantise8(_states((pages, H, P, D), g, 0.2))
        return dict(k_codes=kc, v_codes=vc.transpose(2, 3).contiguous(), k_scales=ks, v_scales=vs)
    kc, kf, ks = _quantise4(_states((pages, H, P, D), g, 0.6))
    vc, vf, vs = _quantise4(_states((pages, H, P, D), g, 0.2))
    return dict(k_codes=_pack_keys(kc), v_codes=_pack_values(vc).transpose(2, 3).contiguous(), k_factors=_four_bytes(kf), v_factors=_four_bytes(vf), k_scales=ks, v_scales=vs)


def _tables(lengths, pages, P, g, width=None):
    """Page numbers of each sequence, from pages handed out in no order, as a server's allocator leaves them."""
    need = [-(-n // P) for n in lengths]
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    rows = torch.arange(width or max(1, max(need)), device="cuda")[None, :]
    count = torch.tensor(need, device="cuda")[:, None]
    first = torch.tensor([0] + need, device="cuda").cumsum(0)[:-1, None]
    return torch.where(rows < count, order[(first + rows).clamp_max(pages - 1)], torch.zeros((), dtype=torch.int32, device="cuda")).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H, P, D, dtype, bits = case["heads"], case["page"], case["dim"], TYPE[case["type"]], case.get("bits", 4)
    s = dict(op=case["op"], dtype=dtype, page=P, bits=bits)
    if case["op"] == "write":
        T, run = case["tokens"], case["run"]
        count = -(-T // run)
        # each sequence writes `run` tokens after some that it has already
        lengths = [(i * 7919 + 3) % P + run for i in range(count)]
        pages = sum(-(-n // P) for n in lengths) + 3
        s["pool"] = _pool(pages, case, g, bits)
        table = _tables(lengths, pages, P, g).long()
        t = torch.arange(T, device="cuda")
        at = t % run + torch.tensor(lengths, device="cuda")[t // run] - run
        s["slots"] = table[t // run, at // P] * P + at % P
        if case["sliced"]:
            fused = _states((T, 6 * H, D), g, 0.4).to(dtype)
            s["k"], s["v"] = fused[:, 4 * H:5 * H], fused[:, 5 * H:]
        else:
            s["k"], s["v"] = _states((T, H, D), g, 0.6).to(dtype), _states((T, H, D), g, 0.2).to(dtype)
        return s
    if case["op"] == "evict":
        S, B = case["sequences"], case["budget"]
        lengths = _spread(S, case["context"], case["ragged"])
        to = [min(n, B) for n in lengths]
        need = sum(-(-n // P) for n in lengths)
        pages = need + sum(-(-n // P) for n in to) + 2
        s["pool"] = _pool(pages, case, g, bits)
        both = _tables(lengths + to, pages, P, g)
        width, most = -(-max(lengths) // P), -(-B // P)
        s["tables"] = both[:S].contiguous()
        s["to"] = torch.nn.functional.pad(both[S:], (0, max(0, most - width)))[:, :most].contiguous()
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        # sums of weights as attention leaves them: few large ones, many next to nothing, some exactly 0 (keys that no later token could see, or underflow)
        sums = torch.exp(2.5 * torch.randn((S, H, width * P), generator=g, device="cuda"))
        s["sums"] = torch.where(torch.rand(sums.shape, generator=g, device="cuda") < 0.1, torch.zeros((), device="cuda"), sums)
        s["budget"], s["recent"] = B, case["recent"]
        r = torch.arange(B, device="cuda")
        s["slots"] = torch.where(r < s["lengths"][:, None], s["to"].long()[:, r // P] * P + r % P, torch.full((), -1, device="cuda")).flatten()      # of what is kept
        return s
    new = _spread(case["sequences"], case["new"], case["ragged"], 0.3)
    s["q_start"] = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    s["most"] = max(new)
    s["one"] = case["new"] == 1
    s["scale"] = D ** -0.5
    lengths = _stock(case) if case["op"] == "passages" else [n + b for n, b in zip(*_lengths(case))]
    pages = sum(-(-n // P) for n in lengths) + 2
    s["pool"] = _pool(pages, case, g, bits)
    s["tables"] = _tables(lengths, pages, P, g)
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    # a spread of about two between the logits of a row
    s["q"] = (1.3 * torch.randn((sum(new), H * case["group"], D), generator=g, device="cuda")).to(dtype)
    if case["op"] == "weights":
        # what earlier tokens gave
        s["before"] = torch.rand((case["sequences"], H, s["tables"].shape[1] * P), generator=g, device="cuda").square()
    if case["op"] == "passages":
        S, k, n = case["sequences"], case["k"], case["stock"]
        # as searches answer: k different passages, some found by many queries; now and then one fewer (-1)
        liked = torch.rand((S, n), generator=g, device="cuda") + torch.rand((1, n), generator=g, device="cuda")
        s["ids"] = liked.topk(k, dim=1).indices
        if k > 1:
            s["ids"][torch.rand(S, generator=g, device="cuda") < 0.1, k - 1] = -1
        s["scores"] = torch.rand((S, k), generator=g, device="cuda").sort(dim=1).values if case["weighted"] else None
        s["weight"] = -4.0
    return s


# ---------------------------------------------------------------------------------------------------------------
# One pass.

def _plain_values4(codes, factors, steps):
    """Values [..., dim] in float of codes [..., dim] in 0 .. 15, bytes of factors [..., dim / 32] and steps [...]."""
    sign = 1 - 2 * (codes >> 3).float()
    size = (codes & 7).float()
    level = torch.where(size < 4, size / 2, torch.where(size < 6, size - 2, 2 * size - 8))
    r = torch.tensor(FACTORS, device=codes.device)[factors.int() - 0x10]
    return (sign * level).unflatten(-1, (-1, 32)).mul(r[..., None]).flatten(-2).mul(steps[..., None])


def _plain_keys(pool, codes, factors, steps):
    """Values of key rows [..., dim] (8 bits) or [..., dim / 2] (4 bits)."""
    if factors is None:
        return codes.float() * steps[..., None]
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    return _plain_values4(code, factors[..., :code.shape[-1] // 32], steps)


def _plain_rows_of_values(pool, codes, factors, steps):
    """The same of rows of the values' codes, turned to [..., dim] or [..., dim / 2]."""
    if factors is None:
        return codes.float() * steps[..., None]
    c = codes.unflatten(-1, (-1, 1, 16))
    code = torch.cat([c & 15, c >> 4], -2).flatten(-3)
    return _plain_values4(code, factors[..., :code.shape[-1] // 32], steps)


def _plain_write(s):
    pool, slots, P = s["pool"], s["slots"], s["page"]
    page, at = slots // P, slots % P
    k, kf, ks = _quantise4(s["k"].float())
    v, vf, vs = _quantise4(s["v"].float())
    pool["k_codes"][page, :, at] = _pack_keys(k)
    pool["v_codes"][page, :, :, at] = _pack_values(v)
    pool["k_factors"][page, :, at] = _four_bytes(kf)
    pool["v_factors"][page, :, at] = _four_bytes(vf)
    pool["k_scales"][page, :, at] = ks
    pool["v_scales"][page, :, at] = vs


def _plain_read(s):
    """Keys and values of the tokens in s["slots"], zeros where a slot is none."""
    pool, slots, P = s["pool"], s["slots"], s["page"]
    here = slots >= 0
    page, at = slots.clamp_min(0) // P, slots.clamp_min(0) % P
    kf, vf = (pool[n][page, :, at] if n in pool else None for n in ("k_factors", "v_factors"))
    k = _plain_keys(pool, pool["k_codes"][page, :, at], kf, pool["k_scales"][page, :, at])
    v = _plain_rows_of_values(pool, pool["v_codes"][page, :, :, at], vf, pool["v_scales"][page, :, at])
    zero = torch.zeros((), device=slots.device)
    return torch.where(here[:, None, None], k, zero).to(s["dtype"]), torch.where(here[:, None, None], v, zero).to(s["dtype"])


def _plain_key_states(s, tables):
    """Keys [n, heads, width * page, dim] of the pages in tables [n, width]."""
    pool, t = s["pool"], tables.long()
    k = _plain_keys(pool, pool["k_codes"][t], pool["k_factors"][t] if "k_factors" in pool else None, pool["k_scales"][t])
    return k.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _plain_value_states(s, tables):
    pool, t = s["pool"], tables.long()
    v = _plain_rows_of_values(pool, pool["v_codes"][t].transpose(3, 4), pool["v_factors"][t] if "v_factors" in pool else None, pool["v_scales"][t])
    return v.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _plain_weights(s, k, seen, bias):
    """Softmax weights [n, heads, most, group, keys] of the padded queries over keys k [n, heads, keys, dim]; seen [n, most, keys] says what a query sees."""
    q, start, most = s["q"], s["q_start"].long(), s["most"]
    n, H, K, D = k.shape
    G = q.shape[1] // H
    row = start[:-1, None] + torch.arange(most, device=q.device)
    x = q[row.clamp_max(q.shape[0] - 1)].float().view(n, most, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, most * G, D)
    a = (x @ k.transpose(2, 3)).mul_(s["scale"]).view(n, H, most, G, K)
    if bias is not None:
        a += bias[:, None, None, None]
    a.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = a.amax(-1, keepdim=True)
    a.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = a.sum(-1, keepdim=True)
    return a.div_(torch.where(total == 0, torch.ones_like(total), total))


def _plain_answers(s, a, v):
    q, start = s["q"], s["q_start"].long()
    n, H, most, G, K = a.shape
    out = (a.view(n, H, most * G, K) @ v).view(n, H, most, G, -1)
    token = torch.arange(q.shape[0], device=q.device)
    of = torch.searchsorted(start, token, right=True) - 1
    return out.permute(0, 2, 1, 3, 4)[of, token - start[of]].reshape(q.shape).to(s["dtype"])


def _plain_seen(s, keys):
    """Which keys of its sequence a query sees [n, most, keys]; queries that are padding see none."""
    new = s["q_start"].diff()[:, None, None]
    at = torch.arange(s["most"], device=new.device)[None, :, None]
    return (torch.arange(keys, device=new.device)[None, None, :] <= s["lengths"][:, None, None] - new + at) & (at < new)


def _plain_passages(s):
    ids = s["ids"]
    n, r = ids.shape
    have = ids >= 0
    at = ids.clamp_min(0)
    pages = s["tables"][at].view(n, -1)
    k = _plain_key_states(s, pages)
    keys = k.shape[2] // r
    length = torch.where(have, s["lengths"][at], torch.zeros((), dtype=torch.int32, device=at.device))
    seen = (torch.arange(keys, device=at.device) < length[:, :, None]).view(n, 1, r * keys).expand(n, s["most"], -1)
    bias = None if s["scores"] is None else (s["weight"] * s["scores"]).repeat_interleave(keys, 1)
    return _plain_answers(s, _plain_weights(s, k, seen, bias), _plain_value_states(s, pages))


def _plain_evict(s):
    pool, P, B, sums, n = s["pool"], s["page"], s["budget"], s["sums"], s["lengths"].long()[:, None, None]
    S, H, K = sums.shape
    j = torch.arange(K, device=sums.device)
    inf = torch.full((), math.inf, device=sums.device)
    order = torch.where(j >= n, -inf, torch.where(j >= n - s["recent"], inf, sums)).sort(dim=2, descending=True, stable=True).indices
    left = n.clamp_max(B)
    r = torch.arange(B, device=sums.device)
    best = torch.nn.functional.pad(order[:, :, :B], (0, max(0, B - K)), value=K)
    kept = torch.where(r < left, best, torch.full((), K, device=sums.device)).sort(dim=2).values
    there = (r < left).expand(S, H, B)
    at = torch.where(there, kept, torch.zeros((), dtype=kept.dtype, device=kept.device))
    kept_sums = torch.where(there, sums.gather(2, at), torch.zeros((), device=sums.device))
    room = s["to"].shape[1] * P
    q, h, i = there.nonzero(as_tuple=True)
    j = at[q, h, i]
    page, off, to_page, to_off = s["tables"][q, j // P].long(), j % P, s["to"][q, i // P].long(), i % P
    pool["v_codes"][to_page, h, :, to_off] = pool["v_codes"][page, h, :, off]
    for name in pool.keys() - {"v_codes"}:
        pool[name][to_page, h, to_off] = pool[name][page, h, off]
    return torch.where(there, kept, torch.full((), -1, device=kept.device)).int(), left.flatten().int(), torch.nn.functional.pad(kept_sums, (0, room - B))


def run(s):
    op = s["op"]
    if not own:
        if op == "write":
            _plain_write(s)
            return _plain_read(s), s["pool"]["k_scales"], s["pool"]["v_scales"]
        if op == "evict":
            return _plain_evict(s), _plain_read(s)
        if op == "passages":
            return _plain_passages(s)
        k = _plain_key_states(s, s["tables"])
        a = _plain_weights(s, k, _plain_seen(s, k.shape[2]), None)
        if op == "chunk":
            return _plain_answers(s, a, _plain_value_states(s, s["tables"]))
        return s["before"] + a.sum((2, 3))
    from paper_2410_18926_amd.states import States
    from paper_2410_18926_amd.states4 import States4
    st = (States if s["bits"] == 8 else States4)(**s["pool"])
    if op == "write":
        st.write(s["k"], s["v"], s["slots"])
        return st.read(s["slots"], s["dtype"]), s["pool"]["k_scales"], s["pool"]["v_scales"]
    if op == "evict":
        return st.evict(s["tables"], s["lengths"], s["sums"], s["budget"], s["to"], recent=s["recent"]), st.read(s["slots"], s["dtype"])
    q_start = None if s["one"] else s["q_start"]
    if op == "chunk":
        return st.attend_chunk(s["q"], s["tables"], s["lengths"], q_start=q_start, scale=s["scale"])
    if op == "weights":
        return st.attend_weights(s["q"], s["tables"], s["lengths"], q_start=q_start, scale=s["scale"], before=s["before"])
    return st.attend_passages(s["q"], s["ids"], s["tables"], s["lengths"], q_start=q_start, scores=s["scores"], score_weight=s["weight"], scale=s["scale"])


# ---------------------------------------------------------------------------------------------------------------
# The same in 64 bits, sequence by sequence and token by token from the definitions.

def _power_of_two(e):
    """2^e as a double, from its bits."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_decode(byte_codes, factors, steps, paired):
    """Values in 64 bits of rows [n, heads, dim / 2] of 4-bit codes; paired: components 16 apart share a byte, else neighbours."""
    n, H, half = byte_codes.shape
    table = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float64, device=byte_codes.device)
    out = torch.empty((n, H, 2 * half), dtype=torch.float64, device=byte_codes.device)
    for g in range(half // 16):
        b = byte_codes[:, :, 16 * g:16 * g + 16].long()
        f = factors[:, :, g].long()
        r = (8 + f % 8).double() * _power_of_two(f // 8 - 18) * steps.double()
        low, high = table[b % 16] * r[..., None], table[b // 16] * r[..., None]
        out[:, :, 32 * g:32 * g + 32] = torch.cat([low, high], 2) if paired else torch.stack([low, high], 3).reshape(n, H, 32)
    return out


def _exact_rows(pool, pages, offsets):
    """Keys and values [tokens, heads, dim] in 64 bits of the tokens at (pages, offsets)."""
    kc, vc = pool["k_codes"][pages, :, offsets], pool["v_codes"][pages, :, :, offsets]
    ks, vs = pool["k_scales"][pages, :, offsets], pool["v_scales"][pages, :, offsets]
    if "k_factors" not in pool:
        return kc.double() * ks.double().unsqueeze(-1), vc.double() * vs.double().unsqueeze(-1)
    return _exact_decode(kc, pool["k_factors"][pages, :, offsets], ks, False), _exact_decode(vc, pool["v_factors"][pages, :, offsets], vs, True)


def _exact_nearest(x):
    """What rows [tokens, heads, dim] are held as, and a / 6."""
    a = x.double()
    top = a.abs().amax(2, keepdim=True)
    out = torch.zeros_like(a)
    table = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    for g in range(a.shape[2] // 32):
        part = a[:, :, 32 * g:32 * g + 32]
        ratio = part.abs().amax(2, keepdim=True) / top
        # the smallest (8 + m) 2^e >= ratio, not below 2^-13
        m, e = torch.frexp(ratio.clamp_min(2.0 ** -13))
        r = torch.ceil(m * 16) * _power_of_two(e - 4)
        unit = top * r                              # 6 |x| and its multiples by the levels are exact
        best, far = torch.zeros_like(part), 6 * part.abs()
        for i in range(1, 8):                       # from the smallest level up: one is taken if it is nearer, or as near and its code is even
            new = (6 * part.abs() - table[i] * unit).abs()
            take = (new < far) | ((new == far) & (i % 2 == 0))
            best, far = torch.where(take, table[i], best), torch.where(take, new, far)
        out[:, :, 32 * g:32 * g + 32] = torch.copysign(best * unit / 6, part)
    return out, top[..., 0] / 6


def _exact_softmax(q, k, scale, seen=None, bias=None):
    """Weights [tokens, keys] of queries q [tokens, dim] over keys k [keys, dim]; rows that see nothing are 0"""
    z = scale * (q @ k.T)
    if bias is not None:
        z = z + bias
    if seen is not None:
        z = z.masked_fill(~seen, -math.inf)
    return torch.nan_to_num(torch.softmax(z, 1))


def _exact_evict(s, case):
    """By sorting, on the host, one sequence and head at a time."""
    pool, P, B, H = s["pool"], s["page"], s["budget"], case["heads"]
    sums, lens = s["sums"].double().cpu().numpy(), s["lengths"].tolist()
    S, room = len(lens), s["to"].shape[1] * P
    kept, out = np.full((S, H, B), -1, np.int32), np.zeros((S, H, room))
    back = [torch.zeros((S * B, H, case["dim"]), dtype=torch.float64, device="cuda") for _ in range(2)]
    for i, n in enumerate(lens):
        page, off = s["tables"][i].long()[torch.arange(n, device="cuda") // P], torch.arange(n, device="cuda") % P
        rows = _exact_rows(pool, page, off)
        for h in range(H):
            old = max(0, n - s["recent"])
            rest = max(0, min(n, B) - (n - old))
            best = np.lexsort((np.arange(old), -sums[i, h, :old]))[:rest]
            mine = np.sort(np.concatenate([best, np.arange(old, n)]))
            mine = mine[-B:] if len(mine) > B else mine
            kept[i, h, :len(mine)] = mine
            out[i, h, :len(mine)] = sums[i, h, mine]
            for b, x in zip(back, rows):
                b[i * B:i * B + len(mine), h] = x[torch.from_numpy(mine).cuda(), h]
    return (kept, np.minimum(lens, B).astype(np.int32), out), tuple(back)


def exact(case, seed):
    s = prepare(case, seed)
    pool, P = s["pool"], s["page"]
    if case["op"] == "write":
        page, at = s["slots"] // P, s["slots"] % P
        back, steps = [], []
        for name, x in (("k_scales", s["k"]), ("v_scales", s["v"])):
            near, step = _exact_nearest(x)
            whole = pool[name].double()
            whole[page, :, at] = step
            back.append(near)
            steps.append(whole)
        return tuple(back), steps[0], steps[1]
    if case["op"] == "evict":
        return _exact_evict(s, case)
    H, G, D = case["heads"], case["group"], case["dim"]
    new = s["q_start"].diff().tolist()
    lens = s["lengths"].tolist()
    # (a loop over sequences, heads and groups: cases of very many small steps are left out)
    if len(new) * H * G > 20_000:
        return None
    ids = s["ids"].tolist() if case["op"] == "passages" else None
    sums = s["before"].double() if case["op"] == "weights" else None
    out, first = [], 0
    for i, n in enumerate(new):
        q = s["q"][first:first + n].double().view(n, H, G, D)
        first += n
        bias = None
        if ids is None:
            t = torch.arange(lens[i], device="cuda")
            k, v = _exact_rows(pool, s["tables"][i].long()[t // P], t % P)
            seen = t[None, :] <= lens[i] - n + torch.arange(n, device="cuda")[:, None]
        else:
            seen, parts = None, []
            for j, p in enumerate(ids[i]):
                if p >= 0:
                    t = torch.arange(lens[p], device="cuda")
                    w = s["weight"] * s["scores"][i, j].double() if s["scores"] is not None else torch.zeros((), dtype=torch.float64, device="cuda")
                    parts.append((*_exact_rows(pool, s["tables"][p].long()[t // P], t % P), w.expand(lens[p])))
            k, v, bias = (torch.cat(x) for x in zip(*parts))
        answer = torch.zeros_like(q)
        for h in range(H):
            for g in range(G):
                w = _exact_softmax(q[:, h, g], k[:, h], s["scale"], seen, bias)
                if sums is None:
                    answer[:, h, g] = w @ v[:, h]
                else:
                    sums[i, h, :k.shape[0]] += w.sum(0)
        out.append(answer)
    return torch.cat(out).view(-1, H * G, D) if sums is None else sums
