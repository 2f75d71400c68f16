"""Timed cases of the state store and of the attention that reads it.

The store keeps the keys and values of tokens in pages, 8 bits a value with one step per token and head.  A case is one pass of one operator:

  op        "write"     a call that quantises new tokens' keys and values into their slots, and one that reads them back
            "read"      reading tokens back as values
            "chunk"     attention of every sequence's newest tokens over its own pages, causal
            "passages"  attention over the states of the passages that a search returned for each sequence
  type      "bf16", "f16" or "f32": what is written, read, asked and answered
  heads, group, dim, page   heads of the store, query heads for each of them, values a head, tokens a page

and the lengths, which follow from the case alone (content, page numbers and passages follow from the seed):

  write, read   tokens; run (tokens of one sequence that lie one after the other); sliced (keys and values are parts of one fused projection)
  chunk         sequences, new (most new tokens of a sequence), context (most tokens before them), ragged
  passages      sequences, new, k (passages of a sequence), length (most tokens of a passage), stock (passages in the store), ragged, weighted
"""
from __future__ import annotations

import math

import torch

own = False

TYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _tokens(name, op, tokens, heads, dim, page, run, type="bf16", sliced=False):
    return dict(name=name, op=op, tokens=tokens, heads=heads, dim=dim, page=page, run=run, type=type, sliced=sliced)


def _chunk(name, sequences, new, context, heads, group, dim, page, type="bf16", ragged=True):
    return dict(name=name, op="chunk", sequences=sequences, new=new, context=context, heads=heads, group=group, dim=dim, page=page, type=type, ragged=ragged)


def _passages(name, sequences, new, k, length, stock, heads, group, dim, page, type="bf16", ragged=True, weighted=False):
    return dict(name=name, op="passages", sequences=sequences, new=new, k=k, length=length, stock=stock, heads=heads, group=group, dim=dim, page=page, type=type,
                ragged=ragged, weighted=weighted)


def listed():
    return [
        # one decoding step of a small batch: a token each, latency counts
        _tokens("write-step", "write", 8, 8, 128, 64, 1),
        # passages taken into the store after an encoder has run over them, in bulk, from slices of its fused projection
        _tokens("write-passages", "write", 50_000, 8, 128, 64, 411, sliced=True),
        # a few states back in float, for a look at them or for another layer: odd sizes
        _tokens("read-few", "read", 333, 5, 96, 16, 37, type="f32"),
        # a long context read back for a kernel that wants 16-bit values
        _tokens("read-context", "read", 65_536, 8, 128, 64, 65_536),
        # the next token of one conversation: latency counts
        _chunk("token-one", 1, 1, 4000, 8, 4, 128, 64, ragged=False),
        # the next token of a serving batch, every conversation of another length
        _chunk("token-batch", 64, 1, 8192, 8, 4, 128, 64),
        # the next token after a very long document
        _chunk("token-long", 1, 1, 131_071, 8, 8, 128, 128, ragged=False),
        # prompts in pieces, mixed with short ones, one key head for each query head
        _chunk("chunk-mixed", 12, 500, 3000, 16, 1, 64, 16, type="f16"),
        # a large piece of a long prompt
        _chunk("chunk-long", 1, 4096, 28_672, 8, 4, 128, 64, ragged=False),
        # one token that reads the ten passages its query found
        _passages("found-token", 1, 1, 10, 256, 2000, 8, 4, 128, 64),
        # a serving batch of single tokens, passages shared between sequences, weighted by the search's scores
        _passages("found-batch", 48, 1, 10, 400, 1500, 8, 4, 128, 32, weighted=True),
        # questions read in full against their passages
        _passages("found-questions", 24, 96, 10, 512, 1200, 8, 4, 128, 64, weighted=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "chunk", "chunk", "passages", "passages"])
    base = dict(op=op, heads=rng.choice([1, 2, 3, 4, 8, 8, 16]), dim=rng.choice([64, 96, 128, 128]), page=rng.choice([16, 32, 64, 128]))
    if op in ("write", "read"):
        tokens = _log_int(rng, 1, 60_000)
        c = dict(base, tokens=tokens, run=min(tokens, _log_int(rng, 1, 5000)), type=rng.choice(["bf16", "f16", "f32"]), sliced=rng.random() < 0.4)
        while work(c)["bytes"] > 3.5e8:
            c["tokens"] = c["tokens"] // 2 + 1
            c["run"] = min(c["run"], c["tokens"])
        return c
    base.update(group=rng.choice([1, 2, 4, 4, 6, 8]), type=rng.choice(["bf16", "bf16", "f16"]), ragged=rng.random() < 0.8)
    new = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 64, 2048)])
    if op == "chunk":
        c = dict(base, sequences=_log_int(rng, 1, 64), new=new, context=_log_int(rng, 1, 60_000))
        shrink = ("sequences", "context")
    else:
        stock = _log_int(rng, 20, 1500)
        c = dict(base, sequences=_log_int(rng, 1, 64), new=min(new, 300), k=min(stock, rng.choice([1, 3, 5, 10, 10, 20])), length=_log_int(rng, 4, 700), stock=stock, weighted=rng.random() < 0.5)
        shrink = ("sequences", "stock")
    # no case costs more than the largest listed ones: products, states held, and the matrix of scores that the plain form makes
    while True:
        keys = c["context"] + c["new"] + c["page"] if op == "chunk" else c["k"] * (c["length"] + c["page"])
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
    new = _spread(case["sequences"], case["new"], case["ragged"], 0.3)
    if case["op"] == "chunk":
        return new, _spread(case["sequences"], case["context"], case["ragged"])
    return new, None


def _stock(case):
    return _spread(case["stock"], case["length"], case["ragged"])


def work(case):
    """Bytes and operations of one pass.  What a passages case reads depends on which passages are named: every sequence's are counted, but no more
    than the whole stock once."""
    H, D, e = case["heads"], case["dim"], 4 if case["type"] == "f32" else 2
    if case["op"] in ("write", "read"):
        T = case["tokens"]
        once = 2 * T * H * D * e + 2 * T * H * (D + 4) + 8 * T
        return {"bytes": 2 * once if case["op"] == "write" else once, "flops": 0}
    new, before = _lengths(case)
    G, N = case["group"], sum(new)
    asked = 2 * N * H * G * D * e
    if case["op"] == "chunk":
        pairs = sum(n * b + n * (n + 1) // 2 for n, b in zip(new, before))
        keys = sum(n + b for n, b in zip(new, before))
    else:
        lens = _stock(case)
        mean = sum(lens) / len(lens)
        pairs = N * case["k"] * mean
        keys = mean * min(case["stock"], case["sequences"] * case["k"])
    return {"bytes": asked + 2 * keys * H * (D + 4), "flops": 4 * H * G * D * pairs}


# ---------------------------------------------------------------------------------------------------------------
# Inputs.

def _quantise(x):
    """Codes and steps of rows along the last axis, as the store holds them."""
    top = x.abs().amax(-1)
    return torch.round(x * 127 / top.clamp_min(2.0 ** -100)[..., None]).to(torch.int8), top / 127


def _states(shape, g, spread):
    """Rows of encoder or decoder states: components of different sizes with a mean of their own, rows of different lengths."""
    d = shape[-1]
    size = torch.exp(spread * torch.randn(d, generator=g, device="cuda"))
    mean = 0.5 * size * torch.randn(d, generator=g, device="cuda")
    x = torch.randn(shape, generator=g, device="cuda").mul_(size).add_(mean)
    return x.mul_(torch.exp(0.2 * torch.randn(shape[:-1], generator=g, device="cuda"))[..., None])


def _pool(pages, case, g):
    """A store of `pages` pages in use: every slot holds the states of some token."""
    H, P, D = case["heads"], case["page"], case["dim"]
    kc, ks = _quantise(_states((pages, H, P, D), g, 0.6))
    vc, vs = _quantise(_states((pages, H, P, D), g, 0.2))
    return dict(k_codes=kc, v_codes=vc.transpose(2, 3).contiguous(), k_scales=ks, v_scales=vs)


def _tables(lengths, pages, P, g):
    """Page numbers of each sequence, from pages handed out in no order, as a server's allocator leaves them."""
    need = [-(-n // P) for n in lengths]
    width = max(1, max(need))
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    rows = torch.arange(width, device="cuda")[None, :]
    count = torch.tensor(need, device="cuda")[:, None]
    first = torch.tensor([0] + need, device="cuda").cumsum(0)[:-1, None]
    return torch.where(rows < count, order[(first + rows).clamp_max(pages - 1)], torch.zeros((), dtype=torch.int32, device="cuda")).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H, P, D, dtype = case["heads"], case["page"], case["dim"], TYPE[case["type"]]
    s = dict(op=case["op"], dtype=dtype, page=P)
    if case["op"] in ("write", "read"):
        T, run = case["tokens"], case["run"]
        count = -(-T // run)
        # each sequence writes `run` tokens after some that it has already
        lengths = [(i * 7919 + 3) % P + run for i in range(count)]
        pages = sum(-(-n // P) for n in lengths) + 3
        s["pool"] = _pool(pages, case, g)
        table = _tables(lengths, pages, P, g).long()
        t = torch.arange(T, device="cuda")
        at = t % run + torch.tensor(lengths, device="cuda")[t // run] - run
        s["slots"] = table[t // run, at // P] * P + at % P
        if case["op"] == "write":
            if case["sliced"]:
                fused = _states((T, 3 * H, D), g, 0.4).to(dtype)
                s["k"], s["v"] = fused[:, H:2 * H], fused[:, 2 * H:]
            else:
                s["k"], s["v"] = _states((T, H, D), g, 0.6).to(dtype), _states((T, H, D), g, 0.2).to(dtype)
        return s
    new, before = _lengths(case)
    s["q_start"] = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    s["most"] = max(new)
    s["one"] = case["new"] == 1
    s["scale"] = D ** -0.5
    lengths = [n + b for n, b in zip(new, before)] if before else _stock(case)
    pages = sum(-(-n // P) for n in lengths) + 2
    s["pool"] = _pool(pages, case, g)
    s["tables"] = _tables(lengths, pages, P, g)
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    # a spread of about two between the logits of a row
    s["q"] = (1.3 * torch.randn((sum(new), H * case["group"], D), generator=g, device="cuda")).to(dtype)
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

def _plain_write(s):
    pool, slots, P = s["pool"], s["slots"], s["page"]
    page, at = slots // P, slots % P
    k, ks = _quantise(s["k"].float())
    v, vs = _quantise(s["v"].float())
    pool["k_codes"][page, :, at] = k
    pool["v_codes"][page, :, :, at] = v
    pool["k_scales"][page, :, at] = ks
    pool["v_scales"][page, :, at] = vs


def _plain_read(s):
    pool, slots, P = s["pool"], s["slots"], s["page"]
    page, at = slots // P, slots % P
    k = pool["k_codes"][page, :, at].float() * pool["k_scales"][page, :, at][..., None]
    v = pool["v_codes"][page, :, :, at].float() * pool["v_scales"][page, :, at][..., None]
    return k.to(s["dtype"]), v.to(s["dtype"])


def _plain_states(s, tables):
    """Keys and values [n, heads, width * page, dim] of the pages in tables [n, width]."""
    pool = s["pool"]
    t = tables.long()
    n, w = t.shape
    H, P, D = pool["k_codes"].shape[1:]
    k = pool["k_codes"][t].float() * pool["k_scales"][t][..., None]
    v = pool["v_codes"][t].float() * pool["v_scales"][t][:, :, :, None, :]
    return k.permute(0, 2, 1, 3, 4).reshape(n, H, w * P, D), v.permute(0, 2, 1, 4, 3).reshape(n, H, w * P, D)


def _plain_attention(s, k, v, seen, bias):
    """Softmax attention of the padded queries over keys k [n, heads, keys, dim]; seen [n, most, keys] says what a query sees."""
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
    out = (a.view(n, H, most * G, K) @ v).view(n, H, most, G, D) / torch.where(total == 0, torch.ones_like(total), total)
    token = torch.arange(q.shape[0], device=q.device)
    of = torch.searchsorted(start, token, right=True) - 1
    return out.permute(0, 2, 1, 3, 4)[of, token - start[of]].reshape(q.shape).to(s["dtype"])


def _plain_chunk(s):
    k, v = _plain_states(s, s["tables"])
    new = s["q_start"].diff()[:, None, None]
    at = torch.arange(s["most"], device=new.device)[None, :, None]
    key = torch.arange(k.shape[2], device=new.device)[None, None, :]
    return _plain_attention(s, k, v, key <= s["lengths"][:, None, None] - new + at, None)


def _plain_passages(s):
    ids = s["ids"]
    n, r = ids.shape
    have = ids >= 0
    at = ids.clamp_min(0)
    k, v = _plain_states(s, s["tables"][at].view(n, -1))
    keys = k.shape[2] // r
    length = torch.where(have, s["lengths"][at], torch.zeros((), dtype=torch.int32, device=at.device))
    seen = (torch.arange(keys, device=at.device) < length[:, :, None]).view(n, 1, r * keys).expand(n, s["most"], -1)
    bias = None if s["scores"] is None else (s["weight"] * s["scores"]).repeat_interleave(keys, 1)
    return _plain_attention(s, k, v, seen, bias)


def run(s):
    if not own:
        if s["op"] == "write":
            _plain_write(s)
            return _plain_read(s), s["pool"]["k_scales"], s["pool"]["v_scales"]
        if s["op"] == "read":
            return _plain_read(s)
        return _plain_chunk(s) if s["op"] == "chunk" else _plain_passages(s)
    from paper_2410_18926_amd.states import States
    st = States(**s["pool"])
    if s["op"] == "write":
        st.write(s["k"], s["v"], s["slots"])
        return st.read(s["slots"], s["dtype"]), s["pool"]["k_scales"], s["pool"]["v_scales"]
    if s["op"] == "read":
        return st.read(s["slots"], s["dtype"])
    q_start = None if s["one"] else s["q_start"]
    if s["op"] == "chunk":
        return st.attend_chunk(s["q"], s["tables"], s["lengths"], q_start=q_start, scale=s["scale"])
    return st.attend_passages(s["q"], s["ids"], s["tables"], s["lengths"], q_start=q_start, scores=s["scores"], score_weight=s["weight"], scale=s["scale"])


# ---------------------------------------------------------------------------------------------------------------
# The same in 64 bits, sequence by sequence and token by token from the definitions.

def _exact_rows(pool, pages, offsets):
    """Keys and values [tokens, heads, dim] in 64 bits of the tokens at (pages, offsets)."""
    k = pool["k_codes"][pages, :, offsets].double() * pool["k_scales"][pages, :, offsets].double().unsqueeze(-1)
    v = pool["v_codes"][pages, :, :, offsets].double() * pool["v_scales"][pages, :, offsets].double().unsqueeze(-1)
    return k, v


def _exact_softmax(q, k, v, scale, seen=None, bias=None):
    """q [tokens, heads of the store, group, dim], k and v [keys, heads, dim]"""
    out = torch.zeros_like(q)
    if k.shape[0] == 0:
        return out
    for h in range(k.shape[1]):
        for g in range(q.shape[2]):
            z = scale * (q[:, h, g] @ k[:, h].T)
            if bias is not None:
                z = z + bias
            if seen is not None:
                z = z.masked_fill(~seen, -math.inf)
            out[:, h, g] = torch.softmax(z, 1) @ v[:, h]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    pool, P = s["pool"], s["page"]
    if case["op"] == "write":
        page, at = s["slots"] // P, s["slots"] % P
        back, steps = [], []
        for name, x in (("k_scales", s["k"].double()), ("v_scales", s["v"].double())):
            top = x.abs().amax(2, keepdim=True)
            back.append(torch.round(127 * x / top) * (top / 127))
            whole = pool[name].double()
            whole[page, :, at] = top[..., 0] / 127
            steps.append(whole)
        return tuple(back), steps[0], steps[1]
    if case["op"] == "read":
        return _exact_rows(pool, s["slots"] // P, s["slots"] % P)
    H, G, D = case["heads"], case["group"], case["dim"]
    new, _ = _lengths(case)
    lens = s["lengths"].tolist()
    # (a loop over sequences, heads and groups: cases of very many small steps are left out)
    if len(new) * H * G > 20_000:
        return None
    ids = s["ids"].tolist() if case["op"] == "passages" else None
    out, first = [], 0
    for i, n in enumerate(new):
        q = s["q"][first:first + n].double().view(n, H, G, D)
        first += n
        if ids is None:
            t = torch.arange(lens[i], device="cuda")
            k, v = _exact_rows(pool, s["tables"][i].long()[t // P], t % P)
            seen = t[None, :] <= lens[i] - n + torch.arange(n, device="cuda")[:, None]
            out.append(_exact_softmax(q, k, v, s["scale"], seen))
        else:
            named = [(j, p) for j, p in enumerate(ids[i]) if p >= 0]
            parts = []
            for j, p in named:
                t = torch.arange(lens[p], device="cuda")
                w = s["weight"] * s["scores"][i, j].double() if s["scores"] is not None else torch.zeros((), dtype=torch.float64, device="cuda")
                parts.append((*_exact_rows(pool, s["tables"][p].long()[t // P], t % P), w.expand(lens[p])))
            k, v, bias = (torch.cat(x) for x in zip(*parts))
            out.append(_exact_softmax(q, k, v, s["scale"], None, bias))
    return torch.cat(out).view(-1, H * G, D)
