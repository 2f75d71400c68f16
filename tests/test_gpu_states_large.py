"""The attention where the largest blocks are taken (8 wavefronts) and where long tables are cut: every answer against the definition in 64 bits on the GPU.

Tolerance, with A = sum_j p_j |v_j| per component (p: the exact weights), n keys of dimension D:
  - the answer's rounding: u |out|, u = 2^-8 (bfloat16), 2^-11 (binary16; 2^-25 at least, half the distance of its numbers below 2^-14);
  - the weights' rounding: 2^-11 A, and 2^-34 of the largest for each key: 2^-34 sum_j |V_j| / sum_j (w_j / sv_j), V the codes, sv the steps, w_j = 2^(y_j) / max_j 2^(y_j);
  - the logits in float: (D + 8) 2^-24 scale max_j <|q|, |k_j|>, and 2^-21 (max |y| + max |bias| + 8) for what follows in units of log2; a relative error e of the weights moves an
    answer by 2 e A at most;
  - sums in float: the numerator grows by a matrix instruction for 16 keys, taken to round twice, the divisor by a term for 64 keys: (2 n / 16 + n / 64 + 64) 2^-24 A."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def S():
    from paper_2410_18926_amd import binding, states
    assert binding.LIB_PATH.exists(), "build the HIP library first (python -m paper_2410_18926_amd.build)"
    assert torch.cuda.is_available(), "these tests need the GPU"
    return states


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


def store_of(S, g, lengths, heads, page, dim, values=None):
    """(store, tables): tokens of several tables on pages in no order, entries beyond a length of no page.  values: a function of the (table, token numbers) giving factors."""
    need = [-(-n // page) for n in lengths]
    st = S.States.empty(sum(need) + 2, heads, page, dim)
    order = torch.randperm(st.pages, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((len(lengths), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(lengths):
        tables[i, :need[i]] = order[at:at + need[i]]
        at += need[i]
        for t0 in range(0, n, 1 << 16):
            t = torch.arange(t0, min(n, t0 + (1 << 16)), device="cuda")
            k, v = randn(g, len(t), heads, dim) + 0.2, (randn(g, len(t), heads, dim) - 0.1) * torch.exp(0.5 * randn(g, len(t), heads, 1))
            if values is not None:
                v = v * values(i, t)[:, None, None]
            st.write(k, v, tables[i, t // page].long() * page + t % page)
    return st, tables


def rows_of(st, table, length, head):
    t = torch.arange(length, device="cuda")
    page, off = table.long()[t // st.page_size], t % st.page_size
    return [x.double() for x in (st.k_codes[page, head, off], st.v_codes[page, head, :, off], st.k_scales[page, head, off], st.v_scales[page, head, off])]


def check(st, q, got, parts_of, start, scale):
    """parts_of(s, head): (key codes, value codes, their steps, bias [n], seen [tokens, n] or None) of sequence s, or None where there are no keys."""
    G, D = q.shape[1] // st.heads, st.dim
    assert not torch.isnan(got).any()
    for s in range(len(start) - 1):
        lo, hi = start[s], start[s + 1]
        if lo == hi:
            continue
        for h in range(st.heads):
            mine = got[lo:hi, h * G:(h + 1) * G].double()
            parts = parts_of(s, h)
            if parts is None:
                assert (mine == 0).all()
                continue
            kc, vc, ks, vs, bias, seen = parts
            n = kc.shape[0]
            k, v = kc * ks[:, None], vc * vs[:, None]
            x = q[lo:hi, h * G:(h + 1) * G].double().reshape(-1, D)
            z = scale * (x @ k.T) + bias
            if seen is not None:
                z = z.masked_fill(~seen.repeat_interleave(G, 0), -math.inf)
            some = ~torch.isneginf(z).all(1)
            p = torch.softmax(z, 1)
            want, A = p @ v, p @ v.abs()
            y = z / math.log(2) + torch.log2(torch.where(vs == 0, torch.full_like(vs, 2.0 ** -84), vs))
            w = torch.exp2(y - y.amax(1, keepdim=True))
            e = (D + 8) * 2.0 ** -24 * abs(scale) * (x.abs() @ k.abs().T).amax(1, keepdim=True)
            e = e + 2.0 ** -21 * (torch.where(torch.isneginf(y), torch.zeros_like(y), y).abs().amax(1, keepdim=True) + bias.abs().max() + 8)
            u, least = (2.0 ** -8, 0.0) if q.dtype == BF16 else (2.0 ** -11, 2.0 ** -25)
            floor = 2.0 ** -34 * ((w > 0).double() @ vc.abs()) / (w / torch.where(vs == 0, torch.full_like(vs, 2.0 ** -84), vs)).sum(1, keepdim=True)
            tol = (u * want.abs()).clamp_min(least) + (2.0 ** -11 + 2 * e + (2 * n / 16 + n / 64 + 64) * 2.0 ** -24) * A + floor
            off = (mine.reshape(-1, D) - want).abs()
            bad = (off > tol) & some[:, None]
            assert not bad.any(), f"sequence {s}, head {h}: off by {float(off[bad].max()):.3g} where {float(tol[bad].min()):.3g} is allowed, {int(bad.sum())} of {bad.numel()}"
            assert (mine.reshape(-1, D)[~some] == 0).all()


def check_chunk(st, q, got, tables, lengths, start, scale):
    def parts(s, h):
        n, T = lengths[s], start[s + 1] - start[s]
        if n == 0:
            return None
        seen = torch.arange(n, device="cuda")[None, :] <= n - T + torch.arange(T, device="cuda")[:, None]
        return (*rows_of(st, tables[s], n, h), torch.zeros(n, dtype=torch.float64, device="cuda"), seen)
    check(st, q, got, parts, start, scale)


def check_passages(st, q, got, ids, scores, weight, tables, lengths, start, scale):
    def parts(s, h):
        found = [(r, i) for r, i in enumerate(ids[s]) if 0 <= i < len(lengths) and lengths[i] > 0]
        if not found:
            return None
        rows = [rows_of(st, tables[i], lengths[i], h) for _, i in found]
        bias = [torch.full((lengths[i],), 0.0 if scores is None else weight * float(scores[s][r]), dtype=torch.float64, device="cuda") for r, i in found]
        return (*(torch.cat([x[j] for x in rows]) for j in range(4)), torch.cat(bias), None)
    check(st, q, got, parts, start, scale)


def starts(new):
    return [0] + [int(x) for x in np.cumsum(new)]


# ---- blocks of 256 rows: dimensions 96 and 128, 1024 rows a sequence and head or more on average, 512 blocks or more ----

UNEVEN = [0, 700, 33, 1500, 0, 900, 1, 411]


@pytest.mark.parametrize("heads,group,dim,page,dtype,new", [
    (8, 8, 128, 16, F16, UNEVEN), (8, 8, 128, 64, F16, UNEVEN), (8, 8, 96, 128, BF16, UNEVEN), (16, 8, 96, 32, F16, [600, 450]), (16, 8, 128, 32, BF16, [520, 520])])
def test_large_blocks_over_uneven_chunks(S, heads, group, dim, page, dtype, new):
    g = gen(31 + dim + page)
    lengths = [n + 100 + 37 * i if i != 3 else n - 200 for i, n in enumerate(new)]           # (one with more queries than tokens)
    st, tables = store_of(S, g, lengths, heads, page, dim)
    start = starts(new)
    q = (1.5 * randn(g, start[-1], heads * group, dim)).to(dtype)
    got = st.attend_chunk(q, tables, dev(lengths), q_start=dev(start))
    check_chunk(st, q, got, tables, lengths, start, dim ** -0.5)
    assert torch.equal(got, st.attend_chunk(q, tables, dev(lengths), q_start=dev(start))), "two runs differ"


@pytest.mark.parametrize("heads,group,dim,page,dtype,new", [
    (8, 8, 128, 64, BF16, [150] * 20), (8, 8, 128, 16, F16, [150] * 20), (8, 8, 96, 64, F16, [0, 300, 1, 170, 260, 250, 140, 0, 320, 350]), (8, 8, 96, 32, BF16, [140] * 24)])
def test_large_blocks_over_passages(S, heads, group, dim, page, dtype, new):
    g, rng = gen(41 + dim + page), np.random.default_rng(dim + page)
    lengths = [int(n) for n in rng.integers(1, 260, 30)]
    lengths[4] = 0
    st, tables = store_of(S, g, lengths, heads, page, dim)
    ids = rng.integers(0, len(lengths), (len(new), 4))
    ids[1, 2], ids[2, 0], ids[3, 1], ids[5] = -1, len(lengths), 4, -1
    scores = rng.normal(size=ids.shape).astype(np.float32)
    start = starts(new)
    q = (1.5 * randn(g, start[-1], heads * group, dim)).to(dtype)
    got = st.attend_passages(q, dev(ids, torch.int64), tables, dev(lengths), q_start=None if len(set(new)) == 1 else dev(start), scores=dev(scores, torch.float32), score_weight=-1.7)
    check_passages(st, q, got, ids, scores, -1.7, tables, lengths, start, dim ** -0.5)


@pytest.mark.parametrize("dim,page,dtype", [(128, 64, BF16), (128, 16, F16), (96, 64, F16), (96, 32, BF16)])
@pytest.mark.parametrize("what", ["tiny values from the middle on", "large values from the middle on", "queries far apart", "both", "keys without values"])
def test_large_blocks_step_by_step(S, dim, page, dtype, what):
    """What the pipelined loop hands over to the loop that goes step by step, in the middle or from the start."""
    g = gen(51 + dim + page)
    heads, group, new, lengths = 16, 8, [400, 600], [700, 900]
    factor = {"tiny values from the middle on": 2.0 ** -60, "large values from the middle on": 2.0 ** 20, "both": 2.0 ** -60, "keys without values": 0.0}.get(what, 1.0)
    if dtype == F16 and factor > 1:
        factor = 2.0 ** 6                  # (answers that binary16 holds; steps up to 2^3)
    every = 7 if what == "keys without values" else 1
    st, tables = store_of(S, g, lengths, heads, page, dim, lambda i, t: torch.where((t >= 330 + 64 * i) & (t % every == 0), factor, 1.0))
    start = starts(new)
    q = 1.5 * randn(g, start[-1], heads * group, dim)
    if what in ("queries far apart", "both"):
        q[::5] *= 2.0 ** -14
        q[3::64] *= 2.0 ** -9
    q = q.to(dtype)
    got = st.attend_chunk(q, tables, dev(lengths), q_start=dev(start))
    check_chunk(st, q, got, tables, lengths, start, dim ** -0.5)


# ---- long tables are cut ----

def test_one_very_long_sequence_among_short_ones(S):
    """A decoding step of 64 conversations, one of them of 131 000 tokens: its keys are cut where 512 blocks would be there without."""
    g = gen(61)
    heads, group, dim, page = 8, 4, 128, 128
    lengths = [900 + 3 * i for i in range(64)]
    lengths[40], lengths[7], lengths[8] = 131_000, 1, 0
    st, tables = store_of(S, g, lengths, heads, page, dim)
    q = (1.5 * randn(g, 64, heads * group, dim)).to(BF16)
    got = st.attend_chunk(q, tables, dev(lengths))
    check_chunk(st, q, got, tables, lengths, list(range(65)), dim ** -0.5)


@pytest.mark.parametrize("heads,group,dim,page,dtype,new,lengths", [
    (2, 8, 64, 16, F16, [1], [200_001]),
    (4, 2, 96, 64, BF16, [5, 0, 9, 2], [70_000, 40_000, 333, 2]),
    (8, 4, 128, 64, BF16, [200, 150, 180, 190], [100_000, 500, 33_000, 100]),           # shared tiles
    (8, 4, 64, 32, F16, [100, 100], [66_000, 65_536]),
    (1, 4, 128, 256, F16, [500], [150_000]),
])
def test_long_contexts(S, heads, group, dim, page, dtype, new, lengths):
    g = gen(sum(lengths) % 1000)
    st, tables = store_of(S, g, lengths, heads, page, dim)
    start = starts(new)
    q = (1.5 * randn(g, start[-1], heads * group, dim)).to(dtype)
    got = st.attend_chunk(q, tables, dev(lengths), q_start=dev(start))
    check_chunk(st, q, got, tables, lengths, start, dim ** -0.5)


@pytest.mark.parametrize("new", [1, 60])
def test_a_long_document_among_passages(S, new):
    g = gen(71)
    heads, group, dim, page = 4, 4, 128, 64
    lengths = [80_000, 300, 64, 1, 0, 170]
    st, tables = store_of(S, g, lengths, heads, page, dim)
    ids = np.array([[1, 0, 5], [3, 2, -1], [4, 0, 0]])
    scores = np.array([[0.3, 0.1, 0.2], [0.0, 0.4, 0.0], [0.5, 1.0, -1.0]], np.float32)
    q = (1.5 * randn(g, 3 * new, heads * group, dim)).to(BF16)
    got = st.attend_passages(q, dev(ids, torch.int64), tables, dev(lengths), scores=dev(scores, torch.float32), score_weight=-2.0)
    check_passages(st, q, got, ids, scores, -2.0, tables, lengths, starts([new] * 3), dim ** -0.5)


# ---- prompts beside single tokens ----

@pytest.mark.parametrize("ones,chunks", [(200, [512]), (63, [1024]), (100, [1, 700, 0, 300]), (300, [40])])
def test_prompts_beside_single_tokens(S, ones, chunks):
    """A serving step in which most sequences have one new token and a few a piece of a prompt, whichever kernel the whole call takes."""
    g, rng = gen(ones), np.random.default_rng(ones)
    heads, group, dim, page = 2, 4, 128, 64
    new = [1] * ones
    for i, c in enumerate(chunks):
        new.insert((37 * i + 11) % len(new), c)
    lengths = [n + int(rng.integers(0, 700)) for n in new]
    st, tables = store_of(S, g, lengths, heads, page, dim)
    start = starts(new)
    q = (1.5 * randn(g, start[-1], heads * group, dim)).to(BF16)
    got = st.attend_chunk(q, tables, dev(lengths), q_start=dev(start))
    check_chunk(st, q, got, tables, lengths, start, dim ** -0.5)
