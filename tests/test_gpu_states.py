"""The state store and its attention on the GPU against their definitions in 64 bits (states_reference.py, where the tolerances are derived)."""
import numpy as np
import pytest
import torch

import states_reference as R

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


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


def filled(S, pages, heads, page, dim, seed=1, spread=1.0):
    """A store whose every slot holds the states of some token: components with a mean, rows of different lengths."""
    g = gen(seed)
    st = S.States.empty(pages, heads, page, dim)
    n = pages * page
    k = (randn(g, n, heads, dim) + 0.3) * torch.exp(0.4 * spread * randn(g, n, heads, 1))
    v = (randn(g, n, heads, dim) - 0.2) * torch.exp(0.8 * spread * randn(g, n, heads, 1))
    st.write(k, v, torch.arange(n, device="cuda"))
    return st


def same(a, b):
    a, b = a.cpu().numpy(), b.cpu().numpy() if isinstance(b, torch.Tensor) else b
    return np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


# ---- writing and reading ----

def rows_in_layout(x, layout):
    """The same values [tokens, heads, dim] in another place: as given, a slice of a fused projection, heads first, one element off 16 bytes."""
    n, h, d = x.shape
    if layout == "plain":
        return x
    if layout == "slice":
        wide = torch.full((n, 3 * h, d), 7.0, dtype=x.dtype, device=x.device)
        wide[:, h:2 * h] = x
        return wide[:, h:2 * h]
    if layout == "heads first":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    assert layout == "odd"
    flat = torch.empty(n * h * (d + 1) + 1, dtype=x.dtype, device=x.device)
    view = flat[1:].view(n, h, d + 1)[:, :, :d]
    view.copy_(x)
    return view


@pytest.mark.parametrize("dim,page,heads,tokens", [(128, 64, 3, 200), (96, 16, 2, 77), (64, 32, 1, 1), (32, 128, 5, 130), (128, 256, 2, 300), (128, 16, 8, 16)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("order", ["shuffled", "run", "runs from odd places", "backwards"])
def test_write_and_read_back(S, dim, page, heads, tokens, dtype, order):
    """Codes and steps are those of the definition bit for bit, in the slots named and nowhere else; what is read is step * code, rounded once."""
    g = gen(dim * 7 + page + tokens)
    pages = -(-tokens // page) + 3
    st = filled(S, pages, heads, page, dim, seed=5)
    before = R.store_arrays(st)
    k, v = randn(g, tokens, heads, dim).to(dtype), (randn(g, tokens, heads, dim) * 3 + 1).to(dtype)
    if tokens > 8:
        k[3, 0] = 0
        v[4, heads - 1] = 0
        k[5, 0, 7] = float("nan")
        v[6, 0, dim - 1] = float("inf")
        v[7, 0] *= 1e-4
        if dtype != F16:
            k[8, 0] = 1e-36 * torch.arange(dim, device="cuda")
            k[2, 0] *= 1e37
    n_slots = pages * page
    if order == "shuffled":
        slots = torch.randperm(n_slots, generator=g, device="cuda")[:tokens]
        slots[tokens // 2] = -1
        slots[tokens // 3] = n_slots
        slots[tokens // 4] = -2 ** 40
    elif order == "run":
        slots = page + torch.arange(tokens, device="cuda")
    elif order == "backwards":
        slots = torch.arange(tokens - 1, -1, -1, device="cuda")
    else:                          # several runs, each from another place of a page, the second half of the tokens before the first
        t = torch.arange(tokens, device="cuda")
        cut = tokens // 2
        slots = torch.where(t < cut, t + (n_slots - cut), t - cut + 1 + (page // 2 - 1))
    layouts = ["plain", "slice", "heads first", "odd"]
    st.write(rows_in_layout(k, layouts[tokens % 4]), rows_in_layout(v, layouts[(tokens + heads) % 4]), slots)
    after = R.store_arrays(st)
    s = slots.cpu().numpy()
    ok = (s >= 0) & (s < n_slots)
    p, o = s[ok] // page, s[ok] % page
    want = {n: a.copy() for n, a in before.items()}
    kc, ks = R.quantise(k.float().cpu().numpy())
    vc, vs = R.quantise(v.float().cpu().numpy())
    want["k_codes"][p, :, o], want["k_scales"][p, :, o] = kc[ok], ks[ok]
    want["v_codes"][p, :, :, o], want["v_scales"][p, :, o] = vc[ok], vs[ok]
    for name in want:
        assert np.array_equal(after[name], want[name], equal_nan=name.endswith("scales")), name
    for out_type in (F32, F16, BF16):
        out = None
        if out_type == dtype:      # into another layout as well
            out = tuple(rows_in_layout(torch.full((tokens, heads, dim), 5.0, dtype=dtype, device="cuda"), layouts[(tokens + i + 1) % 4]) for i in range(2))
        rk, rv = st.read(slots, out_type, out=out)
        for got, c, step in ((rk, kc, ks), (rv, vc, vs)):
            x = torch.from_numpy(np.where(ok[:, None, None], c.astype(np.float32) * step[..., None], np.float32(0))).to(out_type)
            assert np.array_equal(got.float().cpu().numpy(), x.float().numpy(), equal_nan=True), (out_type, order)


def test_read_leaves_the_gaps_between_rows_alone(S):
    st = filled(S, 4, 2, 16, 64)
    wide = torch.full((40, 6, 64), 9.0, dtype=F16, device="cuda")
    st.read(torch.arange(40, device="cuda"), out=(wide[:, :2], wide[:, 3:5]))
    assert (wide[:, 2] == 9).all() and (wide[:, 5] == 9).all() and not (wide[:, :2] == 9).all()


def test_no_tokens(S):
    st = filled(S, 2, 2, 16, 32)
    e = torch.empty((0, 2, 32), dtype=BF16, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    st.write(e, e, none)
    k, v = st.read(none)
    assert k.shape == v.shape == (0, 2, 32)
    out = st.attend_chunk(torch.empty((0, 4, 32), dtype=BF16, device="cuda"), torch.zeros((3, 1), dtype=torch.int32, device="cuda"),
                          torch.ones(3, dtype=torch.int32, device="cuda"), q_start=torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, 4, 32)


# ---- attention ----

def make_tables(g, lengths, pages, page, spare=0, junk=True):
    """Distinct random pages for each; entries beyond a length hold numbers of no page."""
    need = [-(-n // page) for n in lengths]
    width = max(need + [1]) + spare
    order = torch.randperm(pages, generator=g, device="cuda").cpu().numpy()
    assert sum(need) <= pages
    t = np.full((len(lengths), width), 2 ** 31 - 1 if junk else 0, np.int32)
    at = 0
    for i, n in enumerate(need):
        t[i, :n] = order[at:at + n]
        at += n
    return t


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


CHUNKS = [
    # (new tokens, lengths), heads, group, dim, page, type
    ([1], [1], 1, 1, 32, 16, BF16),
    ([1], [2], 2, 4, 128, 64, F16),
    ([1, 1, 1], [63, 64, 65], 2, 3, 64, 16, BF16),
    ([1, 1, 1, 1], [300, 1, 0, 257], 2, 8, 128, 32, BF16),
    ([1], [5000], 2, 4, 128, 128, BF16),
    ([1, 1], [2049, 777], 3, 6, 96, 256, F16),
    ([5, 0, 40, 1], [5, 9, 130, 64], 2, 2, 64, 16, F16),
    ([33, 65], [33, 600], 1, 1, 128, 64, BF16),
    ([7, 3, 12], [4, 0, 12], 2, 4, 32, 16, BF16),            # more queries than tokens: rows without a key
    ([64], [64], 2, 5, 96, 32, F16),
    ([300], [1111], 1, 2, 128, 16, BF16),
    ([130, 1, 257], [130, 900, 300], 2, 1, 64, 64, F16),
    ([100, 100], [100, 350], 1, 7, 128, 32, F16),
]


@pytest.mark.parametrize("new,lengths,heads,group,dim,page,dtype", CHUNKS)
def test_chunk(S, new, lengths, heads, group, dim, page, dtype):
    g = gen(sum(lengths) + dim)
    pages = sum(-(-n // page) for n in lengths) + 3
    st = filled(S, pages, heads, page, dim, seed=sum(new))
    tables = make_tables(g, lengths, pages, page, spare=sum(new) % 3)
    q = (1.5 * randn(g, sum(new), heads * group, dim)).to(dtype)
    start = np.concatenate([[0], np.cumsum(new)])
    scale = dim ** -0.5
    want, tol = R.chunk(st, q, tables, lengths, start, scale)
    got = st.attend_chunk(q, dev(tables), dev(lengths), q_start=dev(start))
    R.assert_close(got, want, tol, "ragged")
    if len(set(new)) == 1:
        R.assert_close(st.attend_chunk(q, dev(tables), dev(lengths), scale=scale), want, tol, "the same number each")
    again = st.attend_chunk(q, dev(tables), dev(lengths), q_start=dev(start))
    assert torch.equal(got, again), "two runs differ"


MORE_CHUNKS = [
    # rows enough for shared tiles at every width, pages smaller and larger than a tile
    ([40, 60], [40, 333], 2, 2, 32, 16, F16),
    ([70], [500], 1, 3, 32, 128, BF16),
    ([50, 20], [300, 700], 2, 3, 96, 128, BF16),
    ([45], [129], 3, 2, 96, 64, F16),
    ([90], [4000], 1, 1, 64, 32, BF16),
    ([33, 0, 64], [33, 50, 4097], 1, 4, 128, 256, F16),
]


@pytest.mark.parametrize("new,lengths,heads,group,dim,page,dtype", MORE_CHUNKS)
def test_chunk_in_shared_tiles(S, new, lengths, heads, group, dim, page, dtype):
    test_chunk(S, new, lengths, heads, group, dim, page, dtype)


@pytest.mark.parametrize("sequences,new,context,heads,group,dim,page", [(4, 600, 300, 8, 8, 128, 64), (4, 513, 100, 16, 4, 96, 32), (3, 700, 777, 8, 4, 64, 64)])
def test_large_chunks(S, sequences, new, context, heads, group, dim, page):
    """Rows enough to fill the GPU with the largest blocks."""
    g = gen(21)
    lengths = [new + context + 17 * i for i in range(sequences)]
    pages = sum(-(-n // page) for n in lengths) + 1
    st = filled(S, pages, heads, page, dim, seed=22, spread=0.3)
    tables = dev(make_tables(g, lengths, pages, page, junk=False))
    q = (1.5 * randn(g, sequences * new, heads * group, dim)).to(BF16)
    want, tol = R.chunk_on_gpu(st, q, tables, lengths, [i * new for i in range(sequences + 1)], dim ** -0.5)
    got = st.attend_chunk(q, tables, dev(lengths))
    off = (got.double() - want).abs() - tol
    assert not (off > 0).any() and not torch.isnan(got).any(), float(off.max())
    start = dev([i * new for i in range(sequences + 1)])
    assert torch.equal(got, st.attend_chunk(q, tables, dev(lengths), q_start=start)), "two runs differ"


def test_many_short_sequences(S):
    """More sequences than a wavefront counts at a time, some without queries."""
    g = gen(3)
    rng = np.random.default_rng(4)
    n, page = 200, 16
    new = rng.integers(0, 4, n)
    new[70:140] = 0
    lengths = new + rng.integers(0, 40, n)
    pages = int(sum(-(-l // page) for l in lengths)) + 1
    st = filled(S, pages, 1, page, 64)
    tables = make_tables(g, list(lengths), pages, page)
    q = randn(g, int(new.sum()), 2, 64).to(BF16)
    start = np.concatenate([[0], np.cumsum(new)])
    want, tol = R.chunk(st, q, tables, lengths, start, 0.125)
    R.assert_close(st.attend_chunk(q, dev(tables), dev(lengths), q_start=dev(start)), want, tol)


@pytest.mark.parametrize("n", [2, 63, 64, 65])
@pytest.mark.parametrize("same", [False, True])
def test_sequences_of_uneven_lengths(S, n, same):
    """Rows enough for shared tiles of as many sequences as a wavefront has lanes, and one more: lengths in no order, several alike, some 0, some without queries."""
    g = gen(n)
    rng = np.random.default_rng(n)
    page, group = 16, 4
    new = np.full(n, 33) if same else rng.choice([0, 1, 20, 33, 70], n)
    if not same:
        new[:2] = 70
    lengths = rng.choice([0, 5, 33, 90, 90, 200], n)
    lengths[1] = 200
    pages = int(sum(-(-l // page) for l in lengths)) + 1
    st = filled(S, pages, 1, page, 32)
    tables = make_tables(g, list(lengths), pages, page)
    q = randn(g, int(new.sum()), group, 32).to(BF16)
    start = np.concatenate([[0], np.cumsum(new)])
    want, tol = R.chunk(st, q, tables, lengths, start, 0.2)
    R.assert_close(st.attend_chunk(q, dev(tables), dev(lengths), scale=0.2, q_start=None if same else dev(start)), want, tol)


PASSAGES = [
    # new tokens, found, stock lengths, heads, group, dim, page, type, weighted
    ([1], 1, [1], 1, 1, 32, 16, BF16, False),
    ([1, 1], 10, [30, 1, 64, 65, 0, 128, 17, 200, 5, 33, 90, 64], 2, 4, 128, 64, BF16, True),
    ([1, 1, 1], 3, [700, 3, 1500, 60], 2, 8, 64, 16, F16, True),
    ([20, 1, 0, 33], 5, [70, 10, 300, 64, 31, 1], 1, 3, 96, 32, BF16, False),
    ([96], 10, [100] * 11, 1, 4, 128, 64, BF16, True),
    ([70, 70], 4, [130, 64, 9, 500, 16], 2, 2, 64, 16, F16, False),
]


@pytest.mark.parametrize("new,found,stock,heads,group,dim,page,dtype,weighted", PASSAGES)
def test_passages(S, new, found, stock, heads, group, dim, page, dtype, weighted):
    g, rng = gen(sum(stock)), np.random.default_rng(sum(stock))
    pages = sum(-(-n // page) for n in stock) + 2
    st = filled(S, pages, heads, page, dim, seed=found)
    tables = make_tables(g, stock, pages, page, spare=1)
    ids = rng.integers(0, len(stock), (len(new), found))         # numbers may stand twice
    scores = rng.normal(size=(len(new), found)).astype(np.float32) if weighted else None
    if found > 2:
        ids[0, 1], ids[-1, 0] = -1, len(stock) + 5
        ids[0, 2] = 2 ** 40
    q = (1.5 * randn(g, sum(new), heads * group, dim)).to(dtype)
    start = np.concatenate([[0], np.cumsum(new)])
    want, tol = R.passages(st, q, ids, tables, stock, start, scores, -2.5, 0.11)
    args = dict(scores=None if scores is None else dev(scores, F32), score_weight=-2.5, scale=0.11)
    got = st.attend_passages(q, dev(ids, torch.int64), dev(tables), dev(stock), q_start=dev(start), **args)
    R.assert_close(got, want, tol, "ragged")
    if len(set(new)) == 1:
        R.assert_close(st.attend_passages(q, dev(ids, torch.int64), dev(tables), dev(stock), **args), want, tol, "the same number each")
    assert torch.equal(got, st.attend_passages(q, dev(ids, torch.int64), dev(tables), dev(stock), q_start=dev(start), **args)), "two runs differ"


MORE_PASSAGES = [
    # more passages than are looked up at a time (found, and numbers outside among them)
    ([1, 1], 50, [30, 64, 5, 100, 0, 17] * 3, 2, 4, 64, 16, BF16, True),
    ([40], 64, [9, 70, 33, 0, 128] * 4, 1, 2, 128, 64, F16, True),
    ([17, 30], 43, [20, 16, 64, 40] * 5, 2, 3, 32, 16, BF16, False),
    ([1], 22, [300, 65], 1, 16, 96, 32, BF16, True),
    # one long passage for one token: cut, and joined
    ([1], 1, [3000], 2, 4, 128, 64, BF16, False),
    ([60], 2, [2500, 900], 1, 2, 64, 128, BF16, True),
]


@pytest.mark.parametrize("new,found,stock,heads,group,dim,page,dtype,weighted", MORE_PASSAGES)
def test_many_and_long_passages(S, new, found, stock, heads, group, dim, page, dtype, weighted):
    test_passages(S, new, found, stock, heads, group, dim, page, dtype, weighted)


@pytest.mark.parametrize("new", [1, 40])
def test_nothing_found(S, new):
    """Every number outside the passages, passages without tokens, terms of -inf, tables of width 0, no passages at all: zeros."""
    st = filled(S, 8, 2, 16, 64)
    g = gen(9)
    q = randn(g, 2 * new, 4, 64).to(BF16)
    tables, lengths = dev(make_tables(g, [20, 0, 30], 8, 16)), dev([20, 0, 30])
    ids = lambda v: dev(v, torch.int64)  # noqa: E731
    fill = lambda: torch.full_like(q, 3.0)  # noqa: E731
    assert (st.attend_passages(q, ids([[-1, 3], [1, 1]]), tables, lengths, out=fill()) == 0).all()
    inf = dev([[float("inf")] * 2] * 2, F32)
    assert (st.attend_passages(q, ids([[0, 2], [2, 0]]), tables, lengths, scores=inf, score_weight=-1.0, out=fill()) == 0).all()
    assert (st.attend_passages(q, ids([[0, 2], [2, 0]]), tables[:, :0].contiguous(), lengths, out=fill()) == 0).all()
    assert (st.attend_passages(q, ids([[0, 2], [2, 0]]), tables[:0], lengths[:0], out=fill()) == 0).all()
    assert (st.attend_chunk(q, tables[:2], dev([-5, 0]), out=fill()) == 0).all()
    # one of two terms -inf: the other passage alone
    half = dev([[0.0, float("inf")]] * 2, F32)
    one = st.attend_passages(q, ids([[0, 2], [2, 0]]), tables, lengths, scores=half, score_weight=-1.0)
    assert torch.equal(one, st.attend_passages(q, ids([[0, -1], [2, -1]]), tables, lengths))


@pytest.mark.parametrize("new,group", [(1, 4), (50, 1), (150, 2)])
def test_what_is_not_seen_does_not_matter(S, new, group):
    """NaN and infinite states beyond a sequence's length, on other pages, and in keys behind a query change nothing for that query; page numbers
    outside the store leave their keys out; lengths beyond the table are taken as the table's."""
    page, dim = 16, 64
    lengths = [200, 333]
    g = gen(11)
    pages = sum(-(-n // page) for n in lengths) + 4
    st = filled(S, pages, 2, page, dim)
    tables = make_tables(g, lengths, pages, page)
    q = randn(g, 2 * new, 2 * group, dim).to(BF16)
    scale = 0.125
    before = st.attend_chunk(q, dev(tables), dev(lengths))
    used = np.zeros((pages, page), bool)
    for s, n in enumerate(lengths):
        t = np.arange(n)
        used[tables[s][t // page], t % page] = True
    free = torch.from_numpy(np.flatnonzero(~used.reshape(-1))).cuda()
    bad = torch.full((len(free), 2, dim), float("nan"), device="cuda")
    st.write(bad, bad, free)
    assert torch.equal(before, st.attend_chunk(q, dev(tables), dev(lengths)))
    # a NaN in the last key of the first sequence: seen by its last query alone
    slot = int(tables[0][199 // page]) * page + 199 % page
    st.write(bad[:1], bad[:1], torch.tensor([slot], device="cuda"))
    got = st.attend_chunk(q, dev(tables), dev(lengths))
    assert torch.isnan(got[new - 1]).all()
    assert torch.equal(got[:new - 1], before[:new - 1]) and torch.equal(got[new:], before[new:])
    # page numbers outside the store
    t2 = tables.copy()
    t2[1, 3], t2[1, 10], t2[0, -1] = -1, pages, -7
    want, tol = R.chunk(st, q, t2, lengths, [0, new, 2 * new], scale)
    R.assert_close(st.attend_chunk(q, dev(t2), dev(lengths)), want, tol, "page numbers")
    # lengths beyond the table (the second sequence's alone fills it)
    over = [200, 10 ** 6]
    want, tol = R.chunk(st, q, t2, over, [0, new, 2 * new], scale)
    R.assert_close(st.attend_chunk(q, dev(t2), dev(over)), want, tol, "length")


def test_steps_of_very_different_sizes(S):
    """Values whose steps span 60 powers of ten, the largest under a small weight; rows of zeros; queries of very different sizes in one tile."""
    g = gen(12)
    st = S.States.empty(8, 1, 16, 64)
    k, v = randn(g, 128, 1, 64), randn(g, 128, 1, 64)
    v[::3] *= 1e-30
    v[5] *= 1e28
    k[5] *= 0.01
    v[7] = 0
    k[9] = 0
    st.write(k, v, torch.arange(128, device="cuda"))
    q = randn(g, 40, 2, 64)
    q[3] *= 1e-20
    q[4] = 0
    q[5, 0, 3:] = 0
    q[6] *= 30
    q = q.to(BF16)
    tables = np.arange(8, dtype=np.int32)[None]
    want, tol = R.chunk(st, q, tables, [128], [0, 40], 0.125)
    R.assert_close(st.attend_chunk(q, dev(tables), dev([128])), want, tol)
    one = q[6:7].contiguous()
    want, tol = R.chunk(st, one, tables, [128], [0, 1], 0.125)
    R.assert_close(st.attend_chunk(one, dev(tables), dev([128])), want, tol)


@pytest.mark.parametrize("new", [1, 150])
def test_nan_and_infinite_queries(S, new):
    """A query that holds a NaN or an infinity answers NaN; its neighbours in the tile answer as before."""
    g = gen(13)
    st = filled(S, 20, 1, 16, 64)
    q = randn(g, new, 4, 64).to(F16)
    tables, lengths = dev(np.arange(20)[None]), dev([300])
    before = st.attend_chunk(q, tables, lengths)
    q[new // 2, 1, 5] = float("nan")
    q[0, 2, 0] = float("inf")
    got = st.attend_chunk(q, tables, lengths)
    hit = torch.zeros((new, 4), dtype=torch.bool, device="cuda")
    hit[new // 2, 1] = hit[0, 2] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], before[~hit])


@pytest.mark.parametrize("new", [1, 70])
def test_strides_and_alignment(S, new):
    """Queries and answers as slices, heads first, and off 16 bytes: the same answers; memory between rows is left alone."""
    g = gen(14)
    st = filled(S, 40, 2, 16, 96)
    q = randn(g, 2 * new, 6, 96).to(BF16)
    tables, lengths = dev(make_tables(g, [300, 222], 40, 16)), dev([300, 222])
    want = st.attend_chunk(q, tables, lengths)
    for layout in ("slice", "heads first", "odd"):
        out = rows_in_layout(torch.zeros_like(q), layout)
        got = st.attend_chunk(rows_in_layout(q, layout), tables, lengths, out=out)
        assert got is out and torch.equal(got, want), layout
    wide = torch.full((2 * new, 8, 96), 2.0, dtype=BF16, device="cuda")
    st.attend_chunk(q, tables, lengths, out=wide[:, 1:7])
    assert (wide[:, 0] == 2).all() and (wide[:, 7] == 2).all() and torch.equal(wide[:, 1:7], want)


@pytest.mark.parametrize("new", [1, 66])
def test_tokens_of_no_sequence_are_left_alone(S, new):
    g = gen(15)
    st = filled(S, 40, 1, 16, 64)
    q = randn(g, 2 * new + 5, 4, 64).to(BF16)
    tables, lengths = dev(make_tables(g, [300, 222], 40, 16)), dev([300, 222])
    out = torch.full_like(q, 4.0)
    st.attend_chunk(q, tables, lengths, q_start=dev([2, 2 + new, 2 + 2 * new]), out=out)
    assert (out[:2] == 4).all() and (out[2 + 2 * new:] == 4).all()
    want = st.attend_chunk(q[2:2 + 2 * new], tables, lengths)
    assert torch.equal(out[2:2 + 2 * new], want)


def test_store_beyond_32_bit_offsets(S):
    """A store of more than 2^32 codes: the last pages are written, read and attended to."""
    pages, heads, page, dim = 2 ** 32 // (4 * 128 * 128) + 9, 4, 128, 128
    codes = lambda *s: torch.empty(s, dtype=torch.int8, device="cuda")  # noqa: E731
    steps = lambda: torch.zeros((pages, heads, page), device="cuda")  # noqa: E731
    st = S.States(codes(pages, heads, page, dim), codes(pages, heads, dim, page), steps(), steps())
    g = gen(16)
    last = [pages - 1, pages - 5, 3]
    slots = torch.cat([p * page + torch.arange(page, device="cuda") for p in last])
    k, v = randn(g, 3 * page, heads, dim).to(BF16), randn(g, 3 * page, heads, dim).to(BF16)
    st.write(k, v, slots)
    small = S.States.empty(3, heads, page, dim)
    small.write(k, v, torch.arange(3 * page, device="cuda"))
    for x, y in zip(st.read(slots, F32), small.read(torch.arange(3 * page, device="cuda"), F32)):
        assert torch.equal(x, y)
    for new in (1, 100):
        q = randn(g, new, heads, dim).to(BF16)
        assert torch.equal(st.attend_chunk(q, dev([last]), dev([350])), small.attend_chunk(q, dev([[0, 1, 2]]), dev([350])))
        ids = dev([[1, 0]], torch.int64)
        assert torch.equal(st.attend_passages(q, ids, dev([[last[0]], [last[1]]]), dev([128, 99])), small.attend_passages(q, ids, dev([[0], [1]]), dev([128, 99])))


def test_streams_and_graph(S):
    """On a stream of its own, and captured into a graph whose replays follow new contents (write, both attentions), the same as eager calls."""
    g = gen(17)
    st = filled(S, 60, 2, 16, 64)
    tables, lengths = dev(make_tables(g, [400, 300], 50, 16)), dev([400, 300])
    q = randn(g, 2, 8, 64).to(BF16)
    ids = dev([[0, 1], [1, -1]], torch.int64)
    k, v = randn(g, 2, 2, 64).to(BF16), randn(g, 2, 2, 64).to(BF16)
    slots = (tables[torch.arange(2), (lengths.long() - 1) // 16].long() * 16 + (lengths.long() - 1) % 16).contiguous()
    ws = torch.empty(max(st.workspace_bytes(q, 2, tables.shape[1]), st.workspace_bytes(q, 2, tables.shape[1], found=2)), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q), torch.empty_like(q)]

    def step():
        st.write(k, v, slots)
        st.attend_chunk(q, tables, lengths, out=outs[0], workspace=ws)
        st.attend_passages(q, ids, tables, lengths, out=outs[1], workspace=ws)

    step()
    torch.cuda.synchronize()
    eager = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in outs:
            o.zero_()
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        k.copy_(randn(g, 2, 2, 64))
        q.copy_(randn(g, 2, 8, 64))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in outs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs)), i


def test_refusals_on_the_gpu(S):
    from paper_2410_18926_amd.binding import LorannError
    st = filled(S, 4, 2, 16, 64)
    q = torch.zeros((2, 4, 64), dtype=BF16, device="cuda")
    tables, lengths = dev([[0, 1], [2, 3]]), dev([20, 20])
    with pytest.raises(LorannError, match="float|F16|BF16"):
        st.attend_chunk(q.float(), tables, lengths)
    with pytest.raises(LorannError, match="multiple"):
        st.attend_chunk(q[:, :3].contiguous(), tables, lengths)
    with pytest.raises(LorannError, match="divide"):
        st.attend_chunk(torch.zeros((3, 4, 64), dtype=BF16, device="cuda"), tables, lengths)
    with pytest.raises(LorannError, match="scale"):
        st.attend_chunk(q, tables, lengths, scale=float("nan"))
    with pytest.raises(LorannError, match="device pointer"):
        st.attend_chunk(q.cpu(), tables, lengths, out=q)
    with pytest.raises(LorannError, match="device pointer"):
        st.attend_chunk(q, tables.cpu(), lengths)
    with pytest.raises(LorannError, match="device pointer"):
        st.write(q[:, :2].contiguous(), q[:, :2].contiguous(), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="int32"):
        st.attend_chunk(q, tables.long(), lengths)
    with pytest.raises(ValueError, match="contiguous"):
        st.attend_chunk(q, dev([[0, 2], [1, 3]]).t(), lengths)
    with pytest.raises(ValueError, match="consecutive"):
        st.attend_chunk(torch.zeros((2, 4, 128), dtype=BF16, device="cuda")[:, :, ::2], tables, lengths)
    long = filled(S, 300, 1, 16, 64)
    table = dev(np.arange(300)[None])
    one = torch.zeros((1, 1, 64), dtype=BF16, device="cuda")
    assert long.workspace_bytes(one, 1, 300) > 0
    with pytest.raises(LorannError, match="workspace"):
        long.attend_chunk(one, table, dev([4800]), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
