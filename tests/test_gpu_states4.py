"""The 4-bit state store and its attention on the GPU against their definitions in 64 bits (states4_reference.py; the attention's tolerances are derived in states_reference.py)."""
import numpy as np
import pytest
import torch

import states4_reference as R4
import states_reference as R
from test_gpu_states import BF16, CHUNKS, F16, F32, MORE_CHUNKS, MORE_PASSAGES, PASSAGES, dev, gen, make_tables, randn, rows_in_layout

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2410_18926_amd import binding, states4
    assert binding.LIB_PATH.exists(), "build the HIP library first (python -m paper_2410_18926_amd.build)"
    assert torch.cuda.is_available(), "these tests need the GPU"
    return states4


def filled(S, pages, heads, page, dim, seed=1, spread=1.0):
    """A store whose every slot holds the states of some token: components with a mean, rows of different lengths, groups of 32 of different sizes."""
    g = gen(seed)
    st = S.States4.empty(pages, heads, page, dim)
    n = pages * page
    size = torch.exp(spread * randn(g, 2, 1, heads, dim // 32)).repeat_interleave(32, -1)
    k = (randn(g, n, heads, dim) + 0.3) * torch.exp(0.4 * spread * randn(g, n, heads, 1)) * size[0]
    v = (randn(g, n, heads, dim) - 0.2) * torch.exp(0.8 * spread * randn(g, n, heads, 1)) * size[1]
    st.write(k / k.std(), v, torch.arange(n, device="cuda"))
    return st


# ---- writing and reading ----

def check_written(st, before, k, v, slots):
    """Codes, factors and steps are those of the definition bit for bit, in the slots named and nowhere else.  Returns what was written (key values, value values, which slots are there)."""
    after, n_slots = R4.arrays(st), st.pages * st.page_size
    s = slots.cpu().numpy()
    ok = (s >= 0) & (s < n_slots)
    p, o = s[ok] // st.page_size, s[ok] % st.page_size
    kc, kf, ks = R4.quantise(k.float().cpu().numpy())
    vc, vf, vs = R4.quantise(v.float().cpu().numpy())
    four = lambda f: np.pad(f, [(0, 0), (0, 0), (0, 4 - f.shape[-1])])  # noqa: E731
    want = {n: a.copy() for n, a in before.items()}
    want["k_codes"][p, :, o], want["k_factors"][p, :, o], want["k_scales"][p, :, o] = R4.pack_keys(kc)[ok], four(kf)[ok], ks[ok]
    want["v_codes"][p, :, :, o], want["v_factors"][p, :, o], want["v_scales"][p, :, o] = R4.pack_values(vc)[ok], four(vf)[ok], vs[ok]
    for name in want:
        assert np.array_equal(after[name], want[name], equal_nan=name.endswith("scales")), name
    return R4.values(kc, kf, ks), R4.values(vc, vf, vs), ok


@pytest.mark.parametrize("dim,page,heads,tokens", [(128, 64, 3, 200), (96, 16, 2, 77), (64, 32, 1, 1), (32, 128, 5, 130), (128, 256, 2, 300), (128, 16, 8, 16), (64, 16, 2, 17)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("order", ["shuffled", "run", "runs from odd places", "backwards"])
def test_write_and_read_back(S, dim, page, heads, tokens, dtype, order):
    g = gen(dim * 7 + page + tokens)
    pages = -(-tokens // page) + 3
    st = filled(S, pages, heads, page, dim, seed=5)
    before = R4.arrays(st)
    k, v = randn(g, tokens, heads, dim).to(dtype), (randn(g, tokens, heads, dim) * 3 + 1).to(dtype)
    if tokens > 8:
        k[3, 0] = 0
        v[4, heads - 1] = 0
        k[5, 0, 7] = float("nan")
        v[6, 0, dim - 1] = float("inf")
        v[7, 0] *= 1e-4
        k[1, 0, :32] *= 2 ** -9
        v[1, 0, dim - 32:] = 0
        if dtype != F16:
            k[8, 0] = 1e-36 * torch.arange(dim, device="cuda")
            k[2, 0] *= 1e37
            v[2, 0, :32] *= 1e-7
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
    wk, wv, ok = check_written(st, before, k, v, slots)
    for out_type in (F32, F16, BF16):
        out = None
        if out_type == dtype:      # into another layout as well
            out = tuple(rows_in_layout(torch.full((tokens, heads, dim), 5.0, dtype=dtype, device="cuda"), layouts[(tokens + i + 1) % 4]) for i in range(2))
        for got, want in zip(st.read(slots, out_type, out=out), (wk, wv)):
            x = torch.from_numpy(np.where(ok[:, None, None], want, np.float32(0))).to(out_type)
            assert np.array_equal(got.float().cpu().numpy(), x.float().numpy(), equal_nan=True), (out_type, order)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_halfway_values(S, dtype):
    """Values exactly between two codes, and those next to them in the type, under factors and maxima of many significant bits."""
    rng = np.random.default_rng(6)
    n, dim = 512, 128
    bits = {F32: 24, F16: 11, BF16: 8}[dtype]
    few = {F32: 12, F16: 4, BF16: 3}[dtype]
    # maxima of `few` bits times 24 / 8 ... : halfway points n r a / 24 are then often numbers of the type
    a = 3 * rng.integers(1, 2 ** few, (n, 1)) * np.exp2(rng.integers(-6, 6, (n, 1)))
    x = rng.choice([1, 3, 5, 7, 10, 14, 20], (n, dim)) * rng.choice([8, 9, 10, 11, 12, 13, 14, 15], (n, dim // 32)).repeat(32, 1) / 16 * a / 24
    x = x * rng.choice([-1, 1], x.shape)
    x[:, 0] = a[:, 0]
    t = torch.from_numpy(x).to(dtype).float().numpy()
    step = np.exp2(np.floor(np.log2(np.abs(t))) - (bits - 1))
    t[n // 2:] += (step * rng.integers(-1, 2, t.shape))[n // 2:]          # the neighbours of some
    k = torch.from_numpy(t)[:, None].to("cuda", dtype)
    assert np.array_equal(k.float().cpu().numpy()[:, 0], t)
    st = S.States4.empty(n // 64, 1, 64, dim)
    before = R4.arrays(st)
    slots = torch.arange(n, device="cuda")
    st.write(k, -k, slots)
    check_written(st, before, k, -k, slots)


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

@pytest.mark.parametrize("new,lengths,heads,group,dim,page,dtype", CHUNKS + MORE_CHUNKS)
def test_chunk(S, new, lengths, heads, group, dim, page, dtype):
    g = gen(sum(lengths) + dim)
    pages = sum(-(-n // page) for n in lengths) + 3
    st = filled(S, pages, heads, page, dim, seed=sum(new))
    tables = make_tables(g, lengths, pages, page, spare=sum(new) % 3)
    q = (1.5 * randn(g, sum(new), heads * group, dim)).to(dtype)
    start = np.concatenate([[0], np.cumsum(new)])
    scale = dim ** -0.5
    want, tol = R.chunk(R4.held(st), q, tables, lengths, start, scale)
    got = st.attend_chunk(q, dev(tables), dev(lengths), q_start=dev(start))
    R.assert_close(got, want, tol, "ragged")
    if len(set(new)) == 1:
        R.assert_close(st.attend_chunk(q, dev(tables), dev(lengths), scale=scale), want, tol, "the same number each")
    assert torch.equal(got, st.attend_chunk(q, dev(tables), dev(lengths), q_start=dev(start))), "two runs differ"


@pytest.mark.parametrize("sequences,new,context,heads,group,dim,page", [(4, 600, 300, 8, 8, 128, 64), (4, 513, 100, 16, 4, 96, 32), (3, 700, 777, 8, 4, 64, 64)])
def test_large_chunks(S, sequences, new, context, heads, group, dim, page):
    """Rows enough to fill the GPU with the largest blocks."""
    g = gen(21)
    lengths = [new + context + 17 * i for i in range(sequences)]
    pages = sum(-(-n // page) for n in lengths) + 1
    st = filled(S, pages, heads, page, dim, seed=22, spread=0.3)
    tables = dev(make_tables(g, lengths, pages, page, junk=False))
    q = (1.5 * randn(g, sequences * new, heads * group, dim)).to(BF16)
    want, tol = R.chunk_on_gpu(R4.held(st), q, tables, lengths, [i * new for i in range(sequences + 1)], dim ** -0.5)
    got = st.attend_chunk(q, tables, dev(lengths))
    off = (got.double() - want).abs() - tol
    assert not (off > 0).any() and not torch.isnan(got).any(), float(off.max())
    start = dev([i * new for i in range(sequences + 1)])
    assert torch.equal(got, st.attend_chunk(q, tables, dev(lengths), q_start=start)), "two runs differ"


@pytest.mark.parametrize("new,found,stock,heads,group,dim,page,dtype,weighted", PASSAGES + MORE_PASSAGES)
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
    want, tol = R.passages(R4.held(st), q, ids, tables, stock, start, scores, -2.5, 0.11)
    args = dict(scores=None if scores is None else dev(scores, F32), score_weight=-2.5, scale=0.11)
    got = st.attend_passages(q, dev(ids, torch.int64), dev(tables), dev(stock), q_start=dev(start), **args)
    R.assert_close(got, want, tol, "ragged")
    assert torch.equal(got, st.attend_passages(q, dev(ids, torch.int64), dev(tables), dev(stock), q_start=dev(start), **args)), "two runs differ"


@pytest.mark.parametrize("new,dim,page", [(1, 128, 64), (12, 96, 16), (60, 64, 32), (300, 128, 16)])
def test_memory_that_was_never_written(S, new, dim, page):
    """A store made over memory that holds anything (bytes of ones: as factors, NaN in binary16; NaN steps): what no length covers changes no answer and no sum."""
    g = gen(new)
    n, heads = 333, 2
    pages = -(-n // page) + 1
    k, v = randn(g, n, heads, dim), randn(g, n, heads, dim)
    q = randn(g, new, 2 * heads, dim).to(BF16)
    tables = torch.arange(pages + 1, dtype=torch.int32, device="cuda")[None].flip(1).contiguous()          # (pages .. 0: page 0, which stands in for pages that are not there, is not written either)
    tables[0, 2] = 10 ** 6
    at = torch.arange(n, device="cuda")
    slots = tables[0, at // page].long() * page + at % page
    got = []
    for fill in (False, True):
        st = S.States4.empty(pages + 1, heads, page, dim)
        if fill:
            for t in (st.k_codes, st.v_codes, st.k_factors, st.v_factors):
                t.fill_(255)
            st.k_scales.fill_(float("nan"))
            st.v_scales.fill_(float("inf"))
        st.write(k, v, slots)
        lengths = dev([n])
        ids, dists = dev([[0, 0, 0]], torch.int64), torch.zeros((1, 3), device="cuda")
        got.append((st.attend_chunk(q, tables, lengths), st.attend_passages(q, ids, tables, lengths, scores=dists), st.attend_weights(q, tables, lengths),
                    *st.read(torch.cat([slots, slots.new_tensor([-1, 10 ** 9])]))))
        assert all(torch.isfinite(x).all() for x in got[-1])
    assert all(torch.equal(x, y) for x, y in zip(*got))


@pytest.mark.parametrize("new,dim,page", [(1, 128, 64), (40, 64, 16), (60, 96, 32)])
def test_keys_that_hold_nothing_or_no_number(S, new, dim, page):
    """Rows of zeros take their share of the weights alone; a NaN reaches the queries that see its key and no others; pages outside the store are left out."""
    g = gen(dim)
    n = 300
    pages = -(-n // page)
    st = S.States4.empty(pages + 1, 2, page, dim)
    k, v = randn(g, n, 2, dim), randn(g, n, 2, dim)
    k[5], v[9], v[50:70] = 0, 0, 0
    st.write(k, v, torch.arange(n, device="cuda"))
    tables = np.arange(pages, dtype=np.int32)[None].copy()
    tables[0, 2 if page > 32 else 5] = 10 ** 6
    q = randn(g, new, 4, dim).to(BF16)
    check = lambda length: R.assert_close(st.attend_chunk(q, dev(tables), dev([length])), *R.chunk(R4.held(st), q, tables, [length], [0, new], dim ** -0.5))  # noqa: E731
    check(n)
    check(new // 2)                # queries without a key: zeros
    check(0)
    v[n - 1, 0, 3] = float("nan")
    k[n - 2, 1, 0] = float("inf")
    st.write(k, v, torch.arange(n, device="cuda"))
    got = st.attend_chunk(q, dev(tables), dev([n])).float()
    # seen by the last query alone (key n - 1, head 0), by the last two (key n - 2, head 1)
    bad = torch.isnan(got).any(2).view(new, 2, 2)
    want = torch.zeros_like(bad)
    want[-1:, 0] = True
    want[-2:, 1] = True
    assert torch.equal(bad, want) and torch.equal(torch.isnan(got).all(2), torch.isnan(got).any(2))


def test_nothing_found(S):
    st = filled(S, 8, 2, 16, 64)
    g = gen(9)
    for new in (1, 40):
        q = randn(g, 2 * new, 4, 64).to(BF16)
        tables, lengths = dev(make_tables(g, [20, 0, 30], 8, 16)), dev([20, 0, 30])
        got = st.attend_passages(q, dev([[-1, 3], [1, 1]], torch.int64), tables, lengths, out=torch.full_like(q, 3.0))
        assert (got == 0).all()


def test_rows_without_a_sequence_and_gaps_stay(S):
    """Rows before the first and behind the last sequence, and what lies between the rows of `out`, are left as they were."""
    st = filled(S, 40, 2, 16, 64)
    g = gen(3)
    for new in (1, 50):
        lengths, total = [200, 77], 2 * new + 7
        tables = make_tables(g, lengths, 40, 16)
        q = randn(g, total, 4, 64).to(F16)
        wide = torch.full((total, 9, 64), 7.0, dtype=F16, device="cuda")
        start = [3, 3 + new, 3 + 2 * new]
        got = st.attend_chunk(q, dev(tables), dev(lengths), q_start=dev(start), out=wide[:, 2:6])
        want, tol = R.chunk(R4.held(st), q, tables, lengths, start, 0.125)
        live = slice(3, 3 + 2 * new)
        R.assert_close(got[live], want[live], tol[live])
        assert (wide[:3] == 7).all() and (wide[3 + 2 * new:] == 7).all() and (wide[:, :2] == 7).all() and (wide[:, 6:] == 7).all()


def test_a_captured_step(S):
    """A decoding step (write, attend) in a graph, replayed with other contents, among eager work."""
    st = filled(S, 64, 2, 16, 128, seed=4)
    g = gen(8)
    k, v = randn(g, 2, 2, 128).to(BF16), randn(g, 2, 2, 128).to(BF16)
    q = randn(g, 2, 8, 128).to(BF16)
    tables, lengths = dev(np.arange(60).reshape(2, 30)), dev([401, 77])
    slots = torch.tensor([400, 480 + 76], device="cuda")
    ws = torch.empty(st.workspace_bytes(q, 2, 30), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)

    def step():
        st.write(k, v, slots)
        st.attend_chunk(q, tables, lengths, out=out, workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        for t in (k, v, q):
            t.copy_(randn(g, *t.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want, tol = R.chunk(R4.held(st), q, tables.cpu().numpy(), [401, 77], [0, 1, 2], 128 ** -0.5)
        R.assert_close(got, want, tol, f"replay {i}")
        step()
        assert torch.equal(out, got)


def test_a_store_beyond_2_gib(S):
    """Offsets that pass 32 bits: pages at the end of a store of 2^31 bytes of key codes and more."""
    page, heads, dim = 256, 16, 128
    pages = (2 ** 31 + 2 ** 28) // (page * heads * dim // 2)
    st = S.States4.empty(pages, heads, page, dim)
    g = gen(2)
    n = 700
    use = torch.tensor([pages - 1, 3, pages - 2], device="cuda")
    t = torch.arange(n, device="cuda")
    slots = use[t // page] * page + t % page
    k, v = randn(g, n, heads, dim), randn(g, n, heads, dim)
    st.write(k, v, slots)
    got_k, got_v = st.read(slots, F32)
    for got, x in ((got_k, k), (got_v, v)):
        assert np.array_equal(got.cpu().numpy(), R4.values(*R4.quantise(x.cpu().numpy())))
    few = S.States4.empty(3, heads, page, dim)
    few.write(k, v, t)
    for new in (1, 70):
        q = randn(g, new, heads, dim).to(BF16)
        assert torch.equal(st.attend_chunk(q, use[None].int(), dev([n])), few.attend_chunk(q, dev([[0, 1, 2]]), dev([n])))
