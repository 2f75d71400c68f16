"""Sums of attention weights, and eviction by them, on the GPU against their definitions (evict_reference.py, where the tolerances are derived)."""
import numpy as np
import pytest
import torch

import evict_reference as E
import states4_reference as R4
import states_reference as R
import test_gpu_states as T8
import test_gpu_states4 as T4
from test_gpu_states import BF16, CHUNKS, F16, F32, MORE_CHUNKS, dev, gen, make_tables, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=[8, 4])
def B(request):
    """(module with the store, a function that makes one in use, what its codes stand for)"""
    from paper_2410_18926_amd import binding, states, states4
    assert binding.LIB_PATH.exists(), "build the HIP library first (python -m paper_2410_18926_amd.build)"
    assert torch.cuda.is_available(), "these tests need the GPU"
    if request.param == 8:
        return states.States, lambda *a, **k: T8.filled(states, *a, **k), lambda st: st
    return states4.States4, lambda *a, **k: T4.filled(states4, *a, **k), R4.held


def arrays(st):
    return R4.arrays(st) if hasattr(st, "k_factors") else R.store_arrays(st)


# ---- weights ----

def check_weights(B, new, lengths, heads, group, dim, page, dtype, spare=0):
    _, filled, held = B
    g = gen(sum(lengths) + dim)
    pages = sum(-(-n // page) for n in lengths) + 3
    st = filled(pages, heads, page, dim, seed=sum(new))
    tables = make_tables(g, lengths, pages, page, spare=spare)
    q = (1.5 * randn(g, sum(new), heads * group, dim)).to(dtype)
    start = np.concatenate([[0], np.cumsum(new)])
    before = torch.rand((len(lengths), heads, tables.shape[1] * page), generator=g, device="cuda")
    want, tol = E.weights(held(st), q, tables, lengths, start, dim ** -0.5, before.cpu().numpy())
    got = st.attend_weights(q, dev(tables), dev(lengths), q_start=dev(start), before=before)
    R.assert_close(got, want, tol, "ragged")
    if len(set(new)) == 1:
        R.assert_close(st.attend_weights(q, dev(tables), dev(lengths), scale=dim ** -0.5, before=before), want, tol, "the same number each")
    assert torch.equal(got, st.attend_weights(q, dev(tables), dev(lengths), q_start=dev(start), before=before)), "two runs differ"
    first = st.attend_weights(q, dev(tables), dev(lengths), q_start=dev(start))
    R.assert_close(first, want - before.double().cpu().numpy(), tol, "from zeros")
    inplace = before.clone()
    assert st.attend_weights(q, dev(tables), dev(lengths), q_start=dev(start), before=inplace, out=inplace) is inplace and torch.equal(inplace, got)


@pytest.mark.parametrize("new,lengths,heads,group,dim,page,dtype", CHUNKS + MORE_CHUNKS)
def test_weights(B, new, lengths, heads, group, dim, page, dtype):
    check_weights(B, new, lengths, heads, group, dim, page, dtype, spare=sum(new) % 3)


@pytest.mark.parametrize("new,lengths,heads,group,dim,page,dtype", [
    ([20, 0, 3, 300], [20, 9, 3, 700], 2, 3, 96, 16, BF16),            # many rows beside few and none
    ([33] * 40, list(range(33, 73)), 1, 1, 32, 32, F16),               # one row more than 32, many sequences
    ([2, 0, 1] * 70, [5, 3, 40] * 70, 1, 4, 64, 16, BF16),             # more sequences than a wavefront counts at a time
    ([128, 129], [128, 1300], 1, 1, 128, 256, F16),
    ([1], [9000], 8, 8, 128, 16, BF16),
    ([70], [9000], 2, 1, 64, 64, BF16),                                # cut, and joined
    ([150], [100], 1, 2, 64, 16, F16),                                 # more queries than tokens
])
def test_weights_of_uneven_sequences(B, new, lengths, heads, group, dim, page, dtype):
    check_weights(B, new, lengths, heads, group, dim, page, dtype)


@pytest.mark.parametrize("new", [3, 50])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 0.3])
def test_weights_of_queries_laid_out_otherwise(B, new, scale):
    """Queries that are slices of a fused projection, at odd distances and addresses, one token for all (distance 0), heads before tokens; negative and zero scales."""
    _, filled, held = B
    g = gen(new)
    lengths, heads, group, dim, page = [210, 77], 2, 3, 64, 32
    st = filled(12, heads, page, dim, seed=5)
    tables = make_tables(g, lengths, 12, page)
    tokens, many = 2 * new, heads * group
    fused = randn(g, tokens, 3 * many, dim).to(BF16)
    odd = randn(g, tokens * (many * (dim + 1) + 3) + 1).to(F16)
    for q in (fused[:, many:2 * many], odd[1:].view(tokens, -1)[:, :many * (dim + 1)].unflatten(1, (many, dim + 1))[:, :, 1:], fused[:1, :many].expand(tokens, -1, -1),
              randn(g, many, tokens, dim).to(BF16).transpose(0, 1)):
        want, tol = E.weights(held(st), q, tables, lengths, [0, new, tokens], scale)
        R.assert_close(st.attend_weights(q, dev(tables), dev(lengths), scale=scale), want, tol, str(q.stride()))


@pytest.mark.parametrize("new,dim", [(1, 64), (40, 128), (300, 32)])
def test_weights_of_large_logits(B, new, dim):
    """Logits of 2^20 to 2^60, keys that differ by little among them: weights stay between 0 and 1 and a row's add up to 1 (900 terms of up to 2^-22 each)."""
    Store, _, _ = B
    g, n, page, heads = gen(new), 900, 64, 2
    st = Store.empty(15, heads, page, dim)
    t = torch.arange(n, device="cuda")
    for power in (20, 24, 28, 31, 34, 45, 60):
        k = torch.zeros((n, heads, dim), device="cuda")
        k[:, :, 5] = 2.0 ** (power - 10) * (1 + (t + torch.randint(0, 40, (n,), generator=g, device="cuda"))[:, None] * 2.0 ** -23)
        k[::7, :, 3] = 2.0 ** (power - 30)
        st.write(k, k, t)
        q = randn(g, new, 4 * heads, dim)
        q[:, :, 5] = 2.0 ** 10
        for scale in (1.0, -0.7):
            got = st.attend_weights(q.to(BF16), dev([list(range(15))]), dev([n]), scale=scale).double()
            assert (got >= 0).all() and (got <= 4 * new * (1 + 2.0 ** -12)).all(), (power, scale)
            assert (got.sum(2) / (4 * new) - 1).abs().max() < 2.0 ** -11, (power, scale)


@pytest.mark.parametrize("new", [2, 40])
@pytest.mark.parametrize("size", [-90, -40, 40, 90])
def test_weights_of_small_and_large_queries(B, new, size):
    """Queries of 2^size under a scale of 2^-size: logits of ordinary size."""
    _, filled, held = B
    g = gen(new)
    st = filled(12, 2, 32, 64, seed=6)
    tables = make_tables(g, [300], 12, 32)
    q = (randn(g, new, 4, 64) * 2.0 ** size).to(BF16)
    want, tol = E.weights(held(st), q, tables, [300], [0, new], 0.3 * 2.0 ** -size)
    R.assert_close(st.attend_weights(q, dev(tables), dev([300]), scale=0.3 * 2.0 ** -size), want, tol)


@pytest.mark.parametrize("new,dtype", [(3, BF16), (3, F16), (40, BF16), (300, F16)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_weights_of_queries_that_are_no_numbers(B, new, dtype, what):
    """A query that holds an infinity (its logits are infinities of both signs) or NaN makes the sums of the keys that it sees NaN, in its head; other heads, keys and sequences are as they would be."""
    _, filled, _ = B
    g = gen(new)
    lengths, page = [400, 333], 64
    st = filled(20, 2, page, 64, seed=8)
    tables = make_tables(g, lengths, 20, page)
    q = randn(g, 2 * new, 4, 64).to(dtype)
    clean = st.attend_weights(q, dev(tables), dev(lengths))
    q[new - 2, 1, 17] = what                               # the last query but one of the first sequence, head 0 of the store
    got = st.attend_weights(q, dev(tables), dev(lengths))
    assert torch.isnan(got[0, 0, :lengths[0] - 1]).all()
    got[0, 0, :lengths[0] - 1] = clean[0, 0, :lengths[0] - 1]
    assert torch.equal(got, clean)


def test_weights_sum_to_the_rows(B):
    """Many blocks of keys: every row's weights add up to 1, within the error of each (2^-20 of it)."""
    _, filled, _ = B
    st = filled(600, 4, 64, 128, seed=2)
    g = gen(5)
    for new, group in ((1, 4), (64, 4)):
        lengths = [9000, 17000, 11003]
        tables = make_tables(g, lengths, 600, 64, junk=False)
        q = randn(g, 3 * new, 4 * group, 128).to(BF16)
        got = st.attend_weights(q, dev(tables), dev(lengths)).double()
        assert (got.sum(2) / (new * group) - 1).abs().max() < 2.0 ** -14
        assert all((got[i, :, n:] == 0).all() for i, n in enumerate(lengths))


@pytest.mark.parametrize("new", [1, 40])
def test_weights_of_keys_that_are_no_numbers_or_not_there(B, new):
    Store, filled, held = B
    g = gen(new)
    n, page, dim = 300, 16, 64
    st = filled(20, 2, page, dim, seed=3)
    tables = np.arange(20, dtype=np.int32)[None].copy()
    tables[0, 4], tables[0, 7] = -1, 10 ** 6
    q = randn(g, new, 4, dim).to(BF16)
    for length in (n, new // 2, 0, 5000):
        want, tol = E.weights(held(st), q, tables, [length], [0, new], dim ** -0.5)
        R.assert_close(st.attend_weights(q, dev(tables), dev([length])), want, tol, str(length))
    k = randn(g, 1, 2, dim)
    k[0, 0, 3] = float("nan")
    slot = torch.tensor([n - 1 - min(new - 1, 3)], device="cuda")          # seen by the last four queries (or the only one)
    st.write(k, k, slot)
    got = st.attend_weights(q, dev(tables), dev([n]))
    assert not torch.isnan(got[0, 1]).any()
    bad = torch.isnan(got[0, 0])
    there = torch.zeros_like(bad)
    there[:n] = True
    there[4 * page:5 * page] = there[7 * page:8 * page] = False
    assert torch.equal(bad, there)


def test_nothing_to_weigh(B):
    _, filled, _ = B
    st = filled(4, 2, 16, 32)
    before = torch.rand((2, 2, 32), device="cuda")
    none = torch.empty((0, 4, 32), dtype=BF16, device="cuda")
    tables, lengths = dev([[0, 1], [2, 3]]), dev([20, 30])
    assert torch.equal(st.attend_weights(none, tables, lengths, before=before), before)
    assert torch.equal(st.attend_weights(none, tables, lengths, q_start=dev([0, 0, 0]), before=before), before)
    assert (st.attend_weights(none, tables, lengths) == 0).all()
    q = torch.ones((2, 4, 32), dtype=BF16, device="cuda")
    assert torch.equal(st.attend_weights(q, tables, dev([0, 0]), before=before), before)
    assert st.attend_weights(q, torch.zeros((2, 0), dtype=torch.int32, device="cuda"), lengths).shape == (2, 2, 0)


# ---- eviction ----

def check_evict(B, lengths, budget, recent, heads, dim, page, kind, holes=False, spare=0):
    _, filled, _ = B
    g, rng = gen(sum(lengths) + budget), np.random.default_rng(sum(lengths) + budget)
    need = [-(-n // page) for n in lengths]
    to_width = -(-budget // page) + spare
    pages = sum(need) + len(lengths) * to_width + 3
    st = filled(pages, heads, page, dim, seed=7)
    tables = make_tables(g, lengths, pages, page, spare=1)
    width = tables.shape[1]
    used = {int(p) for i, n in enumerate(need) for p in tables[i, :n]}
    to = np.array(rng.permutation([p for p in range(pages) if p not in used])[:len(lengths) * to_width], np.int32).reshape(len(lengths), to_width)
    if holes:
        tables[0, 1], tables[-1, 0] = -5, pages
        if to_width > 1:
            to[0, 1] = -1
    sums = rng.exponential(size=(len(lengths), heads, width * page)).astype(np.float32)
    if kind == "ties":
        sums = np.floor(2 * sums)
    elif kind == "alike":
        sums[:] = 0.25
    elif kind == "strange":
        sums = np.where(rng.random(sums.shape) < 0.3, rng.choice(np.float32([np.nan, np.inf, -np.inf, 0.0, -0.0, -1.0, 1e-42]), sums.shape), sums).astype(np.float32)
    before = arrays(st)
    kept, left, kept_sums = st.evict(dev(tables), dev(lengths), dev(sums, F32), budget, dev(to), recent=recent)
    after = arrays(st)
    kept, left, kept_sums = (x.cpu().numpy() for x in (kept, left, kept_sums))
    want = {n: a.copy() for n, a in before.items()}
    assert kept.shape == (len(lengths), heads, budget) and kept_sums.shape == (len(lengths), heads, to_width * page)
    for s, n in enumerate(lengths):
        n = min(n, width * page)
        there = np.repeat((tables[s] >= 0) & (tables[s] < pages), page)
        for h in range(heads):
            keys = np.array(E.choose(sums[s, h], there, n, budget, recent), np.int64)
            assert left[s] == len(keys)
            assert np.array_equal(kept[s, h, :len(keys)], keys) and (kept[s, h, len(keys):] == -1).all(), (s, h)
            assert np.array_equal(kept_sums[s, h, :len(keys)], sums[s, h, keys], equal_nan=True) and (kept_sums[s, h, len(keys):] == 0).all()
            r = np.arange(len(keys))
            ok = (to[s, r // page] >= 0) if len(keys) else np.zeros(0, bool)
            p, o, tp, t_o = tables[s, keys // page][ok], (keys % page)[ok], to[s, r // page][ok], (r % page)[ok]
            for name in want:
                if name == "v_codes":
                    want[name][tp, h, :, t_o] = before[name][p, h, :, o]
                else:
                    want[name][tp, h, t_o] = before[name][p, h, o]
    for name in want:
        assert np.array_equal(after[name], want[name], equal_nan=name.endswith("scales")), name


EVICTIONS = [
    # lengths, budget, recent, heads, dim, page
    ([1], 1, 0, 1, 32, 16),
    ([1, 0, 5], 3, 1, 2, 64, 16),
    ([100, 40, 64, 65], 40, 8, 3, 128, 64),
    ([300, 299, 17], 64, 64, 2, 96, 32),
    ([1000], 333, 100, 2, 128, 16),
    ([5000, 4096, 4097], 1025, 0, 1, 32, 256),
    ([20000], 3001, 77, 2, 64, 128),
    ([130, 131], 129, 128, 1, 128, 128),
    # tables of every size that one block holds, and longer ones in chunks: sequences that end in the first chunk, within one, at the border of one; that have nothing at all
    ([8000, 4000], 1000, 10, 1, 32, 32),
    ([16384, 12000], 5000, 10, 1, 32, 128),
    ([40000, 5, 0, 9000, 8192, 16384, 8193], 2500, 300, 1, 32, 64),
    ([70000], 65536, 0, 1, 32, 256),
    ([17000, 16500], 16400, 16390, 1, 32, 16),
]


@pytest.mark.parametrize("lengths,budget,recent,heads,dim,page", EVICTIONS)
@pytest.mark.parametrize("kind", ["spread", "ties", "alike", "strange"])
def test_evict(B, lengths, budget, recent, heads, dim, page, kind):
    check_evict(B, lengths, budget, recent, heads, dim, page, kind, spare=budget % 2)


@pytest.mark.parametrize("lengths,budget,recent,heads,dim,page", [([100, 40, 64, 65], 40, 8, 3, 128, 16), ([300, 299, 170], 64, 64, 2, 96, 32), ([2000, 900], 700, 100, 1, 64, 64),
                                                                  ([20000, 100], 300, 100, 1, 32, 64)])
@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_evict_around_pages_that_are_not_there(B, lengths, budget, recent, heads, dim, page, kind):
    check_evict(B, lengths, budget, recent, heads, dim, page, kind, holes=True)


def test_keep_nothing(B):
    _, filled, _ = B
    st = filled(6, 2, 16, 32)
    before = arrays(st)
    tables, lengths, sums = dev([[0, 1], [2, 3]]), dev([20, 32]), torch.rand((2, 2, 32), device="cuda")
    kept, left, kept_sums = st.evict(tables, lengths, sums, 0, dev([[4], [5]]))
    assert kept.shape == (2, 2, 0) and (left == 0).all() and (kept_sums == 0).all()
    kept, left, kept_sums = st.evict(torch.zeros((2, 0), dtype=torch.int32, device="cuda"), lengths, torch.zeros((2, 2, 0), device="cuda"), 5, dev([[4], [5]]))
    assert (kept == -1).all() and (left == 0).all() and (kept_sums == 0).all()
    assert all(np.array_equal(before[n], a, equal_nan=True) for n, a in arrays(st).items())


def test_destinations_in_host_memory_are_refused(B):
    """Also where no token is kept: the sums behind the last are written for their pages."""
    from paper_2410_18926_amd.binding import LorannError
    _, filled, _ = B
    st = filled(6, 2, 16, 32)
    tables, lengths, sums = dev([[0, 1], [2, 3]]), dev([20, 32]), torch.rand((2, 2, 32), device="cuda")
    for budget in (0, 5):
        with pytest.raises(LorannError, match="to_tables"):
            st.evict(tables, lengths, sums, budget, torch.tensor([[4], [5]], dtype=torch.int32))


def test_a_conversation_within_a_budget(B):
    """Prompt, its weights, eviction, further tokens behind what was kept, their weights, eviction again: as a decoder would, every step against the definitions."""
    Store, _, held = B
    g = gen(77)
    heads, group, dim, page, new, budget, recent = 2, 4, 128, 16, 90, 48, 16
    scale = dim ** -0.5
    st = Store.empty(64, heads, page, dim)
    free = list(range(64))
    take = lambda n: [free.pop(0) for _ in range(n)]  # noqa: E731
    lengths = [90, 70]
    width = 8
    tables = dev([take(width), take(width)])
    write = lambda s, t0, k, v: st.write(k, v, tables[s, torch.arange(t0, t0 + len(k), device="cuda") // page].long() * page + torch.arange(t0, t0 + len(k), device="cuda") % page)  # noqa: E731
    start = [0, 90, 160]
    for s, n in enumerate(lengths):
        write(s, 0, randn(g, n, heads, dim), randn(g, n, heads, dim))
    q = randn(g, 160, heads * group, dim).to(BF16)
    sums = st.attend_weights(q, tables, dev(lengths), q_start=dev(start))
    for round_ in range(3):
        want, tol = E.weights(held(st), q, tables.cpu().numpy(), lengths, start, scale, None if round_ == 0 else before)
        R.assert_close(sums, want, tol, f"round {round_}")
        R.assert_close(st.attend_chunk(q, tables, dev(lengths), q_start=dev(start)), *R.chunk(held(st), q, tables.cpu().numpy(), lengths, start, scale))
        old_tables, old = tables.cpu().numpy(), arrays(st)
        to = dev([take(width), take(width)])
        kept, left, sums_left = st.evict(tables, dev(lengths), sums, budget, to, recent=recent)
        for s, n in enumerate(lengths):
            for h in range(heads):
                keys = E.choose(sums[s, h].cpu().numpy(), np.ones(width * page, bool), n, budget, recent)
                assert kept[s, h, :len(keys)].tolist() == keys
        now = arrays(st)
        for s in range(2):
            for h in range(heads):
                keys, r = kept[s, h, :int(left[s])].cpu().numpy(), np.arange(int(left[s]))
                for name in ("k_codes", "k_scales", "v_scales"):
                    assert np.array_equal(now[name][to[s].cpu().numpy()[r // page], h, r % page], old[name][old_tables[s, keys // page], h, keys % page])
        free += tables.flatten().tolist()
        tables, lengths, sums = to, left.tolist(), sums_left
        assert lengths == [budget, budget]
        # two decoding steps: a token each
        before = sums.cpu().numpy()
        for s in range(2):
            write(s, lengths[s], randn(g, 1, heads, dim), randn(g, 1, heads, dim))
        lengths, start = [n + 1 for n in lengths], [0, 1, 2]
        q = randn(g, 2, heads * group, dim).to(BF16)
        sums = st.attend_weights(q, tables, dev(lengths), before=sums, out=sums)


def test_captured(B):
    """Weights (few rows and many) and eviction in one graph, replayed with other contents among eager work; two graphs with a workspace each."""
    _, filled, held = B
    st = filled(200, 2, 16, 64, seed=4)
    g = gen(8)
    tables, to = dev(np.arange(120).reshape(2, 60)), dev(np.arange(120, 144).reshape(2, 12))
    lengths = dev([901, 500])

    def make(new):
        q = randn(g, 2 * new, 8, 64).to(BF16)
        before = torch.rand((2, 2, 960), generator=g, device="cuda")
        sums = torch.empty_like(before)
        out = torch.empty((2, 2, 180), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty((2, 2, 192), device="cuda")
        w1 = torch.empty(max(16, st.weights_workspace_bytes(q, 2, 60)), dtype=torch.uint8, device="cuda")
        w2 = torch.empty(max(16, st.evict_workspace_bytes(2, 60)), dtype=torch.uint8, device="cuda")

        def step():
            st.attend_weights(q, tables, lengths, before=before, out=sums, workspace=w1)
            st.evict(tables, lengths, sums, 180, to, recent=20, out=out, workspace=w2)
        return q, before, sums, out, step

    both = [make(1), make(50)]
    graphs = []
    for *_, step in both:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        graphs.append(graph)
    for i in range(4):
        for graph, (q, before, sums, out, step) in zip(graphs, both):
            q.copy_(randn(g, *q.shape))
            before.copy_(torch.rand(before.shape, generator=g, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            got = [sums.clone(), *(x.clone() for x in out)]
            n = q.shape[0] // 2
            want, tol = E.weights(held(st), q, tables.cpu().numpy(), [901, 500], [0, n, 2 * n], 0.125, before.cpu().numpy())
            R.assert_close(got[0], want, tol, f"replay {i}")
            step()
            assert all(torch.equal(a, b) for a, b in zip(got, [sums, *out]))
            for s in range(2):
                assert got[1][s, 1].tolist() == E.choose(got[0][s, 1].cpu().numpy(), np.ones(960, bool), [901, 500][s], 180, 20)


def test_another_stream(B):
    _, filled, held = B
    st = filled(100, 2, 16, 64, seed=4)
    g = gen(18)
    tables, lengths = dev(np.arange(60).reshape(1, 60)), dev([901])
    for new in (1, 60):
        q = randn(g, new, 4, 64).to(F16)
        want, tol = E.weights(held(st), q, tables.cpu().numpy(), [901], [0, new], 0.125)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = st.attend_weights(q, tables, lengths)
        side.synchronize()
        R.assert_close(got, want, tol)


def test_no_gradient_through_sums(B):
    _, filled, _ = B
    st = filled(4, 2, 16, 32)
    q = torch.ones((1, 4, 32), dtype=BF16, device="cuda", requires_grad=True)
    got = st.attend_weights(q, dev([[0, 1]]), dev([20]))
    with pytest.raises(NotImplementedError, match="no gradient"):
        got.sum().backward()
