"""What the attention's answers keep where the weights, the steps of the values and the lengths differ most.  Definitions in 64 bits, tolerances derived beside them."""
import numpy as np
import pytest
import torch

import states_reference as R

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


# ---- one key above very many that weigh next to nothing each ----

@pytest.mark.parametrize("new,group", [(2049, 32), (1, 8)])          # one piece for all keys; cut, and joined
@pytest.mark.parametrize("place", [5, 2 ** 18 + 77])
def test_very_many_small_weights(S, new, group, place):
    """2^19 keys with the value 1 in every component, one of them 20 to 26 octaves above the others: the answer is 1, whatever the weights are.

    Tolerance, relative: the answer's rounding to binary16, 2^-11; the weights' rounding, 2^-11, and 2^-34 of the largest weight for each key; sums in float - the
    numerator grows by a matrix instruction for 16 keys, taken to round twice, the divisor by a term for 64 keys (of 64 terms)."""
    n, dim, page = 2 ** 19, 64, 256
    st = S.States.empty(n // page, 1, page, dim)
    k, v = torch.zeros((n, 1, dim), device="cuda"), torch.ones((n, 1, dim), device="cuda")
    k[:, 0, 0] = -8.0
    k[place] = 0
    st.write(k, v, torch.arange(n, device="cuda"))
    octaves = torch.linspace(20.0, 26.0, group, device="cuda")
    q = torch.zeros((new, group, dim), device="cuda")
    q[:, :, 0] = octaves * np.log(2) / 8
    tables = torch.arange(st.pages, dtype=torch.int32, device="cuda")[None]
    got = st.attend_chunk(q.to(F16), tables, dev([n]), scale=1.0)
    tol = 2.0 ** -11 + 2.0 ** -11 + n * 2.0 ** -34 + (2 * n / 16 + n / 64 + 64) * 2.0 ** -24
    off = (got.double() - 1).abs().amax((0, 2))
    assert (off <= tol).all(), f"off by {off.tolist()} where {tol} is allowed, {octaves.tolist()} octaves"


# ---- keys whose values are all zero ----

def with_zero_values(S, g, lengths, heads, page, dim, size, gap, scale, zero):
    """(store, tables, direction [heads, dim]): values of about `size`; the tokens `zero(length)` of each sequence have none at all, and a logit of about `gap` for queries
    along the direction, where the others' spread by about 1."""
    width = -(-max(lengths) // page)
    st = S.States.empty(len(lengths) * width, heads, page, dim)
    tables = torch.randperm(len(lengths) * width, generator=g, device="cuda").to(torch.int32).view(len(lengths), width)
    along = randn(g, heads, dim)
    for s, n in enumerate(lengths):
        k, v = randn(g, n, heads, dim) / (scale * dim ** 0.5), size * randn(g, n, heads, dim)
        for z in zero(n):
            k[z] = gap / scale * along / (along * along).sum(-1, keepdim=True)
            v[z] = 0
        t = torch.arange(n, device="cuda")
        st.write(k, v, tables[s, t // page].long() * page + t % page)
    return st, tables, along


def queries(g, along, tokens, group, dtype):
    heads, dim = along.shape
    return (along[None, :, None] + 0.05 * randn(g, tokens, heads, group, dim)).reshape(tokens, heads * group, dim).to(dtype)


ZERO_CHUNKS = [
    # new tokens of each sequence, lengths, heads, group, dim, page, type
    (1, [256], 2, 2, 128, 64, BF16),
    (1, [300, 40], 1, 4, 64, 16, F16),
    (1, [3000], 1, 2, 32, 32, F16),                  # cut, and joined
    (70, [256, 133], 1, 2, 128, 64, F16),            # shared tiles
    (50, [200], 1, 3, 64, 16, BF16),
    (60, [1500], 1, 1, 96, 128, F16),                # shared tiles, cut, and joined
]


@pytest.mark.parametrize("new,lengths,heads,group,dim,page,dtype", ZERO_CHUNKS)
@pytest.mark.parametrize("size,gap", [(0.1, 10.0), (0.01, 0.0), (0.01, 6.0), (0.01, 10.0), (1e-3, 6.0), (1e-5, 0.0)])
@pytest.mark.parametrize("place", ["first", "middle", "many"])
def test_keys_without_values(S, new, lengths, heads, group, dim, page, dtype, size, gap, place):
    """A key whose values are all zero takes its share of the weights and changes nothing else, however much it weighs and however small the other values are."""
    if dtype == F16 and size < 1e-2:
        dtype = BF16                                 # (answers that binary16 would hold with few bits)
    zero = {"first": lambda n: [0], "middle": lambda n: [n // 2 - 5], "many": lambda n: list(range(3, n - 8, 9))}[place]
    g = gen(1000 * new + dim + int(gap))
    scale = dim ** -0.5
    st, tables, along = with_zero_values(S, g, lengths, heads, page, dim, size, gap, scale, zero)
    q = queries(g, along, new * len(lengths), group, dtype)
    want, tol = R.chunk(st, q, tables.cpu().numpy(), lengths, [i * new for i in range(len(lengths) + 1)], scale)
    if dtype == F16:
        tol = tol + 2.0 ** -25                       # half the distance of binary16's numbers below 2^-14
    R.assert_close(st.attend_chunk(q, tables, dev(lengths), scale=scale), want, tol)


@pytest.mark.parametrize("new,dim,page", [(1, 128, 64), (60, 64, 16)])
@pytest.mark.parametrize("size,gap", [(0.01, 10.0), (1e-4, 3.0)])
def test_passages_with_padding_in_the_store(S, new, dim, page, size, gap):
    """Passages whose last tokens were written as zeros (padding), one that is nothing else, and tokens of the store that were never written."""
    g = gen(7 + new)
    scale, lengths = dim ** -0.5, [100, 64, 30, 250]
    st, tables, along = with_zero_values(S, g, lengths, 1, page, dim, size, gap, scale, lambda n: range(n) if n == 30 else range(n - n // 4, n))
    blank = torch.arange(-(-50 // page), device="cuda").to(torch.int32) + st.pages          # pages at the end of a larger store, never written
    big = S.States.empty(st.pages + len(blank), 1, page, dim)
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        getattr(big, name)[:st.pages] = getattr(st, name)
    wide = torch.zeros((5, max(tables.shape[1], len(blank))), dtype=torch.int32, device="cuda")
    wide[:4, :tables.shape[1]] = tables
    wide[4, :len(blank)] = blank
    lengths = lengths + [50]
    ids = np.array([[0, 4, 2], [3, 1, -1]])
    scores = np.array([[0.5, 0.1, 0.0], [0.2, 0.3, 0.0]], np.float32)
    q = queries(g, along, 2 * new, 4, BF16)
    want, tol = R.passages(big, q, ids, wide.cpu().numpy(), lengths, [0, new, 2 * new], scores, -1.5, scale)
    got = big.attend_passages(q, dev(ids, torch.int64), wide, dev(lengths), scores=dev(scores, torch.float32), score_weight=-1.5, scale=scale)
    R.assert_close(got, want, tol)


@pytest.mark.parametrize("new", [1, 80])
@pytest.mark.parametrize("size", [1e-8, 1e-14, 1e-20, 1e-28])
def test_keys_without_values_among_the_smallest(S, new, size):
    """The same where the other values are far below what models have: the first tiles hold keys without values alone, or tame values, the later ones tiny values."""
    g = gen(21)
    scale, dim, n = 0.125, 64, 700
    for head in ("zeros", "tame"):
        st = S.States.empty(-(-n // 16), 1, 16, dim)
        k, v = randn(g, n, 1, dim), size * randn(g, n, 1, dim)
        v[:130] = 0
        if head == "tame":
            v[20:60], k[20:60] = 1e-6 * randn(g, 40, 1, dim), 0.01 * k[20:60]
        v[300:310] = 0
        st.write(k, v, torch.arange(n, device="cuda"))
        q = randn(g, new, 2, dim).to(BF16)
        tables = torch.arange(st.pages, dtype=torch.int32, device="cuda")[None]
        want, tol = R.chunk(st, q, tables.cpu().numpy(), [n], [0, new], scale)
        R.assert_close(st.attend_chunk(q, tables, dev([n]), scale=scale), want, tol, head)


@pytest.mark.parametrize("new", [1, 100])
def test_nothing_but_zero_values(S, new):
    """An answer of zeros from 40000 keys without values; with one value among them, its share."""
    n, dim = 40_000, 32
    st = S.States.empty(n // 64, 1, 64, dim)
    tables = torch.arange(st.pages, dtype=torch.int32, device="cuda")[None]
    q = randn(gen(5), new, 2, dim).to(BF16)
    assert (st.attend_chunk(q, tables, dev([n])) == 0).all()
    one = torch.full((1, 1, dim), 3.0, device="cuda")
    st.write(0 * one, one, torch.tensor([n - 500], device="cuda"))
    want = 3.0 / (n - new + 1 + torch.arange(new, dtype=torch.float64, device="cuda"))           # (every logit is 0)
    got = st.attend_chunk(q, tables, dev([n])).double()
    # the answer's rounding, and sums of 40000 terms in float of which each adds the same: at most n 2^-24 relative
    tol = (2.0 ** -8 + n * 2.0 ** -24) * want
    assert ((got - want[:, None, None]).abs() <= tol[:, None, None]).all()


# ---- terms of the passages that are large against their differences ----

@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("level,weight", [(1e5, -1.0), (3e6, -0.25), (-2e5, 3.0)])
def test_large_scores_with_small_differences(S, new, dtype, level, weight):
    """Distances of 10^5 that differ by a few: only their differences count.  Tolerance: as in states_reference for the differences from the largest term (the scores'
    own differences are exact in 64 bits and within 2^-24 in float)."""
    g, rng = gen(91), np.random.default_rng(17)
    heads, group, dim, page, lengths = 2, 4, 64, 16, [130, 64, 300, 17, 1, 90]
    width = -(-max(lengths) // page)
    st = S.States.empty(len(lengths) * width, heads, page, dim)
    n = st.pages * page
    st.write(randn(g, n, heads, dim), randn(g, n, heads, dim), torch.arange(n, device="cuda"))
    tables = np.arange(len(lengths) * width, dtype=np.int32).reshape(len(lengths), width)
    found = 40
    ids = rng.integers(0, len(lengths), (2, found))
    ids[0, 5], ids[1, 30] = -1, 100
    scores = (level + rng.choice([0.0, 0.5, 1.0, 1.75, 3.0], (2, found))).astype(np.float32)
    scores[0, 5] = np.float32(-10 * level)                       # (of no passage)
    if level > 0:
        scores[1, 7] = np.inf                                    # left out
    q = randn(g, 2 * new, heads * group, dim).to(dtype)
    live = np.where((ids >= 0) & (ids < len(lengths)), weight * scores.astype(np.float64), -np.inf)
    differences = np.maximum(live - live.max(1, keepdims=True), -1e30) / weight          # what is left when the largest term is taken off: the same softmax
    differences = np.where(np.isneginf(live), -np.sign(weight) * np.inf, differences)
    want, tol = R.passages(st, q, ids, tables, lengths, [0, new, 2 * new], differences, weight, 0.125)
    args = dict(scores=dev(scores, torch.float32), score_weight=weight, scale=0.125)
    R.assert_close(st.attend_passages(q, dev(ids, torch.int64), dev(tables), dev(lengths), **args), want, tol)
