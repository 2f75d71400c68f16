"""Queries whose logits are all -infinity weigh nothing; a single +infinity makes the keys that the query sees NaN: attention and weights, few rows and many, both stores."""
import numpy as np
import pytest
import torch

import evict_reference as E
import states_reference as R
from test_gpu_evict import B  # noqa: F401
from test_gpu_states import BF16, F16, dev, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,dtype", [(1, BF16), (3, F16), (40, BF16), (300, F16)])
@pytest.mark.parametrize("at", [0, "middle"])
@pytest.mark.parametrize("sign", [-1, 1])
def test_one_sign_alone(B, new, dtype, at, sign):  # noqa: F811
    Store, _, held = B
    g = gen(new)
    at = 0 if at == 0 else new // 2
    page, dim, heads = 16, 64, 2
    st = Store.empty(-(-new // page), heads, page, dim)
    k, v = randn(g, new, heads, dim), randn(g, new, heads, dim)
    k[:, :, 5] = 2 + k[:, :, 5].abs()
    st.write(k, v, torch.arange(new, device="cuda"))
    tables = np.arange(st.pages, dtype=np.int32)[None]
    q = randn(g, new, 2 * heads, dim).to(dtype)
    args = dev(tables), dev([new])
    clean = st.attend_chunk(q, *args)
    q[at, 1, 5] = sign * float("inf")                    # query head 1: head 0 of the store
    got, sums = st.attend_chunk(q, *args), st.attend_weights(q, *args)
    # the sums without that row: those of the rows before and behind it, each over the keys that it sees, and of its other query heads
    want, tol = np.zeros((1, heads, st.pages * page)), np.zeros((1, heads, st.pages * page))
    for head in range(2 * heads):
        for lo, hi in ((0, at), (at, at + 1), (at + 1, new)):
            if hi > lo and not (lo == at and hi == at + 1 and head == 1):
                one, more = E.weights(held(st), q[lo:hi, head:head + 1].repeat(1, heads, 1), tables, [hi], [0, hi - lo], dim ** -0.5)
                want[:, head // 2] += one[:, head // 2]
                tol[:, head // 2] += more[:, head // 2]
    tol += 2 * new * 2.0 ** -24 * want
    if sign > 0:
        assert torch.isnan(got[at, 1]).all() and torch.isnan(sums[0, 0, :at + 1]).all()
        want[0, 0, :at + 1] = np.nan
        got[at, 1] = 0
    R.assert_close(sums, want, tol)
    assert (got[at, 1] == 0).all()
    got[at, 1] = clean[at, 1]
    assert torch.equal(got, clean)
