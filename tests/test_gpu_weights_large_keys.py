"""Sums of weights where keys are very large or very small and queries and scale the other way round: logits of ordinary size, however many rows a call has."""
import numpy as np
import pytest
import torch

import evict_reference as E
import states_reference as R
from test_gpu_evict import B  # noqa: F401
from test_gpu_states import BF16, dev, gen, make_tables, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [2, 40, 300])
@pytest.mark.parametrize("keys,queries", [(123, -99), (110, -100), (110, -60), (100, -100), (-97, 100), (-90, 120), (60, -60)])
@pytest.mark.parametrize("mixed", [False, True])
def test_weights_of_large_and_small_keys(B, new, keys, queries, mixed):  # noqa: F811
    """Keys of 2^keys, queries of 2^queries, a scale that makes their logits ordinary; mixed: beside keys of ordinary size and tiny ones, whose logits are next to nothing or far away."""
    Store, _, held = B
    g = gen(new + keys)
    n, page, dim = 400, 32, 64
    st = Store.empty(n // page + 2, 2, page, dim)
    k = randn(g, n, 2, dim).clamp(-3, 3).double() * 2.0 ** keys
    if mixed:
        k[::3] = randn(g, *k[::3].shape).double() * 2.0 ** min(keys - 5, 0)
        k[1::7] *= 2.0 ** max(-98 - keys, -3)
    slots = torch.arange(n, device="cuda")
    st.write(k.float(), k.float() * 0, slots)
    tables = np.arange(st.pages, dtype=np.int32)[None]
    q = (randn(g, new, 4, dim).double() * 2.0 ** queries).to(BF16)
    scale = 0.3 * 2.0 ** -(keys + queries)
    want, tol = E.weights(held(st), q, tables, [n], [0, new], scale)
    assert np.isfinite(want).all()
    R.assert_close(st.attend_weights(q, dev(tables), dev([n]), scale=scale), want, tol)
