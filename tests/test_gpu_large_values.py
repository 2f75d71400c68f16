"""Attention over very large values: a row's sum of weights is right whatever the values' steps are."""
import numpy as np
import pytest
import torch

import states_reference as R
from test_gpu_evict import B  # noqa: F401
from test_gpu_states import BF16, dev, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,n,dim,page", [(1, 300, 128, 64), (3, 300, 64, 16), (1, 4000, 64, 64), (20, 300, 96, 32), (60, 500, 128, 64), (70, 300, 64, 16), (70, 3000, 32, 128)])
@pytest.mark.parametrize("power", [60, 90, 104, 112, 120, 126])
@pytest.mark.parametrize("what", ["all", "later", "some", "first"])
def test_values_up_to_the_largest(B, new, n, dim, page, power, what):  # noqa: F811
    """Values of up to 2^(power + 1): all of them, those of the later keys, one key in five, the first ones, the others of ordinary size; single keys without values among them."""
    Store, _, held = B
    g = gen(new + power)
    st = Store.empty(-(-n // page), 1, page, dim)
    k, v = randn(g, n, 1, dim), randn(g, n, 1, dim).clamp(-1.9, 1.9)
    large = {"all": slice(None), "later": slice(n // 2, None), "some": slice(2, None, 5), "first": slice(0, 70)}[what]
    v[large] *= 2.0 ** power
    v[11::50] = 0
    st.write(k, v, torch.arange(n, device="cuda"))
    tables = np.arange(st.pages, dtype=np.int32)[None]
    q = randn(g, new, 2, dim).to(BF16)
    want, tol = R.chunk(held(st), q, tables, [n], [0, new], dim ** -0.5)
    R.assert_close(st.attend_chunk(q, dev(tables), dev([n])), want, tol, "chunk")
    want, tol = R.passages(held(st), q, np.array([[0]]), tables, [n], [0, new], None, 0.0, dim ** -0.5)
    R.assert_close(st.attend_passages(q, dev([[0]], torch.int64), dev(tables), dev([n])), want, tol, "passages")
