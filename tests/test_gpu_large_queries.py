"""Attention of very large queries to small keys (and the other way round): logits of ordinary size, in every kernel of both stores' attentions and of the weights."""
import numpy as np
import pytest
import torch

import evict_reference as E
import states_reference as R
from test_gpu_evict import B  # noqa: F401
from test_gpu_states import BF16, dev, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,group,dim,page", [(1, 4, 128, 64), (3, 2, 64, 16), (20, 2, 96, 32), (60, 2, 128, 64), (70, 2, 64, 16)])
@pytest.mark.parametrize("queries,keys", [(124, -96), (118, -90), (-98, 122), (100, -40)])
def test_large_and_small_queries(B, new, group, dim, page, queries, keys):  # noqa: F811
    Store, _, held = B
    g = gen(new + queries)
    n = 300
    st = Store.empty(-(-n // page), 2, page, dim)
    k, v = randn(g, n, 2, dim).clamp(-3, 3).double() * 2.0 ** keys, randn(g, n, 2, dim)
    st.write(k.float(), v, torch.arange(n, device="cuda"))
    tables = np.arange(st.pages, dtype=np.int32)[None]
    q = (randn(g, new, 2 * group, dim).clamp(-3, 3).double() * 2.0 ** queries).to(BF16)
    scale = 0.2 * 2.0 ** -(keys + queries)
    want, tol = R.chunk(held(st), q, tables, [n], [0, new], scale)
    R.assert_close(st.attend_chunk(q, dev(tables), dev([n]), scale=scale), want, tol, "chunk")
    want, tol = R.passages(held(st), q, np.array([[0]]), tables, [n], [0, new], None, 0.0, scale)
    R.assert_close(st.attend_passages(q, dev([[0]], torch.int64), dev(tables), dev([n]), scale=scale), want, tol, "passages")
    want, tol = E.weights(held(st), q, tables, [n], [0, new], scale)
    R.assert_close(st.attend_weights(q, dev(tables), dev([n]), scale=scale), want, tol, "weights")
