"""Sums of weights where (keys behind a sequence's length) x (query heads of a head) passes 32 bits: tables far longer than the sequences, many query heads on one."""
import numpy as np
import pytest
import torch

import evict_reference as E
import states_reference as R
from test_gpu_evict import B  # noqa: F401
from test_gpu_states import BF16, dev, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group,width,page", [(1024, 2 ** 14, 256), (1024, 2 ** 14 + 2 ** 13, 256), (512, 2 ** 17 + 7, 64)])
@pytest.mark.parametrize("new", [1, 2])
def test_short_sequences_in_very_long_tables(B, group, width, page, new):  # noqa: F811
    """The sums of the keys that are there are those of the definition; all others keep what was there before."""
    _, filled, held = B
    g = gen(group + new)
    lengths, used = [300, 1, 700], 4 * 256 // page
    assert (width * page - 1000) * group > 2 ** 31
    st = filled(3 * used, 1, page, 32, seed=3)
    tables = np.full((3, width), 10 ** 6, np.int32)
    tables[:, :used] = np.arange(3 * used).reshape(3, used)
    q = randn(g, 3 * new, group, 32).to(BF16)
    three = np.full((3, 1, used * page), 3.0)
    (want, tol), (more, tol3) = (E.weights(held(st), q, tables[:, :used], lengths, [i * new for i in range(4)], 0.2, b) for b in (None, three))
    tables = dev(tables)
    for start in (None, dev([i * new for i in range(4)])):
        got = st.attend_weights(q, tables, dev(lengths), q_start=start, scale=0.2)
        R.assert_close(got[:, :, :1024], want, tol)
        assert (got[:, :, 1024:] == 0).all()
        before = torch.full_like(got, 3.0)
        got = st.attend_weights(q, tables, dev(lengths), q_start=start, scale=0.2, before=before)
        assert (got[:, :, 1024:] == 3).all()
        R.assert_close(got[:, :, :1024], more, tol3)
