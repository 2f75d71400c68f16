"""Sums of weights of very many rows whose keys are cut and joined: more rows and heads than one dimension of the join's grid takes."""
import numpy as np
import pytest
import torch

import evict_reference as E
import states_reference as R
from test_gpu_evict import B  # noqa: F401
from test_gpu_states import BF16, dev, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,sequences,heads,group", [(2100, 1, 2, 64), (50, 60, 8, 8)])
def test_many_rows_over_cut_tables(B, new, sequences, heads, group):  # noqa: F811
    """Queries of which few differ: the definition is formed once for each of them.  Tables wide enough to be cut, of which the sequences use little."""
    _, filled, held = B
    page, dim, width = 256, 32, 160
    assert heads * sequences * new * group / 32 > 4096 and width * page > 32768
    st = filled(5, heads, page, dim, seed=4)
    tables = np.full((sequences, width), 10 ** 6, np.int32)
    tables[:, :5] = np.arange(5)
    g = gen(new)
    base = randn(g, 1, heads * group, dim).to(BF16)
    base[:, group // 2:group] = base[:, :group - group // 2]
    lengths = [1200 - 3 * s for s in range(sequences)]
    got = st.attend_weights(base.expand(sequences * new, -1, -1), dev(tables), dev(lengths), scale=0.3)
    # the newest queries see one key more each: by the definition, query by query, over the keys that are there
    for s in (0, sequences - 1):
        rows = min(new, lengths[s])
        want = np.zeros((heads, 5 * page))
        kc, ks = held(st).k_codes.double(), held(st).k_scales.double()
        k = (kc * ks[..., None]).permute(1, 0, 2, 3).reshape(heads, 5 * page, dim)[:, :lengths[s]]
        z = 0.3 * torch.einsum("hgd,hkd->hgk", base[0].view(heads, group, dim).double(), k)
        e = torch.exp(z - z.amax(-1, keepdim=True))
        upto = e.cumsum(-1)
        for i in range(rows):
            n = lengths[s] - i
            want[:, :n] += (e[:, :, :n] / upto[:, :, n - 1:n]).sum(1).cpu().numpy()
        size = 0.3 * torch.einsum("hgd,hkd->hgk", base[0].view(heads, group, dim).double().abs(), k.abs()).amax()
        logit = (dim + 8) * 2.0 ** -24 * float(size) + 2.0 ** -21 * (float(z.abs().max()) / np.log(2) + 8)
        tol = (2 * logit + 2.0 ** -21 + 2 * lengths[s] * 2.0 ** -24 + (rows * group + 2) * 2.0 ** -24) * want + rows * group * 2.0 ** -126          # (evict_reference's, row by row)
        R.assert_close(got[s, :, :5 * page], want, tol, str(s))
        assert (got[s, :, lengths[s]:] == 0).all()
