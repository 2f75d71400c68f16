"""Rows of the 4-bit store whose largest value has a reciprocal below the normal floats (above 2^126): codes, factors and steps are those of the definition bit for bit."""
import numpy as np
import pytest
import torch

import states4_reference as R4
from test_gpu_states import BF16, F32, gen, randn
from test_gpu_states4 import S, check_written  # noqa: F401

pytestmark = pytest.mark.gpu

LARGEST = {F32: float(torch.finfo(F32).max), BF16: float(torch.finfo(BF16).max)}


@pytest.mark.parametrize("dim,page,tokens", [(128, 64, 100), (96, 16, 40), (32, 32, 9), (64, 16, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("top", [2.0 ** 100, 2.0 ** 125, 2.0 ** 126, 2.0 ** 126 * (1 + 2.0 ** -7), 1e38, 2.0 ** 127, 3e38, "largest"])
def test_rows_up_to_the_largest_number(S, dim, page, tokens, dtype, top):  # noqa: F811
    g = gen(dim + tokens)
    top = LARGEST[dtype] if top == "largest" else top
    x = randn(g, 2, tokens, 2, dim).double()
    # groups of every size that a factor tells apart, and smaller ones; one value of each row is the largest itself
    size = torch.exp2(-15 * torch.rand((2, tokens, 2, dim // 32, 1), generator=g, device="cuda")).double()
    size[:, :, :, 0] = 1
    x = (x.unflatten(-1, (-1, 32)) * size).flatten(-2)
    x = x / x.abs().amax(-1, keepdim=True)
    k, v = (x * top).to(dtype)
    assert torch.isfinite(k).all() and torch.isfinite(v).all()
    st = S.States4.empty(-(-tokens // page) + 1, 2, page, dim)
    before = R4.arrays(st)
    slots = torch.arange(tokens, device="cuda") + 1
    st.write(k, v, slots)
    with np.errstate(over="ignore"):          # (a float's sixth times 6 may round to more than the largest)
        wk, wv, _ = check_written(st, before, k, v, slots)
    for out_type in (F32, BF16):
        for got, want in zip(st.read(slots, out_type), (wk, wv)):
            assert np.array_equal(got.float().cpu().numpy(), torch.from_numpy(want).to(out_type).float().numpy()), out_type
