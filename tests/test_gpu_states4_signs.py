"""The sign of a code in the 4-bit store is that of the value, also where the value is a zero or rounds to none of the larger magnitudes."""
import numpy as np
import pytest
import torch

import states4_reference as R4
from test_gpu_states import BF16, F16, F32, gen, randn
from test_gpu_states4 import S, check_written  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,page,tokens", [(128, 64, 100), (96, 16, 9), (32, 32, 1), (64, 16, 33)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("top", [1.0, 2.0 ** 14, 2.0 ** 126])
def test_signs_of_zeros_and_of_the_smallest(S, dim, page, tokens, dtype, top):  # noqa: F811
    if dtype == F16 and top > 2.0 ** 14:
        top = 2.0 ** -10
    g = gen(dim + tokens)
    x = (randn(g, 2, tokens, 2, dim).clamp(-1.9, 1.9) * top).to(dtype)
    pick = torch.randint(0, 4, x.shape, generator=g, device="cuda")
    tiny = torch.finfo(dtype).smallest_normal
    x = torch.where(pick == 0, torch.copysign(torch.zeros_like(x), x), torch.where(pick == 1, torch.copysign(torch.full_like(x, tiny), x), x))
    k, v = x
    k[:, 0, :32] = torch.copysign(torch.zeros_like(k[:, 0, :32]), k[:, 0, :32])          # a group of nothing else
    assert (torch.signbit(x) & (x == 0)).any()
    st = S.States4.empty(-(-tokens // page), 2, page, dim)
    before = R4.arrays(st)
    slots = torch.arange(tokens, device="cuda")
    st.write(k, v, slots)
    wk, wv, _ = check_written(st, before, k, v, slots)
    for got, want in zip(st.read(slots, F32), (wk, wv)):
        got = got.cpu().numpy()
        assert np.array_equal(got, want) and np.array_equal(np.signbit(got), np.signbit(want))
