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
