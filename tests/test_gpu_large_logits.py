"""Logits of 2^23 to 2^30, whose neighbours lie 1 to 64 apart: the answer stays a mean of the values that the queries see, in every kernel of both stores' attentions."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,dim,page", [(1, 128, 64), (3, 64, 16), (40, 64, 64), (70, 96, 32), (300, 128, 64), (600, 128, 64)])
@pytest.mark.parametrize("sign", [1, -1])
def test_answers_stay_within_the_values(bits, new, dim, page, sign):
    """Keys and queries of one component: logits of the same size, a few of a float's steps apart, growing along the sequence.  A mean of values v is at most max |v|, and the answer's rounding and that of
    its weights add 2^-8 and 2^-11 of it."""
    from paper_2410_18926_amd import states, states4
    Store = states.States if bits == 8 else states4.States4
    heads = 8 if new == 600 else 1
    g = torch.Generator(device="cuda")
    g.manual_seed(new)
    n = 900
    st = Store.empty(-(-n // page), heads, page, dim)
    t = torch.arange(n, device="cuda")
    v = torch.randn((n, heads, dim), generator=g, device="cuda")
    for power in range(23, 31):
        k = torch.zeros((n, heads, dim), device="cuda")
        k[:, :, 5] = sign * 2.0 ** (power - 10) * (1 + (t + torch.randint(0, 40, (n,), generator=g, device="cuda"))[:, None] * 2.0 ** -23)
        st.write(k, v, t)
        q = torch.zeros((new, 4 * heads, dim), device="cuda")
        q[:, :, 5] = 2.0 ** 10
        values = st.read(t, torch.float32)[1]
        for scale in (1.0, 0.7):
            out = st.attend_chunk(q.bfloat16(), torch.arange(st.pages, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda"), scale=scale)
            most = values.abs().amax(0).repeat_interleave(4, 0) * (1 + 2.0 ** -8 + 2.0 ** -11)
            assert not torch.isnan(out).any() and (out.float().abs() <= most).all(), (power, scale)
            assert (out.float().abs().amax((0, 2)) > 0.01).all()
