"""The example that searches and then reads what it found, against the same layer computed plainly in float from the values that the store gives back."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def plain_attention(q, k, v, seen, bias):
    """q [tokens, heads, group, dim], k, v [keys, heads, dim], seen [tokens, keys], bias [keys]: float on the CPU."""
    out = torch.zeros_like(q)
    for h in range(q.shape[1]):
        for g in range(q.shape[2]):
            a = q[:, h, g] @ k[:, h].T * q.shape[3] ** -0.5 + bias
            out[:, h, g] = torch.softmax(a.masked_fill(~seen, float("-inf")), 1) @ v[:, h]
    return out


def test_answer_reads_what_the_search_found():
    """Ids are the search's own; the hidden states are those of the plain layer.  Tolerance: the layer rounds four times to bfloat16 (2^-9 each on average, 2^-8 at most, of
    values of the size of the hidden states, through products of 48 to 256 terms with weights of unit gain), and tokens build on each other: 8 steps x 4 x 2^-8
    of the largest value."""
    from paper_2410_18926_amd.answer import answer, small_setup
    index, reader, questions, embed = small_setup(seed=3)
    ids, hidden = answer(index, reader, questions, embed, steps=3)
    want_ids, dists = index.search(embed(questions.mean(1)).float().contiguous(), 4, 8, 50)
    assert torch.equal(ids, want_ids) and (ids >= 0).all()
    st, heads, group, dim = reader.states, reader.heads, reader.group, reader.dim
    k_all, v_all = (x.cpu() for x in st.read(torch.arange(st.pages * st.page_size, device="cuda"), torch.float32))
    W = {n: getattr(reader, n).float().cpu() for n in ("q", "o", "cross_q", "cross_o")}
    n, total, width = hidden.shape
    new0 = questions.shape[1]
    rows = [torch.arange(new0)] + [torch.tensor([t]) for t in range(new0, total)]
    P = st.page_size
    for c in range(n):
        own = reader.own[c].long().cpu()
        slot = lambda t: own[t // P] * P + t % P  # noqa: E731
        found = [(int(i), float(d)) for i, d in zip(ids[c], dists[c])]
        pk, pv, pb = [], [], []
        for i, d in found:
            t = torch.arange(int(reader.lengths[i]))
            s = reader.tables[i].long().cpu()[t // P] * P + t % P
            pk.append(k_all[s]); pv.append(v_all[s]); pb.append(torch.full((len(t),), -d))
        pk, pv, pb = torch.cat(pk), torch.cat(pv), torch.cat(pb)
        for t in rows:
            x = questions[c].float().cpu() if len(t) > 1 else hidden[c, t - 1].float().cpu()
            keys = torch.arange(int(t[-1]) + 1)
            q = (x @ W["q"]).view(len(t), heads, group, dim)
            x = x + plain_attention(q, k_all[slot(keys)], v_all[slot(keys)], keys[None, :] <= t[:, None], torch.zeros(len(keys))).reshape(len(t), -1) @ W["o"]
            q = (x @ W["cross_q"]).view(len(t), heads, group, dim)
            x = x + plain_attention(q, pk, pv, torch.ones(len(t), len(pk), dtype=torch.bool), pb).reshape(len(t), -1) @ W["cross_o"]
            got = hidden[c, t].float().cpu()
            assert np.abs((got - x).numpy()).max() <= 8 * 4 * 2.0 ** -8 * float(x.abs().max()), (c, t)
    index.close()
