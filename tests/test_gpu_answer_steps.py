"""The example, operation by operation: every call of the store and of its attentions that a step makes is compared with the definition on what it was given, every product in between
with the exact one, and the passages' answers are shown to need the search's distances."""
import numpy as np
import pytest
import torch

import states_reference as R

pytestmark = pytest.mark.gpu


def product_close(got, x, w, plus=None):
    """got [n, m] bfloat16 = plus + x @ w, the product rounded once and its sum with `plus` once more: 2^-8 of each, and float sums of the terms."""
    exact, size = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    tol = 2.0 ** -8 * exact.abs() + x.shape[1] * 2.0 ** -24 * size
    if plus is not None:
        exact = exact + plus.double()
        tol = tol + 2.0 ** -8 * (exact.abs() + tol)
    off = (got.double() - exact).abs()
    assert (off <= tol).all(), float((off - tol).max())


def test_every_operation_of_every_step():
    from paper_2410_18926_amd.answer import answer, small_setup
    index, reader, questions, embed = small_setup(seed=11)
    st, calls = reader.states, []

    class Recorder:
        """The store, noting what it is asked and what it answers."""

        def write(self, k, v, slots):
            calls.append(("write", k.clone(), v.clone(), slots.clone()))
            st.write(k, v, slots)

        def attend_chunk(self, q, tables, lengths, **more):
            out = st.attend_chunk(q, tables, lengths, **more)
            calls.append(("chunk", q.clone(), tables.clone(), lengths.clone(), more, out.clone()))
            return out

        def attend_passages(self, q, ids, tables, lengths, **more):
            out = st.attend_passages(q, ids, tables, lengths, **more)
            calls.append(("passages", q.clone(), ids.clone(), tables, lengths, more, out.clone()))
            return out

    reader.states = Recorder()
    steps = 4
    ids, hidden = answer(index, reader, questions, embed, steps=steps)
    want_ids, dists = index.search(embed(questions.mean(1)).float().contiguous(), 4, 8, 50)
    assert torch.equal(ids, want_ids) and (ids >= 0).all()
    assert [c[0] for c in calls] == ["write", "chunk", "passages"] * (steps + 1)
    H, G, D, P = reader.heads, reader.group, reader.dim, reader.page_size
    n, tokens = questions.shape[:2]
    past, decided = 0, 0
    for step in range(steps + 1):
        (_, k, v, slots), (_, q, tables, lengths, more, a), (_, q2, asked, stock, stock_lengths, more2, found) = calls[3 * step:3 * step + 3]
        new = tokens if step == 0 else 1
        x = (questions if step == 0 else hidden[:, past - 1:past]).reshape(n * new, -1)
        at = torch.arange(past, past + new, device="cuda")
        past += new
        assert torch.equal(slots.view(n, new), reader.own[:, at // P].long() * P + at % P)
        kv = torch.cat([k, v], 1).reshape(n * new, -1)
        product_close(kv, x, reader.kv)
        product_close(q.reshape(n * new, -1), x, reader.q)
        assert torch.equal(tables, reader.own) and lengths.tolist() == [past] * n and not more
        start = [i * new for i in range(n + 1)]
        want, tol = R.chunk(st, q, tables.cpu().numpy(), [past] * n, start, D ** -0.5)
        R.assert_close(a, want, tol, f"step {step}, own tokens")
        x = x + a.reshape(n * new, -1) @ reader.o
        product_close(x, a.reshape(n * new, -1), reader.o, (questions if step == 0 else hidden[:, past - 2:past - 1]).reshape(n * new, -1))
        product_close(q2.reshape(n * new, -1), x, reader.cross_q)
        assert torch.equal(asked, ids) and more2.pop("score_weight") == -1.0 and torch.equal(more2.pop("scores"), dists) and not more2
        arrays = (st, q2, ids.cpu().numpy(), stock.cpu().numpy(), stock_lengths.tolist(), start)
        want, tol = R.passages(*arrays, dists.cpu().numpy(), -1.0, D ** -0.5)
        R.assert_close(found, want, tol, f"step {step}, passages")
        without, tol0 = R.passages(*arrays, None, 0.0, D ** -0.5)
        decided += int((np.abs(found.double().cpu().numpy() - without) > tol + tol0).sum())
        product_close(hidden[:, past - new:past].reshape(n * new, -1), found.reshape(n * new, -1), reader.cross_o, x)
    assert decided > 0.5 * (steps + tokens) * n * H * G * D, "answers without the distances would pass as well"
    index.close()
