"""The example over 4-bit states and with conversations kept within a budget: every call of the store that its steps make against the definition on what it was given, and its pages."""
import numpy as np
import pytest
import torch

import evict_reference as E
import states4_reference as R4
import states_reference as R

pytestmark = pytest.mark.gpu


class Recorder:
    """The store, noting what it is asked and what it answers."""

    def __init__(self, st):
        self.st, self.calls = st, []
        self.held = (lambda: R4.held(st)) if hasattr(st, "k_factors") else (lambda: st)

    def write(self, k, v, slots):
        self.st.write(k, v, slots)

    def attend_chunk(self, q, tables, lengths):
        out = self.st.attend_chunk(q, tables, lengths)
        new = q.shape[0] // tables.shape[0]
        start = [new * i for i in range(tables.shape[0] + 1)]
        want, tol = R.chunk(self.held(), q, tables.cpu().numpy(), lengths.tolist(), start, q.shape[2] ** -0.5)
        R.assert_close(out, want, tol, f"call {len(self.calls)}")
        self.calls.append(("chunk", lengths.tolist()))
        return out

    def attend_passages(self, q, ids, tables, lengths, scores, score_weight):
        out = self.st.attend_passages(q, ids, tables, lengths, scores=scores, score_weight=score_weight)
        new = q.shape[0] // ids.shape[0]
        start = [new * i for i in range(ids.shape[0] + 1)]
        want, tol = R.passages(self.held(), q, ids.cpu().numpy(), tables.cpu().numpy(), lengths.tolist(), start, scores.cpu().numpy(), score_weight, q.shape[2] ** -0.5)
        R.assert_close(out, want, tol, f"call {len(self.calls)}")
        self.calls.append(("passages", None))
        return out

    def attend_weights(self, q, tables, lengths, before, out):
        assert out is before
        was, new = before.cpu().numpy(), q.shape[0] // tables.shape[0]
        start = [new * i for i in range(tables.shape[0] + 1)]
        want, tol = E.weights(self.held(), q, tables.cpu().numpy(), lengths.tolist(), start, q.shape[2] ** -0.5, was)
        self.st.attend_weights(q, tables, lengths, before=before, out=out)
        R.assert_close(out, want, tol, f"call {len(self.calls)}")
        self.calls.append(("weights", None))

    def evict(self, tables, lengths, sums, budget, to, recent):
        kept, left, kept_sums = self.st.evict(tables, lengths, sums, budget, to, recent=recent)
        assert not set(tables.flatten().tolist()) & set(to.flatten().tolist())
        there = np.ones(sums.shape[2], bool)
        for s, n in enumerate(lengths.tolist()):
            for h in range(sums.shape[1]):
                assert kept[s, h].tolist() == E.choose(sums[s, h].cpu().numpy(), there, n, budget, recent)
        assert (left == budget).all()
        self.calls.append(("evict", (lengths.tolist(), kept)))
        return kept, left, kept_sums


@pytest.mark.parametrize("bits", [8, 4])
def test_every_call_of_a_conversation_within_a_budget(bits):
    from paper_2410_18926_amd.answer import answer, small_setup
    index, reader, questions, embed = small_setup(seed=21, bits=bits, budget=12, recent=4)
    pages = len(reader.pages.free)
    reader.states = recorder = Recorder(reader.states)
    steps = 40
    ids, hidden = answer(index, reader, questions, embed, steps=steps)
    assert hidden.shape == (3, questions.shape[1] + steps, reader.width) and torch.isfinite(hidden.float()).all()
    names = [c[0] for c in recorder.calls]
    assert [n for n in names if n != "evict"] == ["chunk", "weights", "passages"] * (steps + 1)
    # 28 tokens at a time: the 29th cuts to 12, and so does every 17th after it
    assert names.count("evict") == 1 + (questions.shape[1] + steps - 29) // 16
    assert max(c[1][0] for c in recorder.calls if c[0] == "chunk") == 28
    assert len(reader.pages.free) + len(reader.taken) == pages and not set(reader.pages.free) & set(reader.taken)
    index.close()


@pytest.mark.parametrize("bits", [8, 4])
def test_a_budget_that_is_never_reached_changes_nothing(bits):
    from paper_2410_18926_amd.answer import answer, small_setup
    index, reader, questions, embed = small_setup(seed=4, bits=bits)
    ids, want = answer(index, reader, questions, embed, steps=6)
    index.close()
    index, reader, questions, embed = small_setup(seed=4, bits=bits, budget=200)
    again, got = answer(index, reader, questions, embed, steps=6)
    assert torch.equal(ids, again) and torch.equal(want, got)
    index.close()


def test_four_bits_read_the_passages_nearly_as_eight_do():
    """The same weights and passages: what the layer answers to the question differs by the states' rounding alone.  A value is off by at most a sixth of its group's largest (half the widest step, 1 of 6),
    one of 8 bits by 1 / 254: hidden states agree to half their size at the very least, and they do differ."""
    from paper_2410_18926_amd.answer import answer, small_setup
    out = []
    for bits in (8, 4):
        index, reader, questions, embed = small_setup(seed=9, bits=bits)
        out.append(answer(index, reader, questions, embed, steps=0)[1].float())
        index.close()
    off = float((out[0] - out[1]).norm() / out[0].norm())
    assert 0 < off < 0.5


def test_arguments_that_are_refused():
    from paper_2410_18926_amd.answer import Reader
    passages = [torch.randn(5, 48)]
    for bad in (dict(bits=3), dict(budget=0), dict(budget=4, recent=5), dict(budget=4, recent=-1)):
        with pytest.raises(ValueError):
            Reader(passages, **bad)
