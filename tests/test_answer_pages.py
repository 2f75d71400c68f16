"""The example's pages: a reader answers as often as it is asked, a conversation's pages go back when the next one starts."""
import pytest
import torch


def reader_of(pages, page_size):
    """A reader's page-keeping alone (the rest needs the GPU)."""
    from paper_2410_18926_amd.answer import PageAllocator, Reader
    r = Reader.__new__(Reader)
    r.pages, r.taken, r.page_size, r.device = PageAllocator(pages), [], page_size, "cpu"
    return r


def test_pages_go_back_when_the_next_conversations_start():
    r = reader_of(10, 16)
    kept = r.pages.take(2)                        # (the passages' pages)
    for conversations, tokens in [(2, 64), (4, 17), (1, 128), (8, 16), (2, 33)] * 7:
        r.start(conversations, tokens)
        own = r.own.reshape(-1).tolist()
        assert r.own.shape == (conversations, -(-tokens // 16)) and len(set(own)) == len(own) and not set(own) & set(kept)
        assert sorted(own + r.pages.free + kept) == list(range(10))


def test_conversations_that_do_not_fit():
    r = reader_of(4, 16)
    r.start(2, 20)
    with pytest.raises(RuntimeError, match="free pages"):
        r.start(3, 20)
    assert sorted(r.pages.free) == [0, 1, 2, 3]
    with pytest.raises(ValueError, match="started for 0"):        # nothing is left to write to
        r.width = 8
        r.step(torch.zeros(3, 1, 8), None, None)
    r.start(1, 64)
    assert sorted(r.own[0].tolist()) == [0, 1, 2, 3]


@pytest.mark.gpu
def test_a_reader_answers_many_times():
    """More often than its own pages would last without being given back, with the same answer each time."""
    from paper_2410_18926_amd.answer import answer, small_setup
    index, reader, questions, embed = small_setup(seed=5)
    ids, first = answer(index, reader, questions, embed, steps=3)
    assert torch.isfinite(first).all()
    for _ in range(30):
        again, hidden = answer(index, reader, questions, embed, steps=3)
        assert torch.equal(again, ids) and torch.equal(hidden, first)
    index.close()
