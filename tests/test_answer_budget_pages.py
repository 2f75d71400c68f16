"""Conversations within a budget move to fresh pages while their old ones are held: a store without room for both refuses when they start, not after tokens have been written."""
import pytest
import torch

from test_answer_pages import reader_of


class Store:
    """What the page-keeping asks of a store."""

    def __init__(self):
        self.cut = 0

    def evict(self, own, lengths, sums, budget, to, recent):
        self.cut += 1
        assert not set(own.flatten().tolist()) & set(to.flatten().tolist())
        return None, None, sums


def budget_reader(pages, budget, page_size=16):
    r = reader_of(pages, page_size)
    r.budget, r.recent, r.heads, r.states = budget, budget // 4, 2, Store()
    return r


def grow(r, tokens):
    """What step() does to a conversation's length, one token at a time."""
    for _ in range(tokens):
        if r.past > r.budget and r.past + 1 > r.most:
            r._cut()
        assert r.past + 1 <= r.most
        r.past += 1


@pytest.mark.parametrize("pages,conversations,tokens,budget", [(64, 3, 176, 160), (64, 3, 216, 200), (11, 1, 96, 64), (5, 3, 16, 12)])
def test_no_room_for_the_move_is_refused_at_the_start(pages, conversations, tokens, budget):
    r = budget_reader(pages, budget)
    with pytest.raises(RuntimeError, match="free pages"):
        r.start(conversations, tokens)
    assert sorted(r.pages.free) == list(range(pages)) and r.most == 0
    # conversations that are known never to be cut need no second set
    for longest in (tokens, tokens - 1):
        r.start(conversations, tokens, longest=longest)
        grow(r, longest)
        assert r.states.cut == 0
    with pytest.raises(RuntimeError, match="free pages"):
        r.start(conversations, tokens, longest=tokens + 1)


@pytest.mark.parametrize("pages,conversations,tokens,budget", [(66, 3, 176, 160), (12, 1, 96, 64), (6, 3, 16, 12), (64, 3, 28, 12)])
def test_what_starts_is_cut_as_often_as_it_takes(pages, conversations, tokens, budget):
    r = budget_reader(pages, budget)
    for _ in range(3):
        r.start(conversations, tokens)
        grow(r, 5 * tokens)
        assert len(r.pages.free) + len(r.taken) == pages and not set(r.pages.free) & set(r.taken)
    assert r.states.cut >= 9


def test_a_budget_that_holds_all_tokens_needs_no_second_set():
    r = budget_reader(4, 64)
    r.start(1, 64)
    grow(r, 64)
    assert r.states.cut == 0


def test_tokens_that_do_not_fit_even_after_a_cut_leave_the_conversation_as_it_was():
    r = budget_reader(12, 64)
    r.width = 8
    r.start(1, 96)
    grow(r, 90)
    own = r.own.clone()
    with pytest.raises(ValueError, match="started for 96"):
        r.step(torch.zeros(1, 33, 8), None, None)
    assert r.states.cut == 0 and r.past == 90 and torch.equal(r.own, own) and len(r.pages.free) == 6
