"""Search, then read what was found: the index, the state store and its two attentions together.

    python -m paper_2410_18926_amd.answer [--bits 4] [--budget TOKENS]

A question is embedded, Index.search finds the passages nearest to it, and a small decoder (two attention blocks, random weights) reads the question
and then writes tokens: every token attends to the conversation so far (attend_chunk over the conversation's own pages) and to the states
of the passages (attend_passages with the ids and distances as the search left them).  All states live in one 8-bit store: the passages' pages are
filled once, the conversation's as it grows.  Everything stays on the GPU; the ids are never copied to the host.

--bits 4 holds all states in 4 bits (States4).  --budget keeps conversations within so many tokens: the weights that attention gives a conversation's keys are added up as it
goes (attend_weights), and when the next tokens do not fit, the newest ones and those with the largest sums move to fresh pages (evict).
"""
from __future__ import annotations

import argparse

import torch

from . import binding
from .states import States
from .states4 import States4


class PageAllocator:
    """Hands out pages of a store, from the host: page numbers never depend on what the GPU computes."""

    def __init__(self, pages: int):
        self.free = list(range(pages))

    def check(self, n: int):
        if n > len(self.free):
            raise RuntimeError(f"the store has no {n} free pages left")

    def take(self, n: int) -> list:
        self.check(n)
        taken, self.free = self.free[:n], self.free[n:]
        return taken

    def give_back(self, pages: list):
        self.free = self.free + pages


class Reader:
    """A decoder of one layer over a store of passages: self-attention, cross-attention to the found passages, both with `group` query heads to a head of
    the store."""

    budget, recent = None, 0

    def __init__(self, passages: list, heads=2, group=2, dim=64, page_size=16, own_pages=64, dtype=torch.bfloat16, seed=0, device="cuda", bits=8, budget=None, recent=None):
        """passages: encoder outputs [tokens, width] of each passage, one for each corpus row.  bits: of the store, 8 or 4.  budget: tokens that a conversation is cut to when it
        has grown out of its pages, `recent` of them (a quarter) its newest; None: it may not grow out of them."""
        if bits not in (8, 4):
            raise ValueError(f"states are held in 8 or 4 bits, not {bits}")
        if budget is not None:
            self.budget, self.recent = budget, budget // 4 if recent is None else recent
            if budget < 1 or not 0 <= self.recent <= budget:
                raise ValueError(f"a budget of {budget} tokens, {self.recent} of them the newest")
        g = torch.Generator().manual_seed(seed)
        self.width = width = passages[0].shape[1]
        weight = lambda n, m: (torch.randn(n, m, generator=g) * n ** -0.5).to(device, dtype)  # noqa: E731
        self.q, self.kv, self.o = weight(width, heads * group * dim), weight(width, 2 * heads * dim), weight(heads * group * dim, width)
        self.cross_q, self.cross_kv, self.cross_o = weight(width, heads * group * dim), weight(width, 2 * heads * dim), weight(heads * group * dim, width)
        self.heads, self.group, self.dim, self.page_size, self.dtype, self.device = heads, group, dim, page_size, dtype, device
        need = [-(-len(p) // page_size) for p in passages]
        self.states = (States if bits == 8 else States4).empty(sum(need) + own_pages, heads, page_size, dim, device)
        self.pages, self.taken = PageAllocator(self.states.pages), []
        # the passages' states: written once, found by number afterwards
        tables = torch.zeros(len(passages), max(need), dtype=torch.int32)
        for i, n in enumerate(need):
            tables[i, :n] = torch.tensor(self.pages.take(n), dtype=torch.int32)
        self.tables, self.lengths = tables.to(device), torch.tensor([len(p) for p in passages], dtype=torch.int32, device=device)
        token = torch.cat([torch.arange(len(p)) for p in passages])
        of = torch.repeat_interleave(torch.arange(len(passages)), torch.tensor([len(p) for p in passages]))
        slots = tables[of, token // page_size].long() * page_size + token % page_size
        kv = (torch.cat(passages).to(device, dtype) @ self.cross_kv).view(-1, 2 * heads, dim)
        self.states.write(kv[:, :heads], kv[:, heads:], slots.to(device))

    def start(self, conversations: int, tokens: int, longest=None):
        """Pages for conversations of up to `tokens` tokens each (with a budget: at a time).  Those of the conversations before are given back (what reads them has been enqueued on the
        same stream): step() goes on with the new ones.  Conversations that are to be cut need as many pages once more while they move: what the store has no room for is refused here.
        longest: tokens that they will have in all (None: any number); where they stay within `tokens`, none is cut."""
        self.pages.give_back(self.taken)
        self.taken, self.past, self.most = [], 0, 0
        width = -(-tokens // self.page_size)
        if self.budget is not None and self.budget < tokens and (longest is None or longest > tokens):
            self.pages.check(2 * conversations * width)
        self.own = self._own_pages(conversations, width)
        if self.budget is not None:
            self.sums = torch.zeros((conversations, self.heads, width * self.page_size), device=self.device)
        self.most = tokens

    def _own_pages(self, conversations: int, width: int):
        self.taken = self.pages.take(conversations * width)
        return torch.tensor(self.taken, dtype=torch.int32).view(conversations, width).to(self.device)

    def _cut(self):
        """Conversations go on with `budget` of their tokens, on fresh pages; what reads the old ones has been enqueued on the same stream."""
        n, width = self.own.shape
        old = self.taken
        to = self._own_pages(n, width)
        lengths = torch.full((n,), self.past, dtype=torch.int32, device=self.device)
        _, _, self.sums = self.states.evict(self.own, lengths, self.sums, min(self.budget, self.past), to, recent=min(self.recent, self.past))
        self.own, self.past = to, min(self.budget, self.past)
        self.pages.give_back(old)

    def step(self, hidden, ids, dists):
        """Hidden states [conversations, new tokens, width] of the newest tokens -> the same after the layer.  ids, dists [conversations, found] as the
        search returned them."""
        n, new, _ = hidden.shape
        cut = self.budget is not None and self.past > self.budget and self.past + new > self.most
        past = self.budget if cut else self.past
        if past + new > self.most:
            raise ValueError(f"conversations of {past + new} tokens: started for {self.most}")
        if cut:
            self._cut()
        x = hidden.reshape(n * new, self.width)
        at = torch.arange(self.past, self.past + new, device=self.device)
        slots = (self.own[:, at // self.page_size].long() * self.page_size + at % self.page_size).reshape(-1)
        kv = (x @ self.kv).view(n * new, 2 * self.heads, self.dim)
        self.states.write(kv[:, :self.heads], kv[:, self.heads:], slots)
        self.past += new
        lengths = torch.full((n,), self.past, dtype=torch.int32, device=self.device)
        q = (x @ self.q).view(n * new, self.heads * self.group, self.dim)
        x = x + self.states.attend_chunk(q, self.own, lengths).reshape(n * new, -1) @ self.o
        if self.budget is not None:
            self.states.attend_weights(q, self.own, lengths, before=self.sums, out=self.sums)
        q = (x @ self.cross_q).view(n * new, self.heads * self.group, self.dim)
        found = self.states.attend_passages(q, ids, self.tables, self.lengths, scores=dists, score_weight=-1.0)
        return (x + found.reshape(n * new, -1) @ self.cross_o).view(n, new, self.width)


def answer(index: binding.Index, reader: Reader, question, embed, steps: int, k: int = 4, w: int = 8, m: int = 50):
    """question [conversations, tokens, width]; embed(hidden [conversations, width]) -> search vectors.  Returns (ids of the passages, hidden states of the question
    and of `steps` further tokens [conversations, tokens + steps, width]): each further token starts from the one before."""
    index.use_torch_stream()
    ids, dists = index.search(embed(question.mean(1)).float().contiguous(), k, w, m, asynchronous=True)
    tokens = question.shape[1] + steps
    reader.start(question.shape[0], tokens if reader.budget is None else min(tokens, max(question.shape[1], reader.budget) + reader.page_size), longest=tokens)
    out = [reader.step(question, ids, dists)]
    for _ in range(steps):
        out.append(reader.step(out[-1][:, -1:], ids, dists))
    return ids, torch.cat(out, 1)


def small_setup(seed: int = 0, device: str = "cuda", **more):
    """(index over 3000 passages' embeddings, reader over their states, questions, embed) of random content.  more: arguments of Reader."""
    from .synth import build_index, make_dataset
    from .synth.workloads import L2, Workload
    wl = Workload("passages", 91, n=3000, d=32, nq=40, G=12, alpha=None, normalize=False, lognormal_norms=None, metric=L2, L=12, dp=32, r=8, w=4, m=50, n_train=1500, w_train=4)
    corpus, _ = make_dataset(wl)
    index = binding.Index.from_arrays(build_index(corpus, wl))
    g = torch.Generator().manual_seed(seed)
    width = 48
    passages = [torch.randn(int(n), width, generator=g) for n in torch.randint(1, 60, (wl.n,), generator=g)]
    lift = torch.randn(width, wl.d, generator=g).to(device, torch.bfloat16)
    questions = torch.randn(3, 5, width, generator=g).to(device, torch.bfloat16)
    return index, Reader(passages, seed=seed, device=device, **more), questions, lambda h: h @ lift


def main():
    ap = argparse.ArgumentParser(description="Search, then read what was found (random content).")
    ap.add_argument("--bits", type=int, choices=(8, 4), default=8, help="of the states")
    ap.add_argument("--budget", type=int, help="tokens that a conversation is cut to")
    ap.add_argument("--steps", type=int, default=6, help="tokens to write")
    a = ap.parse_args()
    index, reader, questions, embed = small_setup(bits=a.bits, budget=a.budget)
    ids, hidden = answer(index, reader, questions, embed, steps=a.steps)
    torch.cuda.synchronize()
    for i in range(ids.shape[0]):
        print(f"question {i}: passages {ids[i].tolist()}, last token's state begins {[round(float(v), 3) for v in hidden[i, -1, :4]]}")
    index.close()


if __name__ == "__main__":
    main()
