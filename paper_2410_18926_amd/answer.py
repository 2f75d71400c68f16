"""Search, then read what was found: the index, the state store and its two attentions together.

    python -m paper_2410_18926_amd.answer

A question is embedded, Index.search finds the passages nearest to it, and a small decoder (two attention blocks, random weights) reads the question
and then writes tokens: every token attends to the conversation so far (attend_chunk over the conversation's own pages) and to the states
of the passages (attend_passages with the ids and distances as the search left them).  All states live in one 8-bit store: the passages' pages are
filled once, the conversation's as it grows.  Everything stays on the GPU; the ids are never copied to the host.
"""
from __future__ import annotations

import torch

from . import binding
from .states import States


class PageAllocator:
    """Hands out pages of a store, from the host: page numbers never depend on what the GPU computes."""

    def __init__(self, pages: int):
        self.free = list(range(pages))

    def take(self, n: int) -> list:
        if n > len(self.free):
            raise RuntimeError(f"the store has no {n} free pages left")
        taken, self.free = self.free[:n], self.free[n:]
        return taken

    def give_back(self, pages: list):
        self.free = self.free + pages


class Reader:
    """A decoder of one layer over a store of passages: self-attention, cross-attention to the found passages, both with `group` query heads to a head of
    the store."""

    def __init__(self, passages: list, heads=2, group=2, dim=64, page_size=16, own_pages=64, dtype=torch.bfloat16, seed=0, device="cuda"):
        """passages: encoder outputs [tokens, width] of each passage, one for each corpus row."""
        g = torch.Generator().manual_seed(seed)
        self.width = width = passages[0].shape[1]
        weight = lambda n, m: (torch.randn(n, m, generator=g) * n ** -0.5).to(device, dtype)  # noqa: E731
        self.q, self.kv, self.o = weight(width, heads * group * dim), weight(width, 2 * heads * dim), weight(heads * group * dim, width)
        self.cross_q, self.cross_kv, self.cross_o = weight(width, heads * group * dim), weight(width, 2 * heads * dim), weight(heads * group * dim, width)
        self.heads, self.group, self.dim, self.page_size, self.dtype, self.device = heads, group, dim, page_size, dtype, device
        need = [-(-len(p) // page_size) for p in passages]
        self.states = States.empty(sum(need) + own_pages, heads, page_size, dim, device)
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

    def start(self, conversations: int, tokens: int):
        """Pages for conversations of up to `tokens` tokens each.  Those of the conversations before are given back (what reads them has been enqueued on the
        same stream): step() goes on with the new ones."""
        self.pages.give_back(self.taken)
        self.taken, self.past, self.most = [], 0, 0
        width = -(-tokens // self.page_size)
        self.taken = self.pages.take(conversations * width)
        self.own = torch.tensor(self.taken, dtype=torch.int32).view(conversations, width).to(self.device)
        self.most = tokens

    def step(self, hidden, ids, dists):
        """Hidden states [conversations, new tokens, width] of the newest tokens -> the same after the layer.  ids, dists [conversations, found] as the
        search returned them."""
        n, new, _ = hidden.shape
        if self.past + new > self.most:
            raise ValueError(f"conversations of {self.past + new} tokens: started for {self.most}")
        x = hidden.reshape(n * new, self.width)
        at = torch.arange(self.past, self.past + new, device=self.device)
        slots = (self.own[:, at // self.page_size].long() * self.page_size + at % self.page_size).reshape(-1)
        kv = (x @ self.kv).view(n * new, 2 * self.heads, self.dim)
        self.states.write(kv[:, :self.heads], kv[:, self.heads:], slots)
        self.past += new
        lengths = torch.full((n,), self.past, dtype=torch.int32, device=self.device)
        q = (x @ self.q).view(n * new, self.heads * self.group, self.dim)
        x = x + self.states.attend_chunk(q, self.own, lengths).reshape(n * new, -1) @ self.o
        q = (x @ self.cross_q).view(n * new, self.heads * self.group, self.dim)
        found = self.states.attend_passages(q, ids, self.tables, self.lengths, scores=dists, score_weight=-1.0)
        return (x + found.reshape(n * new, -1) @ self.cross_o).view(n, new, self.width)


def answer(index: binding.Index, reader: Reader, question, embed, steps: int, k: int = 4, w: int = 8, m: int = 50):
    """question [conversations, tokens, width]; embed(hidden [conversations, width]) -> search vectors.  Returns (ids of the passages, hidden states of the question
    and of `steps` further tokens [conversations, tokens + steps, width]): each further token starts from the one before."""
    index.use_torch_stream()
    ids, dists = index.search(embed(question.mean(1)).float().contiguous(), k, w, m, asynchronous=True)
    reader.start(question.shape[0], question.shape[1] + steps)
    out = [reader.step(question, ids, dists)]
    for _ in range(steps):
        out.append(reader.step(out[-1][:, -1:], ids, dists))
    return ids, torch.cat(out, 1)


def small_setup(seed: int = 0, device: str = "cuda"):
    """(index over 3000 passages' embeddings, reader over their states, questions, embed) of random content."""
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
    return index, Reader(passages, seed=seed, device=device), questions, lambda h: h @ lift


def main():
    index, reader, questions, embed = small_setup()
    ids, hidden = answer(index, reader, questions, embed, steps=6)
    torch.cuda.synchronize()
    for i in range(ids.shape[0]):
        print(f"question {i}: passages {ids[i].tolist()}, last token's state begins {[round(float(v), 3) for v in hidden[i, -1, :4]]}")
    index.close()


if __name__ == "__main__":
    main()
