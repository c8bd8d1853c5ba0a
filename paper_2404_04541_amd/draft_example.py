"""Serving with drafted tokens on a small random model:

    python -m paper_2404_04541_amd.draft_example

Every step drafts a tree of tokens behind each sequence (two for every node, three levels), runs the model's attention layer over all nodes at once, verifies them against the model's probabilities and
keeps the accepted ones in the cache.  The draft is a table of the model's own, so that it is right more often than not.
"""
import math

import torch

from . import attention as at
from . import binding as sg
from . import drafts as dr

PARENT = [-1, 0, 0, 1, 1, 2, 2]       # the tree's nodes, level by level


class Model:
    """One attention layer between an embedding and its transpose; `draft` guesses from the last token alone."""

    def __init__(self, vocab=300, heads=8, kv_heads=2, head_dim=64, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim, self.vocab = heads, kv_heads, head_dim, vocab
        make = lambda *shape: torch.randn(shape, generator=gen, device="cuda") / math.sqrt(shape[0])  # noqa: E731
        width = heads * head_dim
        self.embed, self.q, self.k, self.v, self.o = make(vocab, width) * math.sqrt(vocab), make(width, width), make(width, kv_heads * head_dim), make(width, kv_heads * head_dim), make(width, width)

    def project(self, ids):
        x = self.embed[ids.long()]
        rows = lambda w, heads: (x @ w).view(-1, heads, self.head_dim).to(torch.bfloat16)  # noqa: E731
        return rows(self.q, self.heads), rows(self.k, self.kv_heads), rows(self.v, self.kv_heads)

    def probabilities(self, ids, attended=None):
        x = self.embed[ids.long()]
        if attended is not None:
            x = x + 0.5 * (attended.float().flatten(1) @ self.o)
        return torch.softmax(x @ self.embed.T * (3.0 / x.shape[1]), -1)


def drafted(model, last, gen):
    """(tokens of every sequence's tree, the rows that they were drawn from, packed): children of a node are drawn one after the other without replacement."""
    n = len(PARENT)
    ids = torch.zeros((len(last), n), dtype=torch.int32, device="cuda")
    rows = torch.zeros((len(last), n, model.vocab), device="cuda")
    ids[:, 0] = last
    for node in range(n):
        rows[:, node] = model.probabilities(ids[:, node])
        children = [i for i, p in enumerate(PARENT) if p == node]
        if children:
            noise = torch.rand((len(last), model.vocab), generator=gen, device="cuda").clamp(min=1e-20)
            best = (rows[:, node].log() - noise.log().neg().log()).topk(len(children)).indices
            ids[:, children] = best.to(torch.int32)
    return ids.flatten(), rows.flatten(0, 1)


def serve(handle, prompts=(40, 7, 130), steps=12, seed=1):
    """-> (tokens of every sequence, how many tokens a step and sequence got)."""
    model, gen = Model(), torch.Generator(device="cuda").manual_seed(seed)
    ints = lambda values, dtype=torch.int32: torch.tensor(values, dtype=dtype, device="cuda")  # noqa: E731
    n, count = len(prompts), len(PARENT)
    text = [torch.randint(0, model.vocab, (p,), generator=gen, device="cuda", dtype=torch.int32).tolist() for p in prompts]
    cache = at.PagedCache.empty(1, 4 * n * (2 + max(prompts) // at.PAGE) + n * steps, model.kv_heads, model.head_dim)

    # the prompts but for their last token, which is the first tree's root
    lens, ptr = ints([p - 1 for p in prompts]), [0]
    for p in prompts:
        ptr.append(ptr[-1] + p - 1)
    table, _ = at.fork(handle, cache, at.PageTable(ints([0], torch.int64), ints([])), ints([]), ints([-1] * n), lens)
    _, k, v = model.project(ints([t for s in text for t in s[:-1]]))
    at.append(handle, cache, 0, table, lens, ints(ptr, torch.int64), k, v)

    rows, nodes = ints(range(n)), ints([count * i for i in range(n + 1)], torch.int64)
    trees = dr.symbolic(handle, nodes, ints(PARENT * n), count)          # (the same tree in every step: its structure is made once)
    got = 0
    for _ in range(steps):
        ids, draft = drafted(model, ints([s[-1] for s in text]), gen)
        full = lens + count
        table, _ = at.fork(handle, cache, table, lens, rows, full)
        q, k, v = model.project(ids)
        at.append(handle, cache, 0, table, full, nodes, k, v)
        o = dr.attend(handle, cache, 0, table, full, trees, q)
        path, kept, follow = dr.verify(handle, trees, ids, torch.rand(n * count, generator=gen, device="cuda"), model.probabilities(ids, o), draft)
        lens = dr.keep(handle, cache, table, full, trees, path, kept)
        table, _ = at.fork(handle, cache, table, lens, rows, lens)       # pages of refused nodes go back
        ids, path = ids.view(n, count), path.view(n, count).tolist()
        for s, (many, token) in enumerate(zip(kept.tolist(), follow.tolist())):
            text[s] += [int(ids[s, i]) for i in path[s][1:many]] + [token]
            got += many
    assert lens.tolist() == [len(t) - 1 for t in text], "the cache holds every token but the last"
    return text, got / (steps * n)


def main():
    text, rate = serve(sg.Handle())
    print(f"sequences of {[len(t) for t in text]} tokens, {rate:.2f} a step")


if __name__ == "__main__":
    main()
