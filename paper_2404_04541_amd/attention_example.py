"""Attention over sparse structures from a product's pattern to serving, on small random tensors:

    python -m paper_2404_04541_amd.attention_example

A graph of tiles (each linked to its neighbours and to the first) is squared by the library's own product: what two steps reach is the pattern of a
training step over packed documents.  Then two prompts go through the forward pass into a paged cache, a few tokens are decoded, the
better sequence is forked, and the pages are compacted.
"""
import torch

from . import attention as at
from . import binding as sg


def two_step_pattern(handle, tiles):
    """Structure of G * G as a DeviceCSR, G the graph of neighbouring tiles with tile 0 linked to all."""
    rows = [sorted({0, max(t - 1, 0), t}) for t in range(tiles)]
    ptr = torch.tensor([0] + [len(r) for r in rows]).cumsum(0)
    cols = torch.tensor([c for r in rows for c in r], dtype=torch.int32)
    graph = sg.DeviceCSR(tiles, tiles, ptr.cuda(), cols.cuda(), torch.ones(len(cols), dtype=torch.float32).cuda())
    return sg.spgemm(handle, graph, graph)


def training_step(handle, lengths=(700, 200, 1148), heads=8, kv_heads=2, head_dim=64):
    """Gradients of one attention layer over packed documents through the pattern."""
    tokens = sum(lengths)
    ptr = torch.tensor([0, *lengths]).cumsum(0).cuda()
    plan = at.symbolic(handle, tokens, tokens, q_ptr=ptr, k_ptr=ptr, tiles=two_step_pattern(handle, -(-tokens // at.TILE)))
    q, k, v = (torch.randn(tokens, n, head_dim, device="cuda", dtype=torch.bfloat16, requires_grad=True) for n in (heads, kv_heads, kv_heads))
    o = at.attention(handle, plan, q, k, v, cap=30.0)
    o.float().square().mean().backward()
    return o, (q.grad, k.grad, v.grad)


def serve(handle, prompts=(100, 37), steps=30, heads=8, kv_heads=2, head_dim=64):
    """Prompts, decoded tokens, a fork, a compaction; returns the last step's output and what the forward pass gives for the same tokens."""
    device = torch.device("cuda")
    n, most = len(prompts), max(prompts) + steps + 1
    make = lambda *shape: torch.randn(*shape, device=device, dtype=torch.bfloat16)  # noqa: E731
    kept = [(make(p, kv_heads, head_dim), make(p, kv_heads, head_dim)) for p in prompts]
    cache = at.PagedCache.empty(1, 4 * n * (-(-most // at.PAGE)), kv_heads, head_dim)
    ints = lambda values, dtype=torch.int32: torch.tensor(values, dtype=dtype, device=device)  # noqa: E731

    # the prompts, packed: their own attention, and their keys and values into pages
    ptr = ints([0, *prompts], torch.int64).cumsum(0)
    total = sum(prompts)
    plan = at.symbolic(handle, total, total, q_ptr=ptr, k_ptr=ptr)
    k, v = (torch.cat([x[i] for x in kept]) for i in (0, 1))
    at.forward(handle, plan, make(total, heads, head_dim), k, v)
    none = at.PageTable(ints([0], torch.int64), ints([]))
    lens = list(prompts)
    table, _ = at.fork(handle, cache, none, ints([]), ints([-1] * n), ints(lens))
    at.append(handle, cache, 0, table, ints(lens), ptr, k, v)

    out = query = None
    for step in range(steps):
        # the next table: every sequence grows by a token; half way the second one ends and the first goes on twice
        parent = [0, 0] if step == steps // 2 else list(range(len(lens)))
        grown = [lens[p] + 1 for p in parent]
        table, _ = at.fork(handle, cache, table, ints(lens), ints(parent), ints(grown))
        kept, lens = [kept[p] for p in parent], grown
        count = len(lens)
        k, v, query = make(count, kv_heads, head_dim), make(count, kv_heads, head_dim), make(count, 1, heads, head_dim)
        kept = [(torch.cat([a, k[i:i + 1]]), torch.cat([b, v[i:i + 1]])) for i, (a, b) in enumerate(kept)]
        at.append(handle, cache, 0, table, ints(lens), torch.arange(count + 1, device=device), k, v)
        out = at.attend(handle, cache, 0, table, ints(lens), query)
    table, live = at.compact(handle, cache, table)
    again = at.attend(handle, cache, 0, table, ints(lens), query)
    assert torch.equal(out, again), "compaction moves pages, not what they hold"

    # the same tokens in 16 bits: one query a document, at its last key
    k_ptr = ints([0, *lens], torch.int64).cumsum(0)
    q_ptr = torch.arange(len(lens) + 1, device=device)
    plan = at.symbolic(handle, len(lens), sum(lens), q_ptr=q_ptr, k_ptr=k_ptr)
    want, _ = at.forward(handle, plan, query[:, 0], torch.cat([a for a, _ in kept]), torch.cat([b for _, b in kept]))
    return out[:, 0], want, live


def main():
    torch.manual_seed(0)
    handle = sg.Handle()
    o, grads = training_step(handle)
    print(f"training step: {tuple(o.shape)}, gradients {[tuple(g.shape) for g in grads]}")
    out, want, live = serve(handle)
    off = float((out.float() - want.float()).norm() / want.float().norm())
    print(f"serving: {live} pages in use, the last tokens' outputs from 8 bits are {100 * off:.1f} % off those from 16 bits")


if __name__ == "__main__":
    main()
