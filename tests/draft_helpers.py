"""Drafted tokens in 64 bits on the CPU, node by node from the definitions, with the bounds that results in 16 bits have to keep (the terms are those of attn_helpers).

The probabilities of a tree's nodes are operands in float16 whatever the type of the result: half a step of 11 digits each, and below its normal range, which begins 2^-26 below the sums' unit (2^-20 where
a page's scale is the smallest that the unit stays for), a step of 2^-37 (2^-31): TINY."""
import math

import torch

from attn_helpers import MOST, PAGE, SLACK, UNIT, HostCache, scale_for, scores, to8  # noqa: F401

OPERAND, TINY = 2.0 ** -11, 2.0 ** -30


def depths(parent):
    out = []
    for p in parent:
        out.append(out[p] + 1 if p >= 0 else 0)
    return out


def ancestors(parent, i):
    """i and what it continues, up to the root."""
    out = []
    while i >= 0:
        out.append(i)
        i = parent[i]
    return out


def tree_reference(host, rows, lens, trees, q, scale, cap=0.0, slopes=None, window=0):
    """(value, bound) of attention of the trees' nodes q [tokens, heads, d] over the host's cache."""
    heads = q.shape[1]
    u = UNIT[q.dtype]
    out, off = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    base = 0
    for pages, length, parent in zip(rows, lens, trees):
        length = min(length, len(pages) * PAGE)
        n, ctx = len(parent), length - len(parent)
        K, V = host.tokens(0, pages, length), host.tokens(1, pages, length)
        depth = depths(parent)
        place = torch.tensor([j if j < ctx else ctx + depth[j - ctx] for j in range(length)], dtype=torch.int64)
        seen, diag = torch.zeros((n, length), dtype=torch.bool), torch.tensor([ctx + x for x in depth], dtype=torch.int64)
        for i in range(n):
            seen[i, :max(ctx, 0)] = True
            for a in ancestors(parent, i):
                if ctx + a >= 0:
                    seen[i, ctx + a] = True
        if window:
            seen &= diag[:, None] - place < window
        group = heads // K.shape[1]
        for h in range(heads):
            kh, v = K[:, h // group], V[:, h // group]
            x, _ = scores(q[base:base + n, h].cpu().double(), kh, diag, scale, cap, 0.0)
            if slopes is not None:
                x = x - float(slopes[h]) * (diag[:, None] - place)
            p = torch.nan_to_num(torch.softmax(torch.where(seen, x, -math.inf), 1), 0.0) if length else torch.zeros((n, 0), dtype=torch.float64)
            sees = [seen[i].nonzero()[:, 0] for i in range(n)]      # (0 times NaN: what is not seen stays out of the sums)
            o = torch.stack([p[i, s] @ v[s] for i, s in enumerate(sees)]) if n else torch.zeros((0, q.shape[2]), dtype=torch.float64)
            mass = torch.stack([p[i, s] @ v[s].abs() for i, s in enumerate(sees)]) if n else o
            some = torch.stack([v[s].abs().sum(0) for s in sees]) if n else o
            out[base:base + n, h] = o
            off[base:base + n, h] = u * o.abs() + (OPERAND + SLACK) * mass + TINY * some
        base += n
    return out, off


def verify_reference(trees, ids, u, target, draft):
    """(path, kept, next): the walk, one child after another."""
    path, kept, follow, base = [], [], [], 0
    ids, u = ids.tolist(), u.double().tolist()
    vocab = target.shape[1]
    proper = lambda row: torch.nan_to_num(row.cpu().double(), nan=0.0).clamp(min=0)  # noqa: E731
    for parent in trees:
        node, way, r = (0 if parent else -1), [], torch.zeros(vocab, dtype=torch.float64)
        while node >= 0:
            way.append(node)
            r = proper(target[base + node])
            q = proper(draft[base + node]) if draft is not None else None
            onward = -1
            for c in range(node + 1, len(parent)):
                x = ids[base + c]
                if parent[c] != node or not 0 <= x < vocab:
                    continue
                if u[base + c] * (float(q[x]) if q is not None else 1.0) < float(r[x]):
                    onward = c
                    break
                one = torch.zeros(vocab, dtype=torch.bool)
                one[x] = True
                left = torch.where(one, 0.0, r) if q is None else (r - q).clamp(min=0)
                r = left / left.sum() if left.sum() > 0 else r
                if q is not None:
                    q = torch.where(one, 0.0, q)
                    q = q / q.sum() if q.sum() > 0 else q
            node = onward
        total = torch.cumsum(r, 0)
        above = torch.nonzero(total > (u[base] if parent else 0.0) * total[-1]).flatten()
        follow.append(int(above[0]) if above.numel() else -1)
        path += way + [-1] * (len(parent) - len(way))
        kept.append(len(way))
        base += len(parent)
    return path, kept, follow


def keep_reference(host, pages, ctx, path):
    """A layer of the host's cache after the nodes of `path` moved together behind ctx tokens."""
    for x, (code, scale) in enumerate(zip(host.code, host.scale)):
        first = 0
        while first < len(path):
            place = (ctx + first) // PAGE
            last = min(len(path), (place + 1) * PAGE - ctx)
            page, src = pages[place], [ctx + a for a in path[first:last]]
            for h in range(code.shape[1]):
                value = [code[pages[a // PAGE], h, a % PAGE] * scale[pages[a // PAGE], h] for a in src]
                away = [v[:host.d].nan_to_num(0, 0, 0).abs().max() for v, a in zip(value, src) if a // PAGE != place]
                now = max([float(scale[page, h])] + [scale_for(float(t)) for t in away])
                if any(a != b for a, b in zip(path[first:last], range(first, last))):
                    until = ctx + last - place * PAGE
                    code[page, h, :until] = to8(code[page, h, :until] * (float(scale[page, h]) / now)).double()
                    for v, i in zip(value, range(first, last)):
                        code[page, h, ctx + i - place * PAGE] = to8(v / now).double()
                    scale[page, h] = now
            first = last
