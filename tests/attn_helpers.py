"""Attention, the paged cache and its tables in 64 bits on the CPU, element by element from the definitions, with the bounds that
results in 16 bits have to keep.

With u the unit roundoff of the type (each rounding is off by at most u times its result), every bound is a sum over the roundings that the
operators make, taken by absolute values: probabilities and their gradients are rounded once as operands and the result once; f32 arithmetic in
between (dot products, tanh, exp2) is allowed SLACK of the probability, which covers score errors up to 2e-4 (scores of a few hundred at
24 bits, tanh off by 2e-7 times a cap of at most 100, sums of a few thousand terms); and an operand of float16 below its normal range is off
by at most TINY."""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # 8 and 11 significant bits
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}
SLACK = 2e-4
PAGE, TILE, MOST = 64, 128, 448.0


def visible(q_len, k_len, q_ptr=None, k_ptr=None, prefix=None, causal=True, window=0, tiles=None):
    """(bool [q_len, k_len], diag [q_len])"""
    q_ptr, k_ptr = q_ptr or [0, q_len], k_ptr or [0, k_len]
    seen = torch.zeros((q_len, k_len), dtype=torch.bool)
    diag = torch.zeros(q_len, dtype=torch.int64)
    for d in range(len(q_ptr) - 1):
        for i in range(q_ptr[d], q_ptr[d + 1]):
            diag[i] = i + k_ptr[d + 1] - q_ptr[d + 1]
            lo, hi = k_ptr[d], k_ptr[d + 1]
            if causal:
                hi = min(hi, max(k_ptr[d] + (prefix[d] if prefix else 0), int(diag[i]) + 1))
            if window:
                lo = max(lo, int(diag[i]) - window + 1)
            if lo < hi:
                seen[i, lo:hi] = True
    if tiles is not None:
        held = torch.zeros((-(-q_len // TILE), -(-k_len // TILE)), dtype=torch.bool)
        for r in range(len(tiles[0]) - 1):
            for c in tiles[1][tiles[0][r]:tiles[0][r + 1]]:
                held[r, c] = True
        seen &= held.repeat_interleave(TILE, 0)[:q_len].repeat_interleave(TILE, 1)[:, :k_len]
    return seen, diag


def scores(q, k, diag, scale, cap, slope):
    """Scores of one head, and the tanh of the capped ones."""
    raw = q @ k.T * scale
    th = torch.tanh(raw / cap) if cap else torch.zeros_like(raw)
    x = cap * th if cap else raw
    return x - slope * (diag[:, None] - torch.arange(k.shape[0])).abs(), th


def reference(q, k, v, d_o, seen, diag, scale, cap=0.0, slopes=None):
    """Results in 64 bits and the bounds of the 16-bit ones: {name: (value, bound)}; o, lse, and with d_o dq, dk, dv."""
    u, tiny = UNIT[q.dtype], TINY[q.dtype]
    group = q.shape[1] // k.shape[1]
    Q, K, V = (t.detach().cpu().double() for t in (q, k, v))
    G = d_o.detach().cpu().double() if d_o is not None else None
    out = {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in (("o", Q), ("dq", Q), ("dk", K), ("dv", K))}
    lse = torch.full((Q.shape[1], Q.shape[0]), -math.inf, dtype=torch.float64)
    for h in range(Q.shape[1]):
        qh, kh, vh = Q[:, h], K[:, h // group], V[:, h // group]
        x, th = scores(qh, kh, diag, scale, cap, float(slopes[h]) if slopes is not None else 0.0)
        x = x.masked_fill(~seen, -math.inf)
        lse[h] = torch.logsumexp(x, 1)
        p = torch.where(seen, torch.exp(x - torch.where(lse[h] == -math.inf, 0.0, lse[h])[:, None]), 0.0)
        o = p @ vh
        mass = p @ vh.abs()
        o_off = u * o.abs() + (u + SLACK) * mass + tiny * (seen.double() @ vh.abs())
        out["o"][0][:, h], out["o"][1][:, h] = o, o_off
        if G is None:
            continue
        g = G[:, h]
        back = 1 - th ** 2
        dp = g @ vh.T
        delta = (g * o).sum(1, keepdim=True)
        delta_off = (g.abs() * o_off).sum(1, keepdim=True) + SLACK * (g.abs() * mass).sum(1, keepdim=True)
        ds = p * (dp - delta) * back
        ds_off = (u + 4 * SLACK) * ds.abs() + p * (delta_off + SLACK * (g.abs() @ vh.abs().T)) + tiny * seen
        for name, a, b, off in (("dq", ds, kh, ds_off), ("dk", ds.T, qh, ds_off.T)):
            at = h if name == "dq" else h // group
            out[name][0][:, at] += a @ b * scale
            out[name][1][:, at] += off @ b.abs() * scale
        out["dv"][0][:, h // group] += p.T @ g
        out["dv"][1][:, h // group] += ((u + SLACK) * p + tiny * seen).T @ g.abs()
    for n in ("dq", "dk", "dv"):
        out[n] = (out[n][0], out[n][1] + u * out[n][0].abs())
    out["lse"] = (lse, torch.full_like(lse, 2 * SLACK))
    return out


def check(name, got, value, bound):
    got, tiny = got.detach().cpu().double(), (2.0 ** -24 if got.dtype == torch.float16 else 0.0)   # (a result below float16's normal range)
    assert got.shape == value.shape, name
    same = got == value          # infinities
    off = torch.where(same, 0.0, (got - value).abs())
    bad = ~(off <= 1.01 * bound + 1e-30 + tiny)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / (bound + 1e-30 + tiny)).max()):.3g} times the bound"


# ---- cache ---------------------------------------------------------------------------------------

def room_of(d):
    return 64 if d <= 64 else 128


def to8(x):
    return x.clamp(-MOST, MOST).float().to(torch.float8_e4m3fn)


def scale_for(most):
    if most == 0:
        return 2.0 ** -100
    e = math.ceil(math.log2(most / MOST))
    while most / 2.0 ** e > MOST:
        e += 1
    while most / 2.0 ** (e - 1) <= MOST:
        e -= 1
    return 2.0 ** min(max(e, -100), 120)


class HostCache:
    """A layer of a cache as numbers: codes [pages, heads, 64, room] (the values that 8 bits stand for, before the scale) and scales [pages, heads]."""

    def __init__(self, cache, layer):
        self.d = cache.head_dim
        self.code = [cache.k[layer].cpu().view(torch.float8_e4m3fn).double(), cache.v[layer].cpu().view(torch.float8_e4m3fn).double().transpose(-1, -2).clone()]
        self.scale = [cache.k_scale[layer].cpu().double(), cache.v_scale[layer].cpu().double()]

    def append(self, rows, lens, new_ptr, k, v):
        """rows: the pages of each sequence."""
        for x, (code, scale) in enumerate(zip(self.code, self.scale)):
            new = (k, v)[x].detach().cpu().double()
            for s, pages in enumerate(rows):
                n = new_ptr[s + 1] - new_ptr[s]
                pos = lens[s] - n
                while pos < lens[s]:
                    end = min(lens[s], (pos // PAGE + 1) * PAGE)
                    if pos // PAGE < len(pages):
                        p, o = pages[pos // PAGE], pos % PAGE
                        part = new[new_ptr[s + 1] - lens[s] + pos:new_ptr[s + 1] - lens[s] + end].transpose(0, 1)       # [heads, tokens, d]
                        for h in range(code.shape[1]):
                            need = scale_for(float(part[h].nan_to_num(0, 0, 0).abs().max()))
                            now = max(float(scale[p, h]), need) if o else need
                            if o:
                                code[p, h, :o] = to8(code[p, h, :o] * (float(scale[p, h]) / now)).double()
                            code[p, h, o:o + end - pos, :self.d] = to8(part[h] / now).double()
                            scale[p, h] = now
                    pos = end

    def tokens(self, x, pages, count):
        """Keys (0) or values (1) [count, heads, d] of a sequence."""
        whole = (self.code[x][pages] * self.scale[x][pages][..., None, None]).transpose(1, 2).reshape(-1, self.code[x].shape[1], self.code[x].shape[3])
        return whole[:count, :, :self.d]

    def same(self, cache, layer, rows, lens):
        """The bytes of every sequence's tokens, and the scales of its pages, are this cache's."""
        other = HostCache(cache, layer)
        for pages, n in zip(rows, lens):
            for x in (0, 1):
                for i, p in enumerate(pages[:-(-n // PAGE)]):
                    live = min(PAGE, n - i * PAGE)
                    assert torch.equal(self.scale[x][p], other.scale[x][p]), ("kv"[x], "scale", p)
                    a, b = self.code[x][p, :, :live, :self.d], other.code[x][p, :, :live, :self.d]
                    assert torch.equal(a.nan_to_num(1e9), b.nan_to_num(1e9)), ("kv"[x], p)


def attend_reference(host, rows, lens, q, scale, cap=0.0, slopes=None, window=0):
    """(value, bound) of attention of q [n, q_len, heads, d] over the host's cache."""
    n, q_len, heads, d = q.shape
    u, tiny = UNIT[q.dtype], TINY[q.dtype]
    out, off = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for s in range(n):
        K, V = host.tokens(0, rows[s], lens[s]), host.tokens(1, rows[s], lens[s])
        diag = torch.arange(q_len) + lens[s] - q_len
        j = torch.arange(lens[s])
        seen = j <= diag[:, None]
        if window:
            seen = seen & (diag[:, None] - j < window)
        group = heads // K.shape[1]
        for h in range(heads):
            x, _ = scores(q[s, :, h].cpu().double(), K[:, h // group], diag, scale, cap, float(slopes[h]) if slopes is not None else 0.0)
            p = torch.nan_to_num(torch.softmax(x.masked_fill(~seen, -math.inf), 1), 0.0) if lens[s] else torch.zeros((q_len, 0), dtype=torch.float64)
            v = V[:, h // group]
            out[s, :, h] = p @ v
            off[s, :, h] = u * out[s, :, h].abs() + (u + SLACK) * (p @ v.abs()) + tiny * (seen.double() @ v.abs())
    return out, off


# ---- tables ---------------------------------------------------------------------------------------

def fork_reference(pages, rows, lens, parent, new_lens):
    """(rows, copies, refs) of the next table by the definition."""
    need = lambda n: -(-n // PAGE)  # noqa: E731
    kept = [min(lens[p], n) if p >= 0 else 0 for p, n in zip(parent, new_lens)]
    take = [list(rows[p][:need(n)]) if p >= 0 else [] for p, n in zip(parent, kept)]
    used = {p for t in take for p in t}
    free = [p for p in range(pages) if p not in used]
    out, copies = [], []
    for r, t in enumerate(take):
        if kept[r] % PAGE:
            users = [(q, kept[q] >= (t2.index(t[-1]) + 1) * PAGE) for q, t2 in enumerate(take) if t[-1] in t2]
            if any(whole for _, whole in users) or users[0][0] != r:
                copies.append((t[-1], free[0]))
                t = t[:-1] + [free.pop(0)]
        grown = need(new_lens[r]) - len(t)
        out.append(t + [free.pop(0) for _ in range(grown)])
    refs = [0] * pages
    for t in out:
        for p in t:
            refs[p] += 1
    return out, copies, refs


def flat(rows, device="cuda"):
    ptr = [0]
    for r in rows:
        ptr.append(ptr[-1] + len(r))
    return torch.tensor(ptr, dtype=torch.int64, device=device), torch.tensor([p for r in rows for p in r], dtype=torch.int32, device=device)


def unflat(table):
    ptr, pages = table.rowptr.tolist(), table.pages.tolist()
    return [pages[a:b] for a, b in zip(ptr, ptr[1:])]
