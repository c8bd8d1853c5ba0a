"""Attention over sparse structures, as measurable cases: what a program asks of these operators, and their plain form.

  train    one attention layer's step over packed documents: the mask's structure, the forward pass and the gradients
  prefill  the forward pass alone, also with more keys than queries and with a pattern of tiles
  decode   one layer's step of serving: the newest tokens go into a cache of 8-bit pages, their queries attend to it
  fork     one step of a page table: rows are copied from others (a beam search's choice), grow, or end
  compact  the pages in use move to the front of the cache

Row i of a mask belongs to a document (q_ptr, k_ptr) and sees the keys lo <= j < hi of it: with diag = i + k_end - q_end,
hi = k_end or, where causal, max(k_begin + prefix, diag + 1), and lo = max(k_begin, diag - window + 1) where there is a
window; with a pattern, only those in tiles of 128 by 128 that it holds.  The score of a visible pair is
s = cap tanh(scale q.k / cap) - slope |diag - j|.  A row that sees nothing has the output 0 and the logarithm -inf.

A page of the cache holds 64 tokens of one sequence.  Every page and key head has a scale for the keys and one for the values: the
smallest power of two with which the largest magnitude that the page holds stays within 448; an entry x is kept as x / scale in
8 bits (e4m3, nearest, ties to even), and when a later token raises the scale, the page is rounded again.

Lengths and structures come from the case alone; values come from the seed.
"""
import functools
import math
import random

import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
TILE = 128     # rows and columns of a pattern's tiles
PAGE = 64      # tokens of a page
MOST = 448.0   # largest value of 8 bits


def listed():
    return [
        # a short document by itself, an odd length: launches and host time are what it costs
        {"name": "train_257", "op": "train", "dtype": "bf16", "layout": 1, "docs": 1, "tq": 257, "extra": 0, "hq": 4, "hkv": 4, "d": 64, "causal": True,
         "window": 0, "prefix": 0.0, "cap": 0.0, "bias": False, "tiles": 0.0},
        # a packed batch of ragged documents, grouped key heads, capped scores: the ordinary training step
        {"name": "train_docs_4096", "op": "train", "dtype": "bf16", "layout": 2, "docs": 11, "tq": 4096, "extra": 0, "hq": 16, "hkv": 4, "d": 128, "causal": True,
         "window": 0, "prefix": 0.0, "cap": 30.0, "bias": False, "tiles": 0.0},
        # a prompt that all of its document sees, distances that count against a key, 16 bits with a short exponent, sizes that divide nothing
        {"name": "train_prefix_2003", "op": "train", "dtype": "f16", "layout": 3, "docs": 3, "tq": 2003, "extra": 0, "hq": 8, "hkv": 8, "d": 64, "causal": True,
         "window": 0, "prefix": 0.4, "cap": 0.0, "bias": True, "tiles": 0.0},
        # long documents: the products of the matrices are what it costs
        {"name": "train_long_8192", "op": "train", "dtype": "bf16", "layout": 4, "docs": 2, "tq": 8192, "extra": 0, "hq": 16, "hkv": 8, "d": 128, "causal": True,
         "window": 0, "prefix": 0.0, "cap": 50.0, "bias": False, "tiles": 0.0},
        # a part of a prompt over the keys that came before it, through a pattern of tiles as a product of graphs gives it
        {"name": "prefill_tiles_5003", "op": "prefill", "dtype": "bf16", "layout": 5, "docs": 2, "tq": 5003, "extra": 6144, "hq": 32, "hkv": 8, "d": 128, "causal": True,
         "window": 0, "prefix": 0.0, "cap": 0.0, "bias": True, "tiles": 0.3},
        # one user's next token
        {"name": "decode_one_2001", "op": "decode", "dtype": "bf16", "layout": 6, "seqs": 1, "most": 2001, "least": 2001, "new": 1, "hq": 16, "hkv": 4, "d": 128,
         "window": 0, "cap": 0.0, "bias": False},
        # many users' next tokens, of any length between a few tokens and thousands
        {"name": "decode_batch_128", "op": "decode", "dtype": "bf16", "layout": 7, "seqs": 128, "most": 8192, "least": 3, "new": 1, "hq": 32, "hkv": 8, "d": 128,
         "window": 0, "cap": 30.0, "bias": False},
        # a few long contexts: one pass over a gigabyte of cache
        {"name": "decode_long_131071", "op": "decode", "dtype": "bf16", "layout": 8, "seqs": 4, "most": 131071, "least": 100000, "new": 1, "hq": 32, "hkv": 8, "d": 128,
         "window": 0, "cap": 0.0, "bias": False},
        # several proposed tokens a sequence at once, a window, distances, every head with keys of its own
        {"name": "decode_proposed_5", "op": "decode", "dtype": "f16", "layout": 9, "seqs": 16, "most": 4000, "least": 40, "new": 5, "hq": 8, "hkv": 8, "d": 64,
         "window": 1000, "cap": 0.0, "bias": True},
        # a small beam search's step: a handful of pages are copied
        {"name": "fork_beams_8", "op": "fork", "layout": 10, "rows": 8, "out": 8, "pages": 256, "most": 700, "layers": 2, "hkv": 4, "d": 64, "shared": 2, "grow": 1},
        # a server's step over many sequences with a common prompt: hundreds of copies in every layer
        {"name": "fork_rows_512", "op": "fork", "layout": 11, "rows": 384, "out": 512, "pages": 4096, "most": 1000, "layers": 4, "hkv": 8, "d": 128, "shared": 3, "grow": 1},
        # a cache of holes made whole
        {"name": "compact_2048", "op": "compact", "layout": 12, "rows": 160, "pages": 2048, "most": 1000, "layers": 4, "hkv": 8, "d": 128, "shared": 2},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["train", "train", "prefill", "decode", "decode", "fork", "compact"])
    layout = rng.randrange(1 << 20)
    d = rng.choice([64, 128, 8 * rng.randint(4, 16)])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4] + ([8] if hkv <= 2 else []))
    bias, cap = rng.random() < 0.3, rng.choice([0.0, 0.0, 30.0, 50.0])
    if op in ("train", "prefill"):
        tq = _log_int(rng, 100, 4500 if hq <= 8 else 3000)
        return {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16"]), "layout": layout, "docs": rng.randint(1, 1 + tq // 200), "tq": tq,
                "extra": rng.choice([0, rng.randint(1, 4000)]) if op == "prefill" else 0, "hq": hq, "hkv": hkv, "d": d, "causal": rng.random() < 0.85,
                "window": rng.choice([0, 0, rng.randint(10, 2000)]), "prefix": rng.choice([0.0, 0.0, 0.3]), "cap": cap, "bias": bias,
                "tiles": rng.choice([0.0, 0.0, 0.4])}
    if op == "decode":
        seqs = _log_int(rng, 1, 200)
        most = _log_int(rng, 20, min(100000, 800000 // seqs))
        new = rng.choice([1, 1, 1, rng.randint(2, 16)])
        return {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16"]), "layout": layout, "seqs": seqs, "most": max(most, new), "least": new, "new": new, "hq": hq,
                "hkv": hkv, "d": d, "window": rng.choice([0, 0, rng.randint(20, 4000)]), "cap": cap, "bias": bias}
    rows, most = _log_int(rng, 4, 200), rng.randint(40, 1000)
    case = {"op": op, "layout": layout, "rows": rows, "most": most, "pages": 64 + 2 * rows * (2 + most // PAGE), "layers": rng.randint(1, 4), "hkv": hkv, "d": d,
            "shared": rng.randint(0, 3)}
    if op == "compact":
        return case
    return case | {"out": max(1, int(rows * rng.uniform(0.3, 1.2))), "grow": rng.choice([0, 1, 1, rng.randint(2, 60)])}


# ---- structures: from the case alone --------------------------------------------------------

def _pieces(rng, total, count):
    """Bounds of `count` ragged pieces of 0 .. total."""
    return [0] + sorted(rng.randint(0, total) for _ in range(count - 1)) + [total]


def _documents(case):
    """Row pointers of the documents' queries and keys, and how many keys of each form its prompt."""
    rng = random.Random(case["layout"])
    q = _pieces(rng, case["tq"], case["docs"])
    more = _pieces(rng, case["extra"], case["docs"])
    k = [a + b for a, b in zip(q, more)]
    prompt = [int(case["prefix"] * rng.random() * 2 * (b - a)) if case["prefix"] else 0 for a, b in zip(k, k[1:])]
    return q, k, [min(p, b - a) for p, a, b in zip(prompt, k, k[1:])]


def _pattern(case):
    """Row pointer and columns of the pattern's tiles: the tiles along the diagonals, the first column, and others at random."""
    rng = random.Random(case["layout"] + 1)
    tq, tk = case["tq"], case["tq"] + case["extra"]
    nq, nk = -(-tq // TILE), -(-tk // TILE)
    ptr, cols = [0], []
    for r in range(nq):
        near = (r * TILE + tk - tq) // TILE
        cols += [c for c in range(nk) if c == 0 or near - 1 <= c <= near + 1 or rng.random() < case["tiles"]]
        ptr.append(len(cols))
    return ptr, cols


def _rows_seen(case):
    """(document's first key, lo, hi) of every query."""
    q, k, prompt = _documents(case)
    for d in range(len(prompt)):
        for i in range(q[d], q[d + 1]):
            diag = i + k[d + 1] - q[d + 1]
            lo = max(k[d], diag - case["window"] + 1) if case["window"] else k[d]
            yield lo, min(k[d + 1], max(k[d] + prompt[d], diag + 1)) if case["causal"] else k[d + 1]


def _pairs(case):
    """Visible pairs of a query and a key."""
    if not case["tiles"]:
        return sum(max(0, hi - lo) for lo, hi in _rows_seen(case))
    ptr, cols = _pattern(case)
    sums = [[0] for _ in range(len(ptr) - 1)]
    for r in range(len(ptr) - 1):
        held = set(cols[ptr[r]:ptr[r + 1]])
        for c in range(-(-(case["tq"] + case["extra"]) // TILE)):
            sums[r].append(sums[r][-1] + (TILE if c in held else 0))
    def upto(r, j):
        c = j // TILE
        return sums[r][c] + (j - c * TILE if j % TILE and sums[r][c + 1] > sums[r][c] else 0)
    return sum(upto(i // TILE, hi) - upto(i // TILE, lo) for i, (lo, hi) in enumerate(_rows_seen(case)) if hi > lo)


def _lengths(case):
    """Tokens of each sequence, the new ones among them: spread over the logarithm, the longest always there."""
    rng = random.Random(case["layout"])
    least, most = max(case["least"], case["new"]), case["most"]
    return [most if s == 0 else _log_int(rng, least, most) for s in range(case["seqs"])]


def _table(case):
    """Lengths and pages of the rows of a table; rows share their first pages with row 0 as far as both have them whole."""
    rng = random.Random(case["layout"])
    lens = [rng.randint(1, case["most"]) for _ in range(case["rows"])]
    free = list(range(case["pages"]))
    rng.shuffle(free)
    rows = []
    for length in lens:
        mine = rows[0][:min(case["shared"], length // PAGE, lens[0] // PAGE)] if rows else []
        rows.append(mine + [free.pop() for _ in range(-(-length // PAGE) - len(mine))])
    return lens, rows


def _choice(case):
    """Which row each new row continues, and its new length: some rows end, others go on several times or are cut short."""
    rng = random.Random(case["layout"] + 2)
    lens, rows = _table(case)
    parent = [rng.randrange(case["rows"]) for _ in range(case["out"])]
    if case["out"] > 2:
        parent[1] = -1                                      # a new row
    new = [max(1, (lens[p] if p >= 0 else 0) + (case["grow"] if rng.random() < 0.9 else -rng.randint(0, 80))) for p in parent]
    return lens, rows, parent, new


def _forked(case):
    """The new table, (from, to) of the pages that are copied, and how often each page is used: the definition, row by row."""
    lens, rows, parent, new = _choice(case)
    keep, whole, first = [], set(), {}
    for r, p in enumerate(parent):
        kept = min(lens[p], new[r]) if p >= 0 else 0
        pages = rows[p][:-(-kept // PAGE)] if p >= 0 else []
        keep.append((kept, pages))
        whole.update(pages[:kept // PAGE])
        if kept % PAGE:
            first.setdefault(pages[-1], r)
    free = iter(sorted(set(range(case["pages"])) - {p for _, pages in keep for p in pages}))
    out, moved = [], []
    for r, (kept, pages) in enumerate(keep):
        mine = list(pages)
        if kept % PAGE and (pages[-1] in whole or first[pages[-1]] != r):
            mine[-1] = next(free)
            moved.append((pages[-1], mine[-1]))
        while len(mine) < -(-new[r] // PAGE):
            mine.append(next(free))
        out.append(mine)
    refs = [0] * case["pages"]
    for pages in out:
        for p in pages:
            refs[p] += 1
    return out, moved, refs


def _compacted(case):
    _, rows = _table(case)
    live = sorted({p for row in rows for p in row})
    held = set(live)
    holes = [p for p in range(len(live)) if p not in held]
    moved = list(zip([p for p in live if p >= len(live)], holes))
    to = dict(moved)
    return [[to.get(p, p) for p in row] for row in rows], moved, len(live)


# ---- inputs: values from the seed ------------------------------------------------------------

def _flat(rows):
    ptr = [0]
    for row in rows:
        ptr.append(ptr[-1] + len(row))
    return _ints(ptr, torch.int64), _ints([p for row in rows for p in row], torch.int32)


def _ints(values, dtype):
    return torch.tensor(values, dtype=dtype).to(DEVICE)


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(dtype)


def _slopes(heads):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], dtype=torch.float32).to(DEVICE)


def _padded(d):
    return 64 if d <= 64 else 128


def _cache(gen, case, layers, pages):
    """Keys page by page as [token, channel], values as [channel, token]; channels up to 64 or 128, the ones past the head's are zero."""
    hkv, d, room = case["hkv"], case["d"], _padded(case["d"])
    keys = torch.zeros((layers, pages, hkv, PAGE, room), dtype=torch.uint8, device=DEVICE)
    values = torch.zeros((layers, pages, hkv, room, PAGE), dtype=torch.uint8, device=DEVICE)
    for layer in range(layers):
        keys[layer, ..., :d] = (torch.randn((pages, hkv, PAGE, d), generator=gen, device=DEVICE) * 70).clamp(-MOST, MOST).to(torch.float8_e4m3fn).view(torch.uint8)
        values[layer, ..., :d, :] = (torch.randn((pages, hkv, d, PAGE), generator=gen, device=DEVICE) * 70).clamp(-MOST, MOST).to(torch.float8_e4m3fn).view(torch.uint8)
    scale = [torch.exp2(torch.randint(-8, -5, (layers, pages, hkv), generator=gen, device=DEVICE).float()) for _ in range(2)]
    return {"k": keys, "v": values, "k_scale": scale[0], "v_scale": scale[1]}


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    s = dict(case, case=dict(case))
    if case["op"] in ("train", "prefill"):
        dtype, d = TYPES[case["dtype"]], case["d"]
        q_ptr, k_ptr, prompt = _documents(case)
        s["k_len"] = case["tq"] + case["extra"]
        s |= {"q_ptr": _ints(q_ptr, torch.int64), "k_ptr": _ints(k_ptr, torch.int64), "prompt": _ints(prompt, torch.int64) if case["prefix"] else None}
        s["pattern"] = tuple(_ints(x, t) for x, t in zip(_pattern(case), (torch.int64, torch.int32))) if case["tiles"] else None
        s["q"] = _normal(gen, (case["tq"], case["hq"], d), dtype, 1.5)
        s["k"] = _normal(gen, (s["k_len"], case["hkv"], d), dtype, 1.5)
        s["v"] = _normal(gen, (s["k_len"], case["hkv"], d), dtype)
        s["do"] = _normal(gen, (case["tq"], case["hq"], d), dtype) if case["op"] == "train" else None
    elif case["op"] == "decode":
        dtype, n, new, d = TYPES[case["dtype"]], case["seqs"], case["new"], case["d"]
        lens = _lengths(case)
        s["most_pages"] = max(-(-x // PAGE) for x in lens)
        need = sum(-(-x // PAGE) for x in lens)
        ids = torch.randperm(need + 8, generator=gen, device=DEVICE).to(torch.int32)   # pages anywhere in the cache
        ptr = [0]
        for x in lens:
            ptr.append(ptr[-1] + -(-x // PAGE))
        s |= {"rowptr": _ints(ptr, torch.int64), "table": ids[:need].contiguous(), "lens": _ints(lens, torch.int32),
              "new_ptr": _ints([new * i for i in range(n + 1)], torch.int64), "cache": _cache(gen, case, 1, need + 8)}
        s["q"] = _normal(gen, (n, new, case["hq"], d), dtype, 1.5)
        s["k"] = _normal(gen, (n * new, case["hkv"], d), dtype, 1.5)
        s["v"] = _normal(gen, (n * new, case["hkv"], d), dtype)
    else:
        lens, rows = _table(case)
        s["rowptr"], s["table"] = _flat(rows)
        s["lens"], s["cache"] = _ints(lens, torch.int32), _cache(gen, case, case["layers"], case["pages"])
        if case["op"] == "fork":
            _, _, parent, new = _choice(case)
            s["out_pages"] = sum(-(-x // PAGE) for x in new)
            s["parent"], s["new_lens"] = _ints(parent, torch.int32), _ints(new, torch.int32)
    if case.get("bias"):
        s["slopes"] = _slopes(case["hq"])
    else:
        s["slopes"] = None
    return s


# ---- the plain form ---------------------------------------------------------------------------

def _bounds(s):
    """lo, hi and diag of every query."""
    i = torch.arange(s["tq"], device=DEVICE)
    doc = torch.searchsorted(s["q_ptr"][1:].contiguous(), i, right=True)
    begin, end = s["k_ptr"][:-1][doc], s["k_ptr"][1:][doc]
    diag = i + end - s["q_ptr"][1:][doc]
    first = begin + s["prompt"][doc] if s["prompt"] is not None else begin
    hi = torch.minimum(end, torch.maximum(first, diag + 1)) if s["causal"] else end
    lo = torch.maximum(begin, diag - s["window"] + 1) if s["window"] else begin
    return lo, hi, diag


def _visible(s):
    lo, hi, diag = _bounds(s)
    j = torch.arange(s["k_len"], device=DEVICE)
    seen = (j >= lo[:, None]) & (j < hi[:, None])
    if s["pattern"] is not None:
        ptr, cols = s["pattern"]
        held = torch.zeros((ptr.numel() - 1, -(-s["k_len"] // TILE)), dtype=torch.bool, device=DEVICE)
        held[torch.repeat_interleave(torch.arange(ptr.numel() - 1, device=DEVICE), ptr[1:] - ptr[:-1], output_size=cols.numel()), cols.long()] = True
        seen &= held[torch.arange(s["tq"], device=DEVICE) // TILE][:, j // TILE]
    return seen, (diag[:, None] - j).abs()


def _softmax(s, score, seen):
    """Probabilities and the logarithm of their sum over the last axis; a row that sees nothing has 0 and -inf."""
    score = score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    base = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - base)
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, 1.0, total), (base + torch.log(total)).squeeze(-1)


def _plain_attention(s):
    group, scale, cap = s["hq"] // s["hkv"], 1.0 / math.sqrt(s["d"]), s["cap"]
    q = s["q"].float().transpose(0, 1).contiguous()
    k = s["k"].float().transpose(0, 1).repeat_interleave(group, 0)
    v = s["v"].float().transpose(0, 1).repeat_interleave(group, 0)
    seen, distance = _visible(s)
    score = torch.matmul(q, k.transpose(1, 2)) * scale
    if cap:
        bent = torch.tanh(score / cap)
        score = cap * bent
    if s["slopes"] is not None:
        score = score - s["slopes"][:, None, None] * distance
    p, lse = _softmax(s, score, seen)
    del score
    o = torch.matmul(p, v)
    out = {"o": o.transpose(0, 1).to(s["q"].dtype).contiguous(), "lse": lse}
    if s["op"] == "prefill":
        return out
    do = s["do"].float().transpose(0, 1).contiguous()
    dv = torch.matmul(p.transpose(1, 2), do)
    ds = p * (torch.matmul(do, v.transpose(1, 2)) - (do * o).sum(-1, keepdim=True))
    if cap:
        ds *= 1 - bent * bent
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(1, 2), q) * scale
    shared = lambda g: g.view(s["hkv"], group, s["k_len"], s["d"]).sum(1).transpose(0, 1).to(s["k"].dtype).contiguous()  # noqa: E731
    return out | {"dq": dq.transpose(0, 1).to(s["q"].dtype).contiguous(), "dk": shared(dk), "dv": shared(dv)}


def _scale_for(most):
    """The smallest power of two that brings `most` to 448 or less."""
    part, power = torch.frexp(most / MOST)
    return torch.ldexp(torch.ones_like(most), torch.where(part == 0.5, power - 1, power).clamp(-100, 120))


def _append(s, pages, scales, new, tokens_last):
    """The new tokens of every sequence into its last pages (two at most are touched), rounded again where the scale rises."""
    n, count, d = s["seqs"], s["new"], s["d"]
    start = s["lens"].long() - count
    slot = torch.stack([start // PAGE, (start + count - 1) // PAGE], 1)                        # [n, 2]
    ids = s["table"].long()[s["rowptr"][:-1, None] + slot]
    pos = start[:, None] + torch.arange(count, device=DEVICE)
    old = pages[0][ids].view(torch.float8_e4m3fn).float()                                     # [n, 2, heads, ...]
    if tokens_last:
        old = old.transpose(-1, -2)
    x = new.float().view(n, count, s["hkv"], d)
    inside = (pos[:, None, :] // PAGE == slot[:, :, None]).float()                            # [n, 2, new]
    most = (x.abs().amax(-1)[:, None] * inside[..., None]).amax(2)                            # [n, 2, heads]
    had = (slot * PAGE < start[:, None])[..., None]
    before = scales[0][ids]
    need = torch.where(most > 0, _scale_for(most), 2.0 ** -100)
    scale = torch.where(had, torch.maximum(before, need), need)
    ratio = torch.where(had, before, 0.0) / scale
    kept = (old * ratio[..., None, None]).clamp(-MOST, MOST)
    at_token = (slot[..., None] * PAGE + torch.arange(PAGE, device=DEVICE))[:, :, None, :, None]
    before_new, after_new = at_token < start[:, None, None, None, None], at_token >= s["lens"].long()[:, None, None, None, None]
    at = (pos[:, None, :] - slot[:, :, None] * PAGE).clamp(0, PAGE - 1)                       # [n, 2, new]
    put = torch.zeros((n, 2, PAGE, count), device=DEVICE).scatter_(2, at[:, :, None, :], inside[:, :, None, :])
    whole = torch.einsum("nspc,nchd->nshpd", put, x) / scale[..., None, None]
    kept[..., :d] = torch.where(before_new, kept[..., :d], whole)
    byte = torch.where(after_new, old, kept.clamp(-MOST, MOST)).to(torch.float8_e4m3fn).view(torch.uint8)   # what is behind the last token stays
    pages[0][ids] = byte.transpose(-1, -2).contiguous() if tokens_last else byte
    scales[0][ids] = scale


def _plain_decode(s):
    n, count, hkv, d, group, scale, cap = s["seqs"], s["new"], s["hkv"], s["d"], s["hq"] // s["hkv"], 1.0 / math.sqrt(s["d"]), s["cap"]
    c = s["cache"]
    _append(s, c["k"], c["k_scale"], s["k"], False)
    _append(s, c["v"], c["v_scale"], s["v"], True)
    slots = torch.arange(s["most_pages"], device=DEVICE)
    have = slots < (s["rowptr"][1:] - s["rowptr"][:-1])[:, None]
    ids = torch.where(have, s["table"].long()[(s["rowptr"][:-1, None] + slots).clamp(max=s["table"].numel() - 1)], 0)
    long = s["most_pages"] * PAGE
    k = c["k"][0][ids].view(torch.float8_e4m3fn)[..., :d].float() * c["k_scale"][0][ids][..., None, None]        # [n, pages, heads, 64, d]
    v = c["v"][0][ids].view(torch.float8_e4m3fn)[..., :d, :].float() * c["v_scale"][0][ids][..., None, None]
    k = k.transpose(1, 2).reshape(n, hkv, long, d)
    v = v.permute(0, 2, 1, 4, 3).reshape(n, hkv, long, d)
    q = s["q"].float().view(n, count, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, count * group, d)
    score = (torch.matmul(q, k.transpose(2, 3)) * scale).view(n, hkv, count, group, long)
    if cap:
        score = cap * torch.tanh(score / cap)
    diag = (s["lens"].long()[:, None] - count + torch.arange(count, device=DEVICE))[:, None, :, None, None]
    j = torch.arange(long, device=DEVICE)
    seen = j <= diag
    if s["window"]:
        seen = seen & (diag - j < s["window"])
    if s["slopes"] is not None:
        score = score - s["slopes"].view(hkv, 1, group, 1) * (diag - j).abs()
    p, _ = _softmax(s, score, seen)
    o = torch.matmul(p.view(n, hkv, count * group, long), v).view(n, hkv, count, group, d)
    return {"o": o.permute(0, 2, 1, 3, 4).reshape(n, count, s["hq"], d).to(s["q"].dtype), "k": c["k"].view(torch.float8_e4m3fn), "k_scale": c["k_scale"],
            "v": c["v"].view(torch.float8_e4m3fn), "v_scale": c["v_scale"]}


def _copy(cache, src, dst):
    for part in cache.values():
        part[:, dst] = part[:, src]


def _cache_out(c):
    return {"k": c["k"].view(torch.float8_e4m3fn), "k_scale": c["k_scale"], "v": c["v"].view(torch.float8_e4m3fn), "v_scale": c["v_scale"]}


def _plain_fork(s):
    n, pages, parent = s["out"], s["pages"], s["parent"].long()
    old = parent.clamp(min=0)
    kept = torch.where(parent >= 0, torch.minimum(s["lens"].long()[old], s["new_lens"].long()), 0)
    ptr = torch.zeros(n + 1, dtype=torch.int64, device=DEVICE)
    torch.cumsum((s["new_lens"].long() + PAGE - 1) // PAGE, 0, out=ptr[1:])
    row = torch.repeat_interleave(torch.arange(n, device=DEVICE), ptr[1:] - ptr[:-1], output_size=s["out_pages"])
    slot = torch.arange(s["out_pages"], device=DEVICE) - ptr[row]
    has = slot < (kept[row] + PAGE - 1) // PAGE
    page = torch.where(has, s["table"].long()[torch.where(has, s["rowptr"][old[row]] + slot, 0)], pages)
    ends = has & ((slot + 1) * PAGE > kept[row])
    owner = torch.full((pages + 1,), n, dtype=torch.int64, device=DEVICE).scatter_reduce(0, page, torch.where(ends, row, -1), "amin")
    copied = ends & (owner[page] != row)
    used = torch.zeros(pages + 1, dtype=torch.int64, device=DEVICE).scatter_add(0, page, torch.ones_like(page))
    fresh = copied | ~has
    free = torch.sort((used[:pages] > 0).to(torch.int8), stable=True).indices
    out = torch.where(fresh, free[torch.cumsum(fresh, 0) - 1], page)
    refs = torch.zeros(pages, dtype=torch.int32, device=DEVICE).scatter_add(0, out, torch.ones_like(out, dtype=torch.int32))
    # at most one page a row is copied, how many is not known on the host: the others of as many copy onto themselves
    which = torch.sort((~copied).to(torch.int8), stable=True).indices[:n]
    mine = copied[which]
    _copy(s["cache"], torch.where(mine, page[which], out[which]).clamp(max=pages - 1), out[which])
    return {"rowptr": ptr, "pages": out.to(torch.int32), "refs": refs} | _cache_out(s["cache"])


def _plain_compact(s):
    pages, table = s["pages"], s["table"].long()
    live = torch.zeros(pages, dtype=torch.bool, device=DEVICE).scatter_(0, table, True)
    count = live.sum()
    at = torch.arange(pages, device=DEVICE)
    moves, holes = live & (at >= count), ~live & (at < count)
    hole = torch.sort((~holes).to(torch.int8), stable=True).indices
    to = torch.where(moves, hole[(torch.cumsum(moves, 0) - 1).clamp(min=0)], at)
    which = torch.sort((~moves).to(torch.int8), stable=True).indices[:pages // 2]
    src = torch.where(moves[which], which, pages - 1)                                          # the last page is never a hole's place
    dst = torch.where(moves[which], to[which], pages - 1)
    _copy(s["cache"], src, dst)
    return {"pages": to[table].to(torch.int32), "live": count.to(torch.int64)} | _cache_out(s["cache"])


# ---- the framework's operators -----------------------------------------------------------------

@functools.lru_cache(None)
def _library():
    from paper_2404_04541_amd import attention, binding
    return attention, binding.Handle()


def _own_cache(at, s):
    c = s["cache"]
    return at.PagedCache(s["d"], c["k"], c["v"], c["k_scale"], c["v_scale"])


def _own(s):
    at, h = _library()
    if s["op"] in ("train", "prefill"):
        plan = at.symbolic(h, s["tq"], s["k_len"], q_ptr=s["q_ptr"], k_ptr=s["k_ptr"], prefix=s["prompt"], causal=s["causal"], window=s["window"], tiles=s["pattern"],
                           check=False)   # (the loader's own row pointers)
        o, lse = at.forward(h, plan, s["q"], s["k"], s["v"], cap=s["cap"], slopes=s["slopes"])
        out = {"o": o, "lse": lse}
        if s["op"] == "prefill":
            return out
        dq, dk, dv = at.backward(h, plan, s["q"], s["k"], s["v"], o, lse, s["do"], cap=s["cap"], slopes=s["slopes"])
        return out | {"dq": dq, "dk": dk, "dv": dv}
    table = at.PageTable(s["rowptr"], s["table"])
    cache = _own_cache(at, s)
    if s["op"] == "decode":
        at.append(h, cache, 0, table, s["lens"], s["new_ptr"], s["k"], s["v"])
        o = at.attend(h, cache, 0, table, s["lens"], s["q"], cap=s["cap"], slopes=s["slopes"], window=s["window"])
        return {"o": o} | _cache_out(s["cache"])
    if s["op"] == "fork":
        out, refs = at.fork(h, cache, table, s["lens"], s["parent"], s["new_lens"], s["out_pages"])
        return {"rowptr": out.rowptr, "pages": out.pages, "refs": refs} | _cache_out(s["cache"])
    out, live = at.compact(h, cache, table)
    return {"pages": out.pages, "live": live} | _cache_out(s["cache"])


def run(state):
    if own:
        return _own(state)
    if state["op"] in ("train", "prefill"):
        return _plain_attention(state)
    return {"decode": _plain_decode, "fork": _plain_fork, "compact": _plain_compact}[state["op"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    if case["op"] in ("train", "prefill"):
        pairs, tk, d = _pairs(case), case["tq"] + case["extra"], case["d"]
        q, k = 2 * case["tq"] * case["hq"] * d, 2 * tk * case["hkv"] * d
        if case["op"] == "prefill":
            return {"bytes": 2 * q + 2 * k + 4 * case["tq"] * case["hq"], "flops": 4 * pairs * case["hq"] * d}
        return {"bytes": 4 * q + 4 * k + 4 * case["tq"] * case["hq"], "flops": 12 * pairs * case["hq"] * d}   # six products, none of them twice
    room = _padded(case["d"])
    if case["op"] == "decode":
        seen = [min(x, case["window"] + case["new"] - 1) if case["window"] else x for x in _lengths(case)]
        tokens, new, row = sum(seen), case["seqs"] * case["new"], case["d"] * case["hkv"]
        return {"bytes": 2 * tokens * row + 4 * 2 * case["hkv"] * sum(-(-x // PAGE) for x in seen) + 4 * new * row + 4 * new * case["hq"] * case["d"],
                "flops": 4 * tokens * case["new"] * case["hq"] * case["d"]}
    page = case["layers"] * case["hkv"] * (2 * PAGE * room + 8)
    if case["op"] == "fork":
        out, moved, _ = _forked(case)
        return {"bytes": 2 * page * len(moved) + 8 * sum(len(r) for r in out) + 4 * case["pages"] + 16 * case["out"], "flops": 0}
    out, moved, _ = _compacted(case)
    return {"bytes": 2 * page * len(moved) + 8 * sum(len(r) for r in out) + 4 * case["pages"], "flops": 0}


# ---- the definition in 64 bits --------------------------------------------------------------------

def _exact_attention(case, s):
    tq, tk, hq, group, d, cap = case["tq"], s["k_len"], case["hq"], case["hq"] // case["hkv"], case["d"], case["cap"]
    rows = list(_rows_seen(case))
    q_ptr, k_ptr, _ = _documents(case)
    diag = torch.cat([torch.arange(a, b) + ke - b for a, b, ke in zip(q_ptr, q_ptr[1:], k_ptr[1:])]).to(DEVICE)
    lo, hi = (torch.tensor([r[x] for r in rows], dtype=torch.int64).to(DEVICE) for x in (0, 1))
    ptr, cols = _pattern(case) if case["tiles"] else ([], [])
    out = {"o": torch.zeros((tq, hq, d), dtype=torch.float64, device=DEVICE), "lse": torch.full((hq, tq), -math.inf, dtype=torch.float64, device=DEVICE)}
    if case["op"] == "train":
        out |= {"dq": torch.zeros_like(out["o"]), "dk": torch.zeros((tk, case["hkv"], d), dtype=torch.float64, device=DEVICE),
                "dv": torch.zeros((tk, case["hkv"], d), dtype=torch.float64, device=DEVICE)}
    j = torch.arange(tk, device=DEVICE)
    for first in range(0, tq, TILE):
        at = slice(first, min(tq, first + TILE))
        seen = (lo[at, None] <= j) & (j < hi[at, None])
        if case["tiles"]:
            held = torch.zeros(-(-tk // TILE), dtype=torch.bool)
            held[cols[ptr[first // TILE]:ptr[first // TILE + 1]]] = True
            seen &= held.to(DEVICE).repeat_interleave(TILE)[:tk]
        some = torch.nonzero(seen.any(0)).flatten()
        if not some.numel():
            continue
        a, b = int(some[0]), int(some[-1]) + 1
        far = (diag[at, None] - j[a:b]).abs()
        for h in range(hq):
            q, k, v = s["q"][at, h].double(), s["k"][a:b, h // group].double(), s["v"][a:b, h // group].double()
            raw = q @ k.T / math.sqrt(d)
            bent = torch.tanh(raw / cap) if cap else None
            x = cap * bent if cap else raw
            if s["slopes"] is not None:
                x = x - s["slopes"][h].double() * far
            x = torch.where(seen[:, a:b], x, -math.inf)
            lse = torch.logsumexp(x, 1)
            p = torch.where(seen[:, a:b], torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
            o = p @ v
            out["o"][at, h], out["lse"][h, at] = o, lse
            if case["op"] == "train":
                do = s["do"][at, h].double()
                g = p * (do @ v.T - (do * o).sum(1, keepdim=True))
                g = (g * (1 - bent ** 2) if cap else g) / math.sqrt(d)
                out["dq"][at, h] = g @ k
                out["dk"][a:b, h // group] += g.T @ q
                out["dv"][a:b, h // group] += p.T @ do
    return out


def _exact_decode(case, s):
    n, new, hkv, d, group, cap = case["seqs"], case["new"], case["hkv"], case["d"], case["hq"] // case["hkv"], case["cap"]
    lens, ptr, table = _lengths(case), s["rowptr"].tolist(), s["table"].tolist()
    c = s["cache"]
    held = {"k": c["k"][0].view(torch.float8_e4m3fn).double(), "v": c["v"][0].view(torch.float8_e4m3fn).double().transpose(-1, -2)}   # [pages, heads, 64, room]
    scale = {x: c[x + "_scale"][0].double() for x in "kv"}
    out = torch.zeros((n, new, case["hq"], d), dtype=torch.float64, device=DEVICE)
    for i in range(n):
        pages = table[ptr[i]:ptr[i + 1]]
        for x in "kv":
            fresh = s[x].view(n, new, hkv, d)[i].double()
            pos = lens[i] - new
            while pos < lens[i]:
                page, end = pages[pos // PAGE], min(lens[i], (pos // PAGE + 1) * PAGE)
                part, off = fresh[pos - lens[i] + new:end - lens[i] + new], pos % PAGE
                need = torch.exp2(torch.ceil(torch.log2(part.abs().amax((0, 2)) / MOST)))
                now = torch.maximum(scale["kv"[x == "v"]][page], need) if off else need
                old = held[x][page, :, :off] * (scale[x][page] / now)[:, None, None]
                held[x][page, :, :off] = old.to(torch.float32).to(torch.float8_e4m3fn).double()
                fitted = (part / now[None, :, None]).to(torch.float32).to(torch.float8_e4m3fn).double()
                held[x][page, :, off:off + end - pos, :d] = fitted.transpose(0, 1)
                scale[x][page] = now
                pos = end
        ids = torch.tensor(pages).to(DEVICE)
        k, v = ((held[x][ids] * scale[x][ids][..., None, None])[..., :d].transpose(0, 1).reshape(hkv, -1, d) for x in "kv")
        far = torch.arange(lens[i] - new, lens[i], device=DEVICE)[:, None] - torch.arange(k.shape[1], device=DEVICE)
        seen = (far >= 0) & (far < case["window"]) if case["window"] else far >= 0
        for h in range(case["hq"]):
            x = s["q"][i, :, h].double() @ k[h // group].T / math.sqrt(d)
            x = cap * torch.tanh(x / cap) if cap else x
            x = x - s["slopes"][h].double() * far if s["slopes"] is not None else x
            out[i, :, h] = torch.softmax(torch.where(seen, x, -math.inf), 1) @ v[h // group]
    return {"o": out, "k": held["k"][None], "k_scale": scale["k"][None], "v": held["v"].transpose(-1, -2).contiguous()[None], "v_scale": scale["v"][None]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("train", "prefill"):
        return _exact_attention(case, s)
    if case["op"] == "decode":
        return _exact_decode(case, s)
    rows, moved, more = _forked(case) if case["op"] == "fork" else _compacted(case)
    src, dst = ([m[x] for m in moved] for x in (0, 1))
    cache = {}
    for name, part in s["cache"].items():
        part[:, dst] = part[:, src].clone()
        cache[name] = (part.view(torch.float8_e4m3fn) if part.dtype == torch.uint8 else part).double()
    ptr, pages = _flat(rows)
    return {"pages": pages} | ({"rowptr": ptr, "refs": _ints(more, torch.int32)} if case["op"] == "fork" else {"live": _ints(more, torch.int64)}) | cache
