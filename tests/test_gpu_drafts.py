"""Trees of drafted tokens over the paged cache: attention against 64 bits, verification token by token, what keeping a path leaves in the pages (bit for bit), tokens read back."""
import ctypes as C
import math
import random

import pytest
import torch

from attn_helpers import MOST, PAGE, HostCache, check, flat, room_of
from draft_helpers import ancestors, keep_reference, tree_reference, verify_reference
from paper_2404_04541_amd import attention as at
from paper_2404_04541_amd import binding as sg
from paper_2404_04541_amd import drafts as dr

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def h():
    return sg.Handle()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def i64(values):
    return torch.tensor(values, dtype=torch.int64, device="cuda")


def randn(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def filled(seed, layers, pages, heads, d):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    room = room_of(d)
    code = lambda *s: (torch.randn(s, generator=gen, device="cuda") * 60).clamp(-MOST, MOST).to(torch.float8_e4m3fn).view(torch.uint8)  # noqa: E731
    scale = [torch.exp2(torch.randint(-8, -4, (layers, pages, heads), generator=gen, device="cuda").float()) for _ in range(2)]
    return at.PagedCache(d, code(layers, pages, heads, PAGE, room), code(layers, pages, heads, room, PAGE), *scale)


def rows_for(lens, pages, seed=0, spare=0):
    rng = random.Random(seed)
    ids = rng.sample(range(pages), pages)
    return [[ids.pop() for _ in range(-(-n // PAGE) + spare)] for n in lens]


def clone(c):
    return at.PagedCache(c.head_dim, c.k.clone(), c.v.clone(), c.k_scale.clone(), c.v_scale.clone())


def grown(n, seed, width=3, roots=1):
    """A tree of n nodes in the order of their parents."""
    rng = random.Random(seed)
    parent = [-1] * min(n, roots)
    for i in range(len(parent), n):
        parent.append(rng.randint(max(0, i - 3 * width), i - 1))
    return sorted(parent)


def sums(counts):
    ptr = [0]
    for c in counts:
        ptr.append(ptr[-1] + c)
    return ptr


def planned(h, trees, most=None, check=True):
    return dr.symbolic(h, i64(sums(map(len, trees))), i32([p for t in trees for p in t]), most or max(max(map(len, trees)), 1), check=check)


# ---- attention ------------------------------------------------------------------------------------

CASES = {
    "one_node": dict(lens=[1], trees=[[-1]], heads=(1, 1), d=64),
    "no_context": dict(lens=[7, 3], trees=[grown(7, 1), [-1, -1, -1]], heads=(2, 1), d=64),
    "ragged": dict(lens=[70, 64, 0, 129, 40, 200], trees=[grown(5, 2), [-1], [], grown(26, 3), [], grown(60, 4)], heads=(4, 2), d=64),
    "chain": dict(lens=[150, 64], trees=[list(range(-1, 9)), list(range(-1, 63))], heads=(8, 2), d=128),
    "chunks": dict(lens=[3000, 2100, 65], trees=[grown(12, 5), grown(3, 6), grown(9, 7)], heads=(8, 2), d=128),
    "most": dict(lens=[500, 256, 300], trees=[grown(256, 8, 4), grown(256, 9, 2), grown(200, 10, 30)], heads=(4, 2), d=64),
    "two_blocks": dict(lens=[1000], trees=[grown(12, 11)], heads=(10, 2), d=128),
    "group_of_24": dict(lens=[200, 70], trees=[grown(9, 12), grown(30, 13)], heads=(24, 1), d=72),
    "group_of_160": dict(lens=[70, 3], trees=[grown(3, 38), [-1, -1]], heads=(160, 1), d=64),
    "wide_roots": dict(lens=[90, 66], trees=[grown(20, 14, 3, 5), grown(33, 15, 8, 33)], heads=(4, 4), d=64),
    "window": dict(lens=[1000, 64, 40, 300], trees=[grown(17, 16, 1), grown(8, 17), grown(30, 18), []], heads=(4, 2), d=64, window=70),
    "window_in_tree": dict(lens=[130, 128, 100], trees=[list(range(-1, 39)), grown(70, 19, 1), grown(20, 20)], heads=(2, 1), d=64, window=3),
    "window_one": dict(lens=[130, 9], trees=[grown(20, 21), grown(9, 22)], heads=(2, 1), d=128, window=1),
    "cap": dict(lens=[700, 90], trees=[grown(10, 23), grown(40, 24)], heads=(8, 4), d=128, cap=10.0),
    "bias": dict(lens=[700, 90, 140], trees=[grown(10, 25), grown(40, 26), grown(100, 27, 2)], heads=(4, 2), d=64, slopes=[0.5, 0.01, 0.0, 0.1]),
    "bias_128": dict(lens=[400, 190], trees=[grown(60, 28), grown(130, 29, 2)], heads=(4, 2), d=128, slopes=[0.2, 0.01, 0.0, 0.1]),
    "cap_bias_window": dict(lens=[333, 80], trees=[grown(50, 30, 2), grown(33, 31)], heads=(4, 2), d=40, slopes=[0.5, 0.01, 0.0, 0.1], cap=6.0, window=100),
    "small_head": dict(lens=[77], trees=[grown(11, 32)], heads=(2, 1), d=8),
    "more_nodes_than_tokens": dict(lens=[3, 0, 70], trees=[grown(8, 33), grown(4, 34), grown(70, 35)], heads=(2, 2), d=64),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
def test_attend(h, name, dtype):
    c = CASES[name]
    (heads, kv), d, lens, trees = c["heads"], c["d"], c["lens"], c["trees"]
    pages = sum(-(-n // PAGE) for n in lens) + 3
    cache = filled(8, 2, pages, kv, d)
    rows = rows_for(lens, pages, 1)
    for pages_of, n in zip(rows, lens):      # behind the last token: NaN
        if n % PAGE:
            cache.k[1, pages_of[-1], :, n % PAGE:] = 0x7F
            cache.v[1, pages_of[-1], :, :, n % PAGE:] = 0xFF
    cache.k[..., d:], cache.v[..., d:, :] = 0x7F, 0xFF      # ... and behind the head's channels
    gen = torch.Generator(device="cuda").manual_seed(9)
    q = randn(gen, (sum(map(len, trees)), heads, d), dtype, 1.5)
    slopes = torch.tensor(c["slopes"], device="cuda") if "slopes" in c else None
    o = dr.attend(h, cache, 1, at.PageTable(*flat(rows)), i32(lens), planned(h, trees), q, cap=c.get("cap", 0.0), slopes=slopes, window=c.get("window", 0))
    check(name, o, *tree_reference(HostCache(cache, 1), rows, lens, trees, q, 1 / math.sqrt(d), c.get("cap", 0.0), slopes, c.get("window", 0)))


@pytest.mark.parametrize("seqs, longest", [(64, 3000), (65, 700), (200, 2000), (512, 1500), (513, 1500), (700, 40)])
def test_attend_many_sequences(h, seqs, longest):
    """Sequences of all lengths, some without a tree or without tokens: long ones among them are cut, and which workgroup has what is found in several steps, or by the table's row pointers."""
    rng = random.Random(seqs)
    trees = [grown(rng.choice([0, 1, 2, rng.randint(3, 40)]), 300 + s) for s in range(seqs)]
    lens = [longest if s % 97 == 5 else len(t) + rng.choice([0, rng.randint(0, 100)]) if s % 11 else 0 for s, t in enumerate(trees)]
    pages = sum(-(-n // PAGE) for n in lens) + 2
    cache, rows = filled(48, 1, pages, 2, 64), rows_for(lens, pages, 3)
    gen = torch.Generator(device="cuda").manual_seed(49)
    q = randn(gen, (sum(map(len, trees)), 8, 64), BF, 1.5)
    o = dr.attend(h, cache, 0, at.PageTable(*flat(rows)), i32(lens), planned(h, trees), q)
    check("o", o, *tree_reference(HostCache(cache, 0), rows, lens, trees, q, 1 / 8))


def test_attend_row_pointers_that_do_not_ascend(h):
    """A table whose rows overlap and fall back: what that gives is not said, but nothing outside of what the call has is written."""
    cache = filled(37, 1, 40, 2, 64)
    before = clone(cache)
    gen = torch.Generator(device="cuda").manual_seed(38)
    trees = [grown(20, 39)] * 6
    out = torch.full((140, 4, 64), 7.0, dtype=BF, device="cuda")
    q, plan, lens = randn(gen, (120, 4, 64), BF), planned(h, trees), i32([2560] * 6)
    table = at.PageTable(i64([0, 40, 0, 40, -9, 90, 40]), i32(list(range(40))))
    rc = dr._lib().spdraft_attend(h.ptr, C.byref(cache._struct), 0, C.byref(table.struct(cache)), lens.data_ptr(), C.byref(plan._struct), plan.memory.data_ptr(), 4, at.BF16, 0.125, 0.0, None, 0,
                                  at._tensor(q, "q"), at.TensorStruct(out.data_ptr(), 256, 64))
    torch.cuda.synchronize()
    assert rc == 0 and (out[120:] == 7.0).all() and torch.equal(cache.k, before.k) and torch.equal(cache.v, before.v)


@pytest.mark.parametrize("most", [9, 64, 65, 256])
def test_attend_most_is_a_bound(h, most):
    """A larger `most` than any tree has changes nothing but memory."""
    trees, lens = [grown(9, 40), grown(4, 41)], [300, 66]
    cache, rows = filled(42, 1, 12, 2, 64), rows_for([300, 66], 12)
    gen = torch.Generator(device="cuda").manual_seed(43)
    q = randn(gen, (13, 4, 64), BF)
    o = dr.attend(h, cache, 0, at.PageTable(*flat(rows)), i32(lens), planned(h, trees, most), q)
    check("o", o, *tree_reference(HostCache(cache, 0), rows, lens, trees, q, 1 / 8))


def test_attend_strides(h):
    """Queries that are a part of a larger tensor, and a layout of heads before tokens."""
    trees, lens = [grown(9, 44), grown(20, 45)], [150, 80]
    cache, rows = filled(46, 1, 12, 2, 72), rows_for(lens, 12)
    gen = torch.Generator(device="cuda").manual_seed(47)
    table, plan = at.PageTable(*flat(rows)), planned(h, trees)
    whole = randn(gen, (29, 3, 4, 80), BF)
    turned = randn(gen, (4, 29, 72), BF).transpose(0, 1)
    for q in (whole[:, 1, :, :72], turned):
        o = dr.attend(h, cache, 0, table, i32(lens), plan, q)
        assert torch.equal(o, dr.attend(h, cache, 0, table, i32(lens), plan, q.contiguous()))
        check("o", o, *tree_reference(HostCache(cache, 0), rows, lens, trees, q, 1 / math.sqrt(72)))


@pytest.mark.parametrize("d", [64, 128])
def test_attend_what_is_not_seen_is_not_felt(h, d):
    """A node whose key and value are NaN reaches its descendants and itself, in the channels that are NaN, and nobody else; so does a token before some windows."""
    trees, lens = [grown(40, 50, 2), grown(12, 51)], [190, 100]
    rows = rows_for(lens, 12, 5)
    gen = torch.Generator(device="cuda").manual_seed(52)
    q = randn(gen, (52, 4, d), BF, 1.5)
    table, plan = at.PageTable(*flat(rows)), planned(h, trees)
    for part, window in (("k", 0), ("v", 0), ("v", 30)):
        cache = filled(53, 1, 12, 2, d)
        clean = dr.attend(h, cache, 0, table, i32(lens), plan, q, window=window)
        node, early = 7, 150 - 25        # of sequence 0: a node, and a token that the window of 30 hides from all nodes deeper than 4
        for token in (150 + node, early) if window else (150 + node,):
            if part == "k":
                cache.k[0, rows[0][token // PAGE], 0, token % PAGE, 3] = 0x7F
            else:
                cache.v[0, rows[0][token // PAGE], 0, 3, token % PAGE] = 0xFF
        o = dr.attend(h, cache, 0, table, i32(lens), plan, q, window=window)
        for i in range(52):
            parent = trees[0] if i < 40 else trees[1]
            up = ancestors(parent, i if i < 40 else i - 40)
            felt = i < 40 and (node in up[:window or 99] or (window and len(up) - 1 + 25 < window))
            if felt:
                got = o[i, :2]
                assert got.isnan().all() if part == "k" else got[:, 3].isnan().all() and not got[:, :3].isnan().any(), (part, window, i)
                assert torch.equal(o[i, 2:], clean[i, 2:])
            else:
                assert torch.equal(o[i], clean[i]), (part, window, i)


@pytest.mark.parametrize("dtype, large, small", [(BF, 2.0 ** 30, 0.0), (BF, 2.0 ** 30, 2.0 ** -90), (BF, 2.0 ** 100, 2.0 ** -100), (F16, 3e4, 0.0), (F16, 3e4, 2.0 ** -20), (BF, 1.0, 2.0 ** -9)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("first", [0, 4])
def test_attend_pages_of_very_different_scales(h, dtype, large, small, d, first):
    """Four pages of large values and four of zeros or tiny ones in turn: sums stay finite, and what the large ones leave room for is right."""
    gen = torch.Generator(device="cuda").manual_seed(55)
    tokens, kv, heads = 6400, 2, 8
    cache, rows = at.PagedCache.empty(1, 100, kv, d), rows_for([tokens], 100, 3)
    k, v = randn(gen, (tokens, kv, d), dtype), torch.rand((tokens, kv, d), generator=gen, device="cuda") + 0.5
    page = torch.arange(tokens, device="cuda") // PAGE
    v = (v * torch.where((page + first) % 8 < 4, large, small)[:, None, None]).to(dtype)
    table = at.PageTable(*flat(rows))
    at.append(h, cache, 0, table, i32([tokens]), i64([0, tokens]), k, v)
    trees = [grown(30, 56)]
    q = randn(gen, (30, heads, d), dtype)
    o = dr.attend(h, cache, 0, table, i32([tokens]), planned(h, trees), q)
    check("o", o, *tree_reference(HostCache(cache, 0), rows, [tokens], trees, q, 1 / math.sqrt(d)))


@pytest.mark.parametrize("large", [2.0 ** 20, 2.0 ** 50])
def test_attend_weight_on_pages_of_small_scale(h, large):
    """Queries that look at the small values alone get them in full digits, though pages of large values with no weight lie before and behind."""
    gen = torch.Generator(device="cuda").manual_seed(57)
    tokens = 8 * PAGE
    cache, rows = at.PagedCache.empty(1, 8, 1, 64), [list(range(8))]
    page = torch.arange(tokens, device="cuda") // PAGE
    small = (page % 4 == 2)
    k = torch.zeros((tokens, 1, 64), dtype=BF, device="cuda")
    k[:, 0, 0] = torch.where(small, 8.0, -8.0)
    v = ((torch.rand((tokens, 1, 64), generator=gen, device="cuda") + 0.5) * torch.where(small, 1.0, large)[:, None, None]).to(BF)
    table = at.PageTable(*flat(rows))
    at.append(h, cache, 0, table, i32([tokens]), i64([0, tokens]), k, v)
    trees = [[-1]]
    q = torch.zeros((1, 2, 64), dtype=BF, device="cuda")
    q[..., 0] = 40.0
    o = dr.attend(h, cache, 0, table, i32([tokens]), planned(h, trees), q)
    host = HostCache(cache, 0)
    want, bound = tree_reference(host, rows, [tokens], trees, q, 1 / 8)
    assert want.abs().max() < 4
    # weights of 2^-115 on the large pages are below what float16 holds: they are not in the result, so that TINY times the large values is not owed
    mass = tree_reference(host, rows, [tokens], trees, q, 1 / 8)[0].abs()
    check("o", o, want, (2.0 ** -8 + 2.0 ** -11 + 2e-4) * mass)


def test_attend_shared_and_missing_pages(h):
    """A table with fewer pages than its lengths (the last tokens that it has count) and ids that do not exist."""
    cache = filled(60, 1, 10, 2, 64)
    gen = torch.Generator(device="cuda").manual_seed(61)
    trees = [grown(6, 62), grown(4, 63), grown(5, 64)]
    q = randn(gen, (15, 4, 64), BF)
    rows = [[2, 4, 6], [2, 4, 8], [2]]
    o = dr.attend(h, cache, 0, at.PageTable(*flat(rows)), i32([190, 150, 500]), planned(h, trees), q)
    check("shared", o, *tree_reference(HostCache(cache, 0), rows, [190, 150, 64], trees, q, 1 / 8))
    o = dr.attend(h, cache, 0, at.PageTable(*flat([[2, 99, -5, 6]])), i32([256]), planned(h, [[-1]]), q[:1])
    host = HostCache(cache, 0)
    ks, vs = (host.tokens(x, [2, 6], 128) for x in (0, 1))
    for head in range(4):
        p = torch.softmax(q[0, head].cpu().double() @ ks[:, head // 2].T / 8, 0)
        assert (o[0, head].cpu().double() - p @ vs[:, head // 2]).abs().max() <= (2 * 2.0 ** -8 + 2e-4) * (p @ vs[:, head // 2].abs()).max()


def test_attend_far_pages(h):
    """Offsets of more than 32 bits: the last pages of a cache of 5 GB, written, attended to, kept and read."""
    heads, d, pages = 16, 128, 20000
    k = torch.empty((1, 2 * pages, heads, PAGE, d), dtype=torch.uint8, device="cuda")
    v = torch.empty((1, 2 * pages, heads, d, PAGE), dtype=torch.uint8, device="cuda")
    cache = at.PagedCache(d, k, v, *[torch.ones((1, 2 * pages, heads), device="cuda") for _ in range(2)])
    near = at.PagedCache.empty(1, 3, heads, d)
    gen = torch.Generator(device="cuda").manual_seed(14)
    trees = [grown(30, 65)]
    plan = planned(h, trees)
    kk, vv, q = randn(gen, (100, heads, d), BF), randn(gen, (100, heads, d), BF), randn(gen, (30, heads, d), BF)
    out = []
    for c, rows in ((cache, [[2 * pages - 1, 2 * pages - 3]]), (near, [[1, 2]])):
        table = at.PageTable(*flat(rows))
        at.append(h, c, 0, table, i32([100]), i64([0, 100]), kk, vv)
        out.append([dr.attend(h, c, 0, table, i32([100]), plan, q)])
        path = ancestors(trees[0], 29)[::-1]
        new = dr.keep(h, c, table, i32([100]), plan, i32(path + [-1] * (30 - len(path))), i32([len(path)]))
        out[-1] += [new, *at.read(h, c, 0, table, new, i64([0, 70 + len(path)]), 70 + len(path))]
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_unchecked_trees(h):
    """Without a check a parent that is not an earlier node counts as -1, ptr is cut to what exists, and nodes behind `most` are left out."""
    cache, rows = filled(66, 1, 6, 1, 64), [[0, 1], [2, 3]]
    table, lens = at.PageTable(*flat(rows)), [100, 90]
    gen = torch.Generator(device="cuda").manual_seed(67)
    q = randn(gen, (9, 2, 64), BF)
    bad, good = [[-1, 0, 5, -7, 2 ** 30], [-1, 1, 0, 3]], [[-1, 0, -1, -1, -1], [-1, -1, 0, -1]]
    o = dr.attend(h, cache, 0, table, i32(lens), planned(h, bad, check=False), q)
    check("parents", o, *tree_reference(HostCache(cache, 0), rows, lens, good, q, 1 / 8))
    parents = [-1, 0, 0, -1, 0, -1, 0, 1, 2]
    t = dr.symbolic(h, i64([-4, 5, 70]), i32(parents), 5, check=False)
    want = dr.attend(h, cache, 0, table, i32(lens), dr.symbolic(h, i64([0, 5, 9]), i32(parents), 5), q)
    assert torch.equal(dr.attend(h, cache, 0, table, i32(lens), t, q), want)
    # nodes behind `most`: a tree of three in which only the first two count, so its context is one token longer
    most = dr.symbolic(h, i64([0, 5, 9]), i32(parents), 2, check=False)
    out = torch.full_like(q, 7.0)
    rc = dr._lib().spdraft_attend(h.ptr, C.byref(cache._struct), 0, C.byref(table.struct(cache)), i32(lens).data_ptr(), C.byref(most._struct), most.memory.data_ptr(), 2, at.BF16, 0.125, 0.0,
                                  None, 0, at._tensor(q, "q"), at._result(out))
    torch.cuda.synchronize()
    assert rc == 0 and (out[[2, 3, 4, 7, 8]] == 7.0).all()
    check("most", out[[0, 1, 5, 6]], *tree_reference(HostCache(cache, 0), rows, lens, [[-1, 0], [-1, 0]], q[[0, 1, 5, 6]], 1 / 8))


@pytest.mark.parametrize("ptr, parent, most", [([0, 2, 4], [-1, 1, -1, 0], 4), ([0, 2, 4], [-1, 0, 0, 0], 4), ([0, 2, 4], [-1, 0, -2, 0], 4), ([0, 3, 2], [-1, 0, -1, 0], 4),
                                               ([1, 2, 4], [-1, -1, -1, 0], 4), ([0, 2, 3], [-1, 0, -1, 0], 4), ([0, 2, 5], [-1, 0, -1, 0], 4), ([0, 3, 4], [-1, 0, 0, -1], 2), ([0], [-1], 1)])
def test_checked_trees(h, ptr, parent, most):
    with pytest.raises(sg.SpgemmError) as e:
        dr.symbolic(h, i64(ptr), i32(parent), most)
    assert e.value.status == -8


def test_nothing_at_all(h):
    """No sequences, and sequences without nodes."""
    cache = filled(68, 1, 4, 2, 64)
    none = dr.symbolic(h, i64([0]), i32([]), 8)
    q = torch.empty((0, 4, 64), dtype=BF, device="cuda")
    assert dr.attend(h, cache, 0, at.PageTable(i64([0]), i32([])), i32([]), none, q).shape == q.shape
    empty = dr.symbolic(h, i64([0, 0, 0]), i32([]), 8)
    table = at.PageTable(*flat([[1], []]))
    assert dr.attend(h, cache, 0, table, i32([5, 0]), empty, q).shape == q.shape
    rows = torch.empty((0, 50), device="cuda")
    path, kept, token = dr.verify(h, empty, i32([]), rows[:, 0], rows, rows)
    assert path.numel() == 0 and kept.tolist() == [0, 0] and token.tolist() == [-1, -1]
    assert dr.keep(h, cache, table, i32([5, 0]), empty, path, kept).tolist() == [5, 0]
    assert [t.shape[0] for t in at.read(h, cache, 0, table, i32([5, 0]), i64([0, 0, 0]), 0)] == [0, 0]


# ---- verification -----------------------------------------------------------------------------------

def drawn(gen, trees, vocab, dtype, spread=3.0, noise=0.7, top=0):
    """Rows of a target and a draft, and every node's token as its parent's row of the draft gives it, one child after the other without replacement."""
    n = sum(map(len, trees))
    thought = torch.randn((n, vocab), generator=gen, device="cuda") * spread
    target = torch.softmax(thought + torch.randn((n, vocab), generator=gen, device="cuda") * noise, -1)
    if top:
        keep = target >= target.topk(min(top, vocab), -1).values[:, -1:]
        target = target * keep / (target * keep).sum(-1, keepdim=True)
    target, draft = target.to(dtype), torch.softmax(thought, -1).to(dtype)
    order = (draft.float().log() - torch.rand((n, vocab), generator=gen, device="cuda").clamp(min=1e-20).log().neg().log()).argsort(-1, descending=True)
    ids, base = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32).tolist(), 0
    for parent in trees:
        for i, p in enumerate(parent):
            if p >= 0:
                ids[base + i] = int(order[base + p, parent[:i].count(p) % vocab])
        base += len(parent)
    return target, draft, i32(ids), torch.rand((n,), generator=gen, device="cuda")


def verified(h, trees, ids, u, target, draft, most=None):
    path, kept, token = dr.verify(h, planned(h, trees, most), ids, u, target, draft)
    got = path.tolist(), kept.tolist(), token.tolist()
    want = verify_reference(trees, ids, u, target, draft)
    assert got[1] == want[1] and got[0] == want[0] and got[2] == want[2]
    return got


@pytest.mark.parametrize("vocab", [1, 2, 7, 255, 257, 1000, 4099, 32003])
@pytest.mark.parametrize("dtype", [F32, BF, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("by_draft", [True, False], ids=["drawn", "chosen"])
def test_verify(h, vocab, dtype, by_draft):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    trees = [grown(n, 70 + n, w) for n, w in ((1, 1), (8, 1), (26, 4), (0, 1), (60, 3), (5, 5), (13, 2))] + [list(range(-1, 6))]
    for noise, top in ((0.7, 0), (3.0, 0), (0.5, 20)):
        target, draft, ids, u = drawn(gen, trees, vocab, dtype, noise=noise, top=top)
        verified(h, trees, ids, u, target, draft if by_draft else None)


@pytest.mark.parametrize("by_draft", [True, False], ids=["drawn", "chosen"])
def test_verify_large(h, by_draft):
    """A vocabulary of several parts, trees of 256 nodes, many children of a node."""
    gen = torch.Generator(device="cuda").manual_seed(71)
    trees = [grown(256, 72, 2), grown(100, 73, 40), [-1] + [0] * 90]
    target, draft, ids, u = drawn(gen, trees, 150001, F32, spread=2.0, noise=1.5)
    verified(h, trees, ids, u, target, draft if by_draft else None)
    verified(h, trees, ids, u * 0 + 0.999999, target, draft if by_draft else None)     # nearly all are refused
    path, kept, _ = verified(h, trees, ids, u * 0, target, draft if by_draft else None)
    assert min(kept) > 1                                                                # (u = 0 takes what has any weight)


def test_verify_strides(h):
    """Rows apart from each other and at any element, with NaN between them."""
    gen = torch.Generator(device="cuda").manual_seed(74)
    trees = [grown(20, 75), grown(9, 76)]
    for dtype, vocab, pad, first in ((F32, 1001, 3, 1), (BF, 5003, 10, 3), (F16, 999, 1, 7)):
        target, draft, ids, u = drawn(gen, trees, vocab, dtype)
        apart = torch.full((29, 2, vocab + pad), math.nan, dtype=dtype, device="cuda")
        apart[:, 0, first % pad:first % pad + vocab], apart[:, 1, :vocab] = target, draft
        a = dr.verify(h, planned(h, trees), ids, u, apart[:, 0, first % pad:first % pad + vocab], apart[:, 1, :vocab])
        b = dr.verify(h, planned(h, trees), ids, u, target, draft)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def rows_of(*rows):
    return torch.tensor(rows, dtype=torch.float32, device="cuda")


def test_verify_by_hand(h):
    u = lambda *v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    # one root, children 1 and 2 with the tokens 0 and 1; r = (.2, .3, .5), q = (.6, .3, .1)
    tree, ids = [[-1, 0, 0]], i32([9, 0, 1])
    p, q = rows_of([.2, .3, .5], [1, 0, 0], [0, 1, 0]), rows_of([.6, .3, .1], [1, 0, 0], [1, 0, 0])
    # token 0 is taken below .2 / .6; else r = (0, 0, .4) / .4, so token 1 never; the next is 2
    assert verified(h, tree, ids, u(.5, .3, .5), p, q) == ([0, 1, -1], [2], [0])
    assert verified(h, tree, ids, u(.5, .4, 0), p, q) == ([0, -1, -1], [1], [2])
    # chosen: token 0 below .2, else r = (0, .375, .625): token 1 below .375, else the next is 2
    assert verified(h, tree, ids, u(.9, .19, .5), p, None) == ([0, 1, -1], [2], [0])
    assert verified(h, tree, ids, u(.9, .21, .37), p, None) == ([0, 2, -1], [2], [1])
    assert verified(h, tree, ids, u(0, .21, .38), p, None) == ([0, -1, -1], [1], [2])
    # a target that is the draft takes every first child; one that is all at one token ends there
    assert verified(h, tree, ids, u(0, .999, .999), p, p)[1] == [2]
    # rows of nothing: no token follows; NaN and negative entries count as nothing
    assert verified(h, [[-1]], i32([0]), u(.5), rows_of([0, 0, 0]), None)[2] == [-1]
    assert verified(h, [[-1]], i32([0]), u(.0), rows_of([math.nan, -1, .25]), None)[2] == [2]
    # no residual (the row is all at a token that u refuses only by a q above it): r stays
    assert verified(h, [[-1, 0]], i32([0, 0]), u(.7, .9), rows_of([.5, 0, 0], [0, 1, 0]), rows_of([1, 0, 0], [1, 0, 0])) == ([0, -1], [1], [0])
    # tokens that are not in the vocabulary are passed over
    for bad in (-1, 3, 2 ** 31 - 1, -2 ** 31):
        assert verified(h, tree, i32([0, bad, 2]), u(.9, 0, .4), p, None) == ([0, 2, -1], [2], [1])
    # several nodes without a parent: the walk begins at the first
    assert verified(h, [[-1, -1, 0]], i32([0, 1, 1]), u(.1, 0, .2), p, None) == ([0, 2, -1], [2], [1])
    # the same token twice
    assert verified(h, [[-1, 0, 0, 0]], i32([0, 0, 0, 2]), u(.9, .9, .9, .7), rows_of([.5, .2, .3], [1, 0, 0], [1, 0, 0], [0, 0, 1]), rows_of([.9, .05, .05], [1, 0, 0], [1, 0, 0], [1, 0, 0]))


@pytest.mark.parametrize("by_draft", [True, False], ids=["drawn", "chosen"])
def test_verify_entries_that_are_none(h, by_draft):
    """NaN and negative entries anywhere in both rows count as 0."""
    gen = torch.Generator(device="cuda").manual_seed(63)
    trees = [grown(30, 64, 4), grown(12, 65, 3), [-1, 0, 0, 0]]
    for dtype, vocab in ((F32, 5003), (BF, 1000)):
        target, draft, ids, u = drawn(gen, trees, vocab, dtype, noise=1.5)
        for t in (target, draft):
            strange = torch.rand(t.shape, generator=gen, device="cuda")
            t[strange < 0.2] = math.nan
            t[strange > 0.8] *= -1
        verified(h, trees, ids, u, target, draft if by_draft else None)


def test_verify_rows_that_are_not_asked(h):
    """The draft's rows of nodes without children may hold anything, as may both rows of nodes that no first child's way leads to."""
    gen = torch.Generator(device="cuda").manual_seed(78)
    trees = [grown(20, 79), grown(9, 80), [-1], list(range(-1, 7))]
    for noise in (0.1, 2.0):
        target, draft, ids, u = drawn(gen, trees, 3001, F32, noise=noise)
        want = verified(h, trees, ids, u, target, draft)
        base = 0
        for parent in trees:
            for i in range(len(parent)):
                if i not in parent:
                    draft[base + i] = (math.inf, math.nan)[i % 2]
            base += len(parent)
        got = dr.verify(h, planned(h, trees), ids, u, target, draft)
        assert [t.tolist() for t in got] == list(want)


def test_verify_last_number(h):
    """u just below 1 gives the last token above 0, u = 0 the first, in rows with zeros at both ends."""
    for vocab in (50, 5000, 70001):
        row = torch.zeros((2, vocab), device="cuda")
        row[:, vocab // 3:vocab // 2] = 1.0 / (vocab // 2 - vocab // 3)
        u = torch.tensor([0.0, 1 - 2.0 ** -24], device="cuda")
        _, _, token = dr.verify(h, planned(h, [[-1], [-1]]), i32([0, 0]), u, row, None)
        assert token.tolist() == [vocab // 3, vocab // 2 - 1]


def test_verify_gives_the_targets_tokens(h):
    """The first token behind the root, taken or drawn, comes as often as the target says: 40 000 trees of a root and three children drawn without replacement."""
    gen = torch.Generator(device="cuda").manual_seed(77)
    n, vocab = 40000, 6
    p = torch.tensor([.05, .3, .1, .25, .2, .1], device="cuda")
    q = torch.tensor([.3, .1, .2, .05, .05, .3], device="cuda")
    order = (q.log() - torch.rand((n, vocab), generator=gen, device="cuda").clamp(min=1e-20).log().neg().log()).argsort(-1, descending=True)[:, :3]
    ids = torch.cat([torch.zeros((n, 1), dtype=torch.int64, device="cuda"), order], 1).to(torch.int32).flatten().contiguous()
    plan = dr.symbolic(h, i64([4 * i for i in range(n + 1)]), i32([-1, 0, 0, 0] * n), 4)
    path, kept, token = dr.verify(h, plan, ids, torch.rand((4 * n,), generator=gen, device="cuda"), p.expand(4 * n, vocab), q.expand(4 * n, vocab))
    taken = ids.view(n, 4).gather(1, path.view(n, 4)[:, 1:2].clamp(min=0).long())[:, 0]
    share = torch.bincount(torch.where(kept > 1, taken, token).long(), minlength=vocab) / n
    assert (kept > 1).float().mean() > 0.5
    assert ((share - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all(), share      # (five standard deviations)


# ---- keep -----------------------------------------------------------------------------------------

def path_of(parent, node):
    return ancestors(parent, node)[::-1] if parent else []


@pytest.mark.parametrize("d", [8, 64, 72, 128])
@pytest.mark.parametrize("seed", range(4))
def test_keep(h, d, seed):
    rng = random.Random(seed)
    trees = [grown(n, 80 + seed + n, w) for n, w in ((1, 1), (12, 3), (60, 2), (0, 1), (26, 4), (130, 2), (256, 1), (9, 1))]
    context = [rng.randint(0, 150) for _ in trees]
    lens = [c + len(t) for c, t in zip(context, trees)]
    cache = filled(81 + seed, 3, 60, 2, d)
    cache.k_scale *= torch.exp2(torch.randint(-3, 4, cache.k_scale.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).float())
    rows = rows_for(lens, 60, seed, spare=seed % 2)
    paths = [path_of(t, rng.randrange(len(t)) if t else -1) for t in trees]
    if seed == 1:
        paths = [p[:rng.randint(0, len(p))] for p in paths]
    hosts = [HostCache(cache, layer) for layer in range(3)]
    flat_path = [x for p, t in zip(paths, trees) for x in p + [-1] * (len(t) - len(p))]
    got = dr.keep(h, cache, at.PageTable(*flat(rows)), i32(lens), planned(h, trees), i32(flat_path), i32([len(p) for p in paths]))
    assert got.tolist() == [c + len(p) for c, p in zip(context, paths)]
    for layer, host in enumerate(hosts):
        for pages, ctx, p in zip(rows, context, paths):
            keep_reference(host, pages, ctx, p)
        now = HostCache(cache, layer)
        for x in (0, 1):
            assert torch.equal(now.scale[x], host.scale[x])
            assert torch.equal(now.code[x][..., :d].nan_to_num(1e9), host.code[x][..., :d].nan_to_num(1e9))


def test_keep_unusual_values(h):
    """NaN and the largest values move as they are, and a scale follows what moved in, not what was refused."""
    for d in (64, 128):
        cache = filled(82, 1, 4, 1, d)
        cache.k_scale[0, 2], cache.v_scale[0, 2] = 2.0 ** 3, 2.0 ** 3
        cache.k[0, 2, 0, 5], cache.v[0, 2, 0, :, 5] = 0x7E, 0x7E          # 448: refused
        cache.k[0, 2, 0, 6], cache.v[0, 2, 0, :, 6] = 0x01, 0x01          # the smallest: taken
        cache.k[0, 2, 0, 6, 3], cache.v[0, 2, 0, 3, 6] = 0xFF, 0x7F
        host = HostCache(cache, 0)
        parent = list(range(-1, 9)) + [4]
        lens = [64 + 7]                                                   # nodes at 60 .. 70
        keep_reference(host, [1, 2], 60, [0, 1, 2, 10])
        new = dr.keep(h, cache, at.PageTable(*flat([[1, 2]])), i32(lens), planned(h, [parent]), i32([0, 1, 2, 10] + [-1] * 7), i32([4]))
        now = HostCache(cache, 0)
        assert new.tolist() == [64]
        for x in (0, 1):
            assert torch.equal(now.scale[x], host.scale[x]) and now.scale[x][1, 0] <= 2.0 ** -4
            assert torch.equal(now.code[x].nan_to_num(1e9), host.code[x].nan_to_num(1e9)) and now.code[x][1, 0, 63, 3].isnan()


def test_keep_refused_paths(h):
    """Paths that do not ascend or leave the tree end there; a sequence with fewer tokens than its tree, or without the pages, is left as it is."""
    cache = filled(83, 1, 8, 1, 64)
    before = clone(cache)
    trees = [[-1, 0, 0, 1]] * 6
    plan = planned(h, trees)
    rows = [[0], [1], [2], [3], [9], [5, 6]]
    lens = [20, 3, 20, 80, 20, 66]
    path = i32([1, 1, 2, 3] + [0, 2, -1, -1] + [-1, 0, 1, 2] + [0, 2, 3, -1] + [0, 3, -1, -1] + [0, 4, 9, -1])
    kept = i32([4, 2, 3, 3, 2, 3])
    new = dr.keep(h, cache, at.PageTable(*flat(rows)), i32(lens), plan, path, kept)
    assert new.tolist() == [17, 3, 16, 80, 20, 63]
    assert torch.equal(cache.k[0, 1:], before.k[0, 1:]) and torch.equal(cache.v[0, 1:], before.v[0, 1:])
    want = before.k[0, 0].clone()
    want[:, 16] = want[:, 17]
    assert torch.equal(cache.k[0, 0], want)
    # kept that is out of range is cut
    assert dr.keep(h, before, at.PageTable(*flat([[0]])), i32([20]), planned(h, trees[:1]), i32([0, 1, 2, 3]), i32([99])).tolist() == [20]
    assert dr.keep(h, before, at.PageTable(*flat([[0]])), i32([20]), planned(h, trees[:1]), i32([0, 1, 2, 3]), i32([-5])).tolist() == [16]


# ---- read -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [8, 64, 72, 128])
def test_read(h, dtype, d):
    """Ragged parts: nothing, the last token, from a page's begin, several pages, more than there is, pages that are not there."""
    lens = [200, 64, 0, 130, 63, 1000, 5, 70, 300]
    count = [200, 1, 0, 66, 0, 129, 9, 70, 300]
    cache = filled(90, 2, 60, 3, d)
    cache.k[1, :, :, 5], cache.v[1, :, :, :, 6] = 0x7F, 0xFE            # NaN; the largest negative
    cache.k[1, ..., d:], cache.v[1, ..., d:, :] = 0x7F, 0xFF
    rows = rows_for(lens, 60, 2)
    rows[7], rows[8] = rows[7][:1], [rows[8][0], 99, -3] + rows[8][3:]
    ptr = sums(count)
    k, v = at.read(h, cache, 1, at.PageTable(*flat(rows)), i32(lens), i64(ptr), ptr[-1], dtype)
    host = HostCache(cache, 1)
    for x, got in enumerate((k, v)):
        for s, pages in enumerate(rows):
            want = torch.zeros((count[s], 3, d), dtype=torch.float64)
            for i in range(count[s]):
                pos = lens[s] - count[s] + i
                if pos >= 0 and pos // PAGE < len(pages) and 0 <= pages[pos // PAGE] < 60:
                    p = pages[pos // PAGE]
                    want[i] = host.code[x][p, :, pos % PAGE, :d] * host.scale[x][p][:, None]
            assert torch.equal(got[ptr[s]:ptr[s + 1]].cpu().nan_to_num(1e4), want.to(dtype).nan_to_num(1e4)), (s, x)


def test_read_values_out_of_range(h):
    """What float16 cannot hold becomes infinite, what it holds in fewer digits is rounded to nearest."""
    cache = filled(91, 1, 2, 1, 64)
    cache.k_scale[:], cache.v_scale[:] = 2.0 ** 10, 2.0 ** -22
    k, v = at.read(h, cache, 0, at.PageTable(*flat([[1, 0]])), i32([128]), i64([0, 128]), 128, F16)
    host = HostCache(cache, 0)
    for x, got in ((0, k), (1, v)):
        assert torch.equal(got.cpu(), host.tokens(x, [1, 0], 128).to(F16))
    assert k.isinf().any()


def test_read_into_rows_apart(h):
    """Outputs at strides of their own; what lies between and behind them stays."""
    cache, rows = filled(92, 1, 4, 2, 72), [[2, 0], [1]]
    ptr, lens = [0, 100, 130], [100, 40]
    table = at.PageTable(*flat(rows))
    want = at.read(h, cache, 0, table, i32(lens), i64(ptr), 130)
    wide = [torch.full((150, 3, 88), 5.0, dtype=BF, device="cuda") for _ in range(2)]
    part = [at.TensorStruct(w[:, 1:].data_ptr(), w.stride(0), w.stride(1)) for w in wide]
    lengths, begins = i32(lens), i64(ptr)
    assert at._lib().spcache_read(h.ptr, C.byref(cache._struct), 0, C.byref(table.struct(cache)), lengths.data_ptr(), begins.data_ptr(), 130, at.BF16, *part) == 0
    torch.cuda.synchronize()
    for w, t in zip(wide, want):
        assert torch.equal(w[:130, 1:, :72], t)
        w[:130, 1:, :72] = 5.0
        assert (w == 5.0).all()


def test_read_is_what_forward_takes(h):
    """A long part of a prompt over what is cached of it: read, then the forward pass, and the same tokens by the cache's own attention."""
    gen = torch.Generator(device="cuda").manual_seed(93)
    lens, part = [500, 180], [120, 100]
    cache, rows = filled(94, 1, 12, 2, 64), rows_for(lens, 12)
    table = at.PageTable(*flat(rows))
    k, v = at.read(h, cache, 0, table, i32(lens), i64([0, 500, 680]), 680)
    q = randn(gen, (220, 4, 64), BF)
    plan = at.symbolic(h, 220, 680, q_ptr=i64([0, 120, 220]), k_ptr=i64([0, 500, 680]))
    o, _ = at.forward(h, plan, q, k, v)
    host = HostCache(cache, 0)
    trees = [list(range(-1, n - 1)) for n in part]
    want, bound = tree_reference(host, rows, lens, trees, q, 1 / 8)
    mass = bound / (2.0 ** -11 + 2e-4)
    check("forward", o, want, bound + (2.0 ** -8 - 2.0 ** -11) * mass)       # (its probabilities are operands in bfloat16)
    check("tree", dr.attend(h, cache, 0, table, i32(lens), planned(h, trees), q), want, bound)


# ---- together -------------------------------------------------------------------------------------

def test_steps_of_serving(h):
    """Trees appended, attended to, verified and kept in two layers, pages given back: the cache then holds the accepted tokens, as one that was given them alone would, but for a rounding more where a scale
    rose in between, and attention over it is that of the accepted chain."""
    gen = torch.Generator(device="cuda").manual_seed(95)
    n, kv, heads, d, layers, vocab = 5, 2, 8, 64, 2, 500
    cache = at.PagedCache.empty(layers, 60, kv, d)
    lens = [70, 3, 128, 61, 1]
    table, _ = at.fork(h, cache, at.PageTable(i64([0]), i32([])), i32([]), i32([-1] * n), i32(lens))
    held = [[(randn(gen, (x, kv, d), BF), randn(gen, (x, kv, d), BF)) for x in lens] for _ in range(layers)]
    for layer in range(layers):
        at.append(h, cache, layer, table, i32(lens), i64(sums(lens)), torch.cat([a for a, _ in held[layer]]), torch.cat([b for _, b in held[layer]]))
    accepted = 0
    for step in range(6):
        trees = [grown(random.Random(10 * step + s).randint(1, 30), 10 * step + s) for s in range(n)]
        count = list(map(len, trees))
        ptr, full = sums(count), [a + b for a, b in zip(lens, count)]
        table, _ = at.fork(h, cache, table, i32(lens), i32(range(n)), i32(full))
        plan = planned(h, trees)
        fresh = []
        for layer in range(layers):
            k, v, q = randn(gen, (ptr[-1], kv, d), BF), randn(gen, (ptr[-1], kv, d), BF), randn(gen, (ptr[-1], heads, d), BF)
            at.append(h, cache, layer, table, i32(full), plan.ptr, k, v)
            o = dr.attend(h, cache, layer, table, i32(full), plan, q)
            ptrs, pages = table.rowptr.tolist(), table.pages.tolist()
            rows = [pages[a:b] for a, b in zip(ptrs, ptrs[1:])]
            check("tree", o, *tree_reference(HostCache(cache, layer), rows, full, trees, q, 1 / 8))
            fresh.append((k, v))
        target, draft, ids, u = drawn(gen, trees, vocab, F32, noise=0.3)
        path, kept, token = dr.verify(h, plan, ids, u, target, draft)
        assert [path.tolist(), kept.tolist(), token.tolist()] == list(verify_reference(trees, ids, u, target, draft))
        new = dr.keep(h, cache, table, i32(full), plan, path, kept)
        kept = kept.tolist()
        assert new.tolist() == [a + b for a, b in zip(lens, kept)]
        for s in range(n):
            stays = [ptr[s] + x for x in path[ptr[s]:ptr[s] + kept[s]].tolist()]
            for layer in range(layers):
                held[layer][s] = tuple(torch.cat([old, t[stays]]) for old, t in zip(held[layer][s], fresh[layer]))
        table, _ = at.fork(h, cache, table, new, i32(range(n)), new)
        lens = new.tolist()
        accepted += sum(kept) - n
    assert accepted > 10
    for layer in range(layers):
        k, v = at.read(h, cache, layer, table, i32(lens), i64(sums(lens)), sum(lens))
        for got, x in ((k, 0), (v, 1)):
            want = torch.cat([held[layer][s][x] for s in range(n)]).double()
            # values of up to 5 lie within 448 of a scale of 2^-6 at most.  Each of up to three roundings (appended, moved, rounded again as a scale rose twice) is off by half a step: 2^-4 of the value, or 2^-10 of the scale
            assert ((got.double() - want).abs() <= 4 * (2.0 ** -4 * want.abs() + 2.0 ** -16)).all()
            assert ((got.double() - want).norm() / want.norm()) < 0.04        # (2^-4 / sqrt 3 at most, once)


def test_graph(h):
    """A step, captured: trees, lengths, rows and numbers live on the GPU, so each replay is another step; eager calls of other sizes and on another handle between the replays."""
    stream = torch.cuda.Stream()
    handle = sg.Handle(stream=stream)
    gen = torch.Generator(device="cuda").manual_seed(96)
    n, kv, heads, d, vocab, most = 3, 2, 4, 64, 1000, 16
    base = filled(97, 2, 12, kv, d)
    cache, eager = clone(base), clone(base)
    rows = [[1, 3, 5, 7], [0, 2, 4, 6], [8, 9, 10, 11]]
    table = at.PageTable(*flat(rows))
    lens, ptr, parent = i32([100, 70, 190]), i64([0, 16, 20, 36]), i32(grown(16, 1) + grown(4, 2) + grown(16, 3))
    q, k = randn(gen, (36, heads, d), BF), randn(gen, (36, kv, d), BF)
    target, draft = torch.empty((36, vocab), device="cuda"), torch.empty((36, vocab), device="cuda")
    ids, u = torch.zeros(36, dtype=torch.int32, device="cuda"), torch.zeros(36, device="cuda")

    def step(c):
        trees = dr.symbolic(handle, ptr, parent, most, check=False)
        at.append(handle, c, 1, table, lens, ptr, k, k)
        o = dr.attend(handle, c, 1, table, lens, trees, q)
        path, kept, token = dr.verify(handle, trees, ids, u, target, draft)
        new = dr.keep(handle, c, table, lens, trees, path, kept)
        return o, path, kept, token, new, *at.read(handle, c, 1, table, new, i64_ptr, 60)

    i64_ptr = i64([0, 20, 40, 60])

    def fill(i):
        counts = [(16, 4, 16), (1, 16, 3), (0, 16, 16), (9, 9, 9)][i % 4]
        trees = [grown(c, 10 * i + j) for j, c in enumerate(counts)]
        p, dft, x, numbers = drawn(gen, trees, vocab, F32)
        total = sum(counts)
        ptr.copy_(i64(sums(counts)))
        parent[:total] = i32([x for t in trees for x in t])
        for t, new in ((target, p), (draft, dft), (ids, x), (u, numbers)):
            t[:total] = new
        lens.copy_(i32([84 + counts[0], 66 + counts[1], 150 + counts[2]]))
        q.copy_(randn(gen, q.shape, BF))
        k.copy_(randn(gen, k.shape, BF))

    fill(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(clone(base))
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = step(cache)
    for i in range(6):
        fill(i)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            want = step(eager)
        torch.cuda.synchronize()
        total = int(ptr[-1])
        for a, b in zip(out, want):
            assert torch.equal(a[:total] if a.shape[0] == 36 else a, b[:total] if b.shape[0] == 36 else b), i
        assert torch.equal(cache.k, eager.k) and torch.equal(cache.v, eager.v) and torch.equal(cache.k_scale, eager.k_scale)
        trees = [grown(60, 98 + i)]                                     # eager work that needs more scratch memory than the graph
        many = planned(handle, trees)
        with torch.cuda.stream(stream):
            dr.attend(handle, eager, 0, at.PageTable(*flat([list(range(12)) * 8])), i32([6000]), many, randn(gen, (60, heads, d), BF))
        stream.synchronize()


def test_two_handles_at_once(h):
    """Two handles on streams of their own, with calls of different sizes in flight together, and results that each alone gives."""
    gen = torch.Generator(device="cuda").manual_seed(101)
    trees = [[grown(30, 1), grown(17, 2)], [grown(60, 3)]]
    lens = [[3000, 500], [5000]]
    caches = [filled(102 + i, 1, 90, 2, 64) for i in range(2)]
    tables = [at.PageTable(*flat(rows_for(n, 90, i))) for i, n in enumerate(lens)]
    qs = [randn(gen, (sum(map(len, t)), 8, 64), BF) for t in trees]
    plans = [planned(h, t) for t in trees]
    want = [dr.attend(h, caches[i], 0, tables[i], i32(lens[i]), plans[i], qs[i]) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    handles = [sg.Handle(stream=s) for s in streams]
    lengths = [i32(n) for n in lens]
    torch.cuda.synchronize()
    got = [[dr.attend(handles[i], caches[i], 0, tables[i], lengths[i], plans[i], qs[i]) for i in range(2)] for _ in range(20)]
    torch.cuda.synchronize()
    assert all(torch.equal(g[i], want[i]) for g in got for i in range(2))


def test_same_bits_again(h):
    gen = torch.Generator(device="cuda").manual_seed(99)
    trees, lens = [grown(40, 1), grown(13, 2)], [4000, 900]
    cache, rows = filled(98, 1, 90, 2, 128), rows_for(lens, 90)
    table, plan, q = at.PageTable(*flat(rows)), planned(h, trees), randn(gen, (53, 8, 128), BF)
    first = dr.attend(h, cache, 0, table, i32(lens), plan, q)
    for _ in range(3):
        assert torch.equal(dr.attend(h, cache, 0, table, i32(lens), plan, q), first)


def test_arguments(h):
    cache = filled(100, 1, 4, 2, 64)
    table, lens, trees = at.PageTable(*flat([[1]])), i32([10]), planned(h, [[-1, 0]])
    q = torch.zeros((2, 4, 64), dtype=BF, device="cuda")
    rows, u, ids = torch.zeros((2, 30), device="cuda"), torch.zeros(2, device="cuda"), i32([0, 1])
    path, kept = i32([0, 1]), i32([1])
    for call, kind in ((lambda: dr.symbolic(h, i32([0, 2]), i32([-1, 0]), 2), ValueError),
                       (lambda: dr.symbolic(h, i64([0, 2]), i64([-1, 0]), 2), ValueError),
                       (lambda: dr.symbolic(h, i64([]), i32([]), 2), ValueError),
                       (lambda: dr.symbolic(h, i64([0, 2]).cpu(), i32([-1, 0]), 2), ValueError),
                       (lambda: dr.symbolic(h, i64([0, 2]), i32([-1, 0]), 0), sg.SpgemmError),
                       (lambda: dr.symbolic(h, i64([0, 2]), i32([-1, 0]), 257), sg.SpgemmError),
                       (lambda: dr.attend(h, cache, 1, table, lens, trees, q), sg.SpgemmError),
                       (lambda: dr.attend(h, cache, 0, table, lens, trees, q[:1]), ValueError),
                       (lambda: dr.attend(h, cache, 0, table, lens, trees, q[..., :32]), ValueError),
                       (lambda: dr.attend(h, cache, 0, table, lens, trees, q.cpu()), ValueError),
                       (lambda: dr.attend(h, cache, 0, table, lens, trees, q.float()), TypeError),
                       (lambda: dr.attend(h, cache, 0, table, lens, trees, q[:, :3]), sg.SpgemmError),
                       (lambda: dr.attend(h, cache, 0, table, lens.long(), trees, q), ValueError),
                       (lambda: dr.attend(h, cache, 0, at.PageTable(*flat([[1], [2]])), i32([10, 3]), trees, q), sg.SpgemmError),
                       (lambda: dr.attend(h, cache, 0, table, lens, trees, q, slopes=torch.zeros(3, device="cuda")), ValueError),
                       (lambda: dr.attend(h, cache, 0, table, lens, trees, q, window=-1), sg.SpgemmError),
                       (lambda: dr.verify(h, trees, ids, u, rows[:1]), ValueError),
                       (lambda: dr.verify(h, trees, ids, u, rows.t()), ValueError),
                       (lambda: dr.verify(h, trees, ids, u, rows.double()), TypeError),
                       (lambda: dr.verify(h, trees, ids, u, rows, rows.half()), ValueError),
                       (lambda: dr.verify(h, trees, ids, u, rows[:, :0]), sg.SpgemmError),
                       (lambda: dr.verify(h, trees, ids.long(), u, rows), ValueError),
                       (lambda: dr.verify(h, trees, ids, u[:1], rows), ValueError),
                       (lambda: dr.keep(h, cache, table, lens, trees, path[:1], kept), ValueError),
                       (lambda: dr.keep(h, cache, table, lens, trees, path, i32([1, 1])), ValueError),
                       (lambda: at.read(h, cache, 0, table, lens, i64([0]), 2), ValueError),
                       (lambda: at.read(h, cache, 0, table, lens, i64([0, 2]), 2, F32), TypeError),
                       (lambda: at.read(h, cache, 0, table, lens, i64([0, 2]), -1), ValueError),
                       (lambda: at.read(h, cache, 5, table, lens, i64([0, 2]), 2), sg.SpgemmError)):
        with pytest.raises(kind):
            call()
