"""Drafted tokens at the ends of the ranges."""
import ctypes as C
import math
import random

import pytest
import torch

from attn_helpers import PAGE, HostCache, check, flat
from draft_helpers import keep_reference, tree_reference
from paper_2404_04541_amd import attention as at
from paper_2404_04541_amd import binding as sg
from paper_2404_04541_amd import drafts as dr
from test_gpu_drafts import filled, grown, i32, i64, planned, randn, rows_for, sums

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def h():
    return sg.Handle()


def kept_as_by_hand(h, cache, rows, ctx, parent, path):
    host = HostCache(cache, 0)
    keep_reference(host, rows[0], ctx, path)
    new = dr.keep(h, cache, at.PageTable(*flat(rows)), i32([ctx + len(parent)]), planned(h, [parent]), i32(path + [-1] * (len(parent) - len(path))), i32([len(path)]))
    now = HostCache(cache, 0)
    assert new.tolist() == [ctx + len(path)]
    for x in (0, 1):
        assert torch.equal(now.scale[x], host.scale[x])
        assert torch.equal(now.code[x][..., :host.d].nan_to_num(1e9), host.code[x][..., :host.d].nan_to_num(1e9))
    return now


@pytest.mark.parametrize("exponent", [20, 27, 28, 30, 120])
@pytest.mark.parametrize("d", [8, 64, 128])
def test_keep_zeros_of_a_large_page_into_an_empty_one(h, exponent, d):
    """A token of zeros on a page of the scale 2^exponent comes to one that holds nothing but zeros so far, of the scale 2^-100: zeros it stays, and NaN in it NaN."""
    cache = at.PagedCache.empty(1, 4, 1, d)
    cache.k_scale[0, 1], cache.v_scale[0, 1] = 2.0 ** -100, 2.0 ** -100
    cache.k_scale[0, 2], cache.v_scale[0, 2] = 2.0 ** exponent, 2.0 ** exponent
    cache.k[0, 2], cache.v[0, 2] = 0x38, 0x38                           # 1: refused
    cache.k[0, 2, 0, 5], cache.v[0, 2, 0, :, 5] = 0x00, 0x00            # zeros: taken
    cache.k[0, 2, 0, 6], cache.v[0, 2, 0, :, 6] = 0x80, 0x80            # ... and those below 0
    cache.k[0, 2, 0, 6, 3], cache.v[0, 2, 0, 3, 6] = 0x7F, 0xFF
    parent = list(range(-1, 8)) + [2, 9]                                # nodes at 60 .. 70: 4 .. 10 lie in the second page
    now = kept_as_by_hand(h, cache, [[1, 2]], 60, parent, [0, 1, 9, 10])
    for x in (0, 1):
        token = now.code[x][1, 0, 63, :d]
        assert token[3].isnan() and (token.nan_to_num(0) == 0).all() and (now.code[x][1, 0, :63] == 0).all() and now.scale[x][1, 0] == 2.0 ** -100


@pytest.mark.parametrize("d", [8, 64, 128])
def test_keep_the_largest_values(h, d):
    """What bfloat16's largest value becomes in 8 bits, 256 times 2^120, is more than 32 bits hold as a number; it moves to a page of small values all the same, whose scale grows for it."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache, rows = at.PagedCache.empty(1, 4, 1, d), [[1, 2]]
    k, v = randn(gen, (70, 1, d), BF), randn(gen, (70, 1, d), BF)
    k[66], v[66] = torch.finfo(BF).max, -torch.finfo(BF).max
    at.append(h, cache, 0, at.PageTable(*flat(rows)), i32([70]), i64([0, 70]), k, v)
    assert cache.k_scale[0, 2, 0] == 2.0 ** 120
    parent = list(range(-1, 8)) + [0]
    parent[6] = 1
    now = kept_as_by_hand(h, cache, rows, 60, parent, [0, 1, 6])
    for x, sign in ((0, 1), (1, -1)):
        assert now.scale[x][1, 0] == 2.0 ** 120 and (now.code[x][1, 0, 62, :d] == sign * 256).all()
    cache.k[0, 2, 0, 4], cache.v[0, 2, 0, :, 4] = 0x7E, 0xFE            # 448 times 2^120
    kept_as_by_hand(h, cache, [[3, 2]], 60, parent, [0, 6, 8])


@pytest.mark.parametrize("nodes", [12, 40], ids=["few_rows", "many_rows"])
@pytest.mark.parametrize("first", [0, 4], ids=["large_first", "zeros_first"])
@pytest.mark.parametrize("where", ["context", "tree"])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_feels_nan_on_a_page_of_next_to_no_scale(h, nodes, first, where, d):
    """Pages that hold zeros and a value that is NaN have the scale 2^-100: next to pages of large values nothing else shows of them, but NaN does, to every node that sees it and in its channel.  (Among so many
    sequences a workgroup has eight pages.)"""
    gen = torch.Generator(device="cuda").manual_seed(3)
    pages, seqs, mine = 16, 520, 300
    tokens = pages * PAGE + (nodes - PAGE if where == "tree" else 20)
    lens, trees = [0] * seqs, [[]] * seqs
    lens[mine], trees[mine] = tokens, grown(nodes, 5, 2)
    cache, rows = at.PagedCache.empty(1, pages + 1, 2, d), rows_for(lens, pages + 1, 4)
    table, plan = at.PageTable(*flat(rows)), planned(h, trees)
    k, v = randn(gen, (tokens, 2, d), BF), torch.zeros((tokens, 2, d), device="cuda")
    page = torch.arange(tokens, device="cuda") // PAGE
    large = (page + first) % 8 < 4 if where == "context" else page < pages - 1
    v[large] = (torch.rand((int(large.sum()), 2, d), generator=gen, device="cuda") + 0.5) * 2.0 ** 20
    at.append(h, cache, 0, table, i32(lens), i64([0] * (mine + 1) + [tokens] * (seqs - mine)), k, v.to(BF))
    q = randn(gen, (nodes, 8, d), BF)
    attend = lambda: dr.attend(h, cache, 0, table, i32(lens), plan, q)  # noqa: E731
    clean = attend()
    check("clean", clean, *tree_reference(HostCache(cache, 0), rows, lens, trees, q, 1 / math.sqrt(d)))
    # NaN in channel 3 of key head 0: in each of the pages of zeros, or in the tree's root
    zeros = [x * PAGE + 7 for x in range(pages) if not large[x * PAGE]]
    for token in [tokens - nodes] if where == "tree" else zeros:
        at_page = rows[mine][token // PAGE]
        assert cache.v_scale[0, at_page, 0] == 2.0 ** -100
        cache.v[0, at_page, 0, 3, token % PAGE] = 0x7F
        o = attend()
        assert o[:, :4, 3].isnan().all(), token
        o[:, :4, 3] = clean[:, :4, 3]
        assert torch.equal(o, clean)
        cache.v[0, at_page, 0, 3, token % PAGE] = 0


def test_attend_rows_that_overlap_and_have_more_pieces_than_the_launch(h):
    """A table of 1000 entries whose row pointers go back and forth, so that the rows have 256 times as many pages: what that gives is not said, but the call ends, whatever its memory holds
    of sequences that no workgroup came to, and writes its output alone."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    own = sg.Handle()
    cache = filled(14, 1, 50, 1, 64)
    before = cache.k.clone(), cache.v.clone()
    plan, lens = planned(own, [[-1]] * 512), i32([64000] * 512)
    table = at.PageTable(i64([0, 1000] * 256 + [0]), i32([i % 50 for i in range(1000)]))
    q = randn(gen, (512, 1, 64), BF)
    out = torch.full((520, 1, 64), 7.0, dtype=BF, device="cuda")
    for pattern in ([0, 0, 2 ** 31 - 1, 1], [0, 1, 2 ** 31 - 1, 1], [2 ** 31 - 1] * 4, [-1, 0, -1, 0], [-2 ** 31, 1, 2 ** 31 - 1, 1]):
        for memory in own._live.values():                            # (of the first call: none)
            words = memory[:memory.numel() // 16 * 16].view(torch.int32).view(-1, 4)
            words.copy_(i32(pattern).expand_as(words))
        rc = dr._lib().spdraft_attend(own.ptr, C.byref(cache._struct), 0, C.byref(table.struct(cache)), lens.data_ptr(), C.byref(plan._struct), plan.memory.data_ptr(), 1, at.BF16, 0.125, 0.0, None, 0,
                                      at._tensor(q, "q"), at.TensorStruct(out.data_ptr(), 64, 64))
        torch.cuda.synchronize()
        assert rc == 0 and (out[512:] == 7.0).all() and torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])


def times(run, n=5):
    """us of the fastest of n runs, after one that does not count."""
    out = []
    for _ in range(n + 1):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        run()
        end.record()
        torch.cuda.synchronize()
        out.append(begin.elapsed_time(end) * 1e3)
    return min(out[1:])


def test_attend_one_long_sequence_among_nearly_as_many_as_fill_the_card(h):
    """A few sequences fewer than four turns of the card take does not mean that the long one among them stays whole."""
    gen = torch.Generator(device="cuda").manual_seed(15)
    took = {}
    cache = filled(16, 1, 3100, 8, 128)
    for seqs in (200, 250, 255, 257):
        lens, trees = [60000] + [500] * (seqs - 1), [grown(8, s) for s in range(seqs)]
        table, plan, lengths = at.PageTable(*flat(rows_for(lens, 3100, 7))), planned(h, trees), i32(lens)
        q = randn(gen, (8 * seqs, 8, 128), BF)
        took[seqs] = times(lambda: dr.attend(h, cache, 0, table, lengths, plan, q))
    assert max(took.values()) < 2 * took[257], took


# places of workgroups are 768 for heads of up to 64 channels, else 512, with four turns: numbers of units on both sides of three and of four, in sequences of 8 key heads
@pytest.mark.parametrize("seqs, d", [(190, 128), (193, 128), (254, 128), (255, 128), (256, 128), (300, 128), (287, 64), (383, 64), (384, 64), (385, 64), (512, 64), (520, 64), (520, 128)])
@pytest.mark.parametrize("window", [0, 400])
def test_attend_as_many_units_as_places(h, seqs, d, window):
    """Long sequences among many short ones are cut, whether or not units fill the turns, with trees of more than 128 rows among them; sequences without tokens or nodes in between count as nothing."""
    rng = random.Random(seqs + d)
    some = sorted(rng.sample(range(seqs), 12))
    empty = {s for s in some[6:9]}
    trees = [[] if s in empty else grown(40 if s in some[:3] else 1 + s % 5, s, 2) for s in range(seqs + len(empty))]
    lens = [2500 + 200 * s // seqs if s in some[1:5] else len(t) + rng.randint(1, 60) for s, t in enumerate(trees)]
    lens[some[6]] = 0
    pages = sum(-(-n // PAGE) for n in lens) + 1
    cache, rows = filled(17, 1, pages, 8, d), rows_for(lens, pages, 8)
    gen = torch.Generator(device="cuda").manual_seed(18)
    q = randn(gen, (sum(map(len, trees)), 32, d), BF, 1.5)
    o = dr.attend(h, cache, 0, at.PageTable(*flat(rows)), i32(lens), planned(h, trees), q, window=window)
    ptr, host = sums(map(len, trees)), HostCache(cache, 0)
    shown = sorted(set(some) | set(range(0, len(trees), 25)) | {len(trees) - 1})
    for head in (0, 5, 7):
        of = lambda t: torch.cat([t[ptr[s]:ptr[s + 1], 4 * head:4 * head + 4] for s in shown])  # noqa: E731
        one = HostCache(cache, 0)
        one.code, one.scale = [c[:, head:head + 1] for c in host.code], [c[:, head:head + 1] for c in host.scale]
        check(f"head {head}", of(o), *tree_reference(one, [rows[s] for s in shown], [lens[s] for s in shown], [trees[s] for s in shown], of(q), 1 / math.sqrt(d), window=window))


def held(handle):
    return sum(t.numel() for t in handle._live.values())


@pytest.mark.parametrize("most, window", [(64, 0), (256, 0), (64, 300)])
def test_attend_memory_of_many_sequences(most, window):
    """More sequences than every workgroup looks through: memory is for what is cut, so that one sequence more does not cost gigabytes."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    d, kv, heads, use = 128, 8, 64, {}
    for seqs in (512, 600):
        h = sg.Handle()
        trees = [grown(1 + s % 3 + (40 if s % 200 == 9 else 0), s) for s in range(seqs)]
        lens = [3000 + s if s % 97 == 5 else len(t) + s % 70 for s, t in enumerate(trees)]
        pages = sum(-(-n // PAGE) for n in lens)
        cache, rows = filled(12, 1, pages, kv, d), rows_for(lens, pages, 6)
        q = randn(gen, (sum(map(len, trees)), heads, d), BF)
        o = dr.attend(h, cache, 0, at.PageTable(*flat(rows)), i32(lens), planned(h, trees, most), q, window=window)
        torch.cuda.synchronize()
        use[seqs] = held(h)
        some = [s for s in range(seqs) if s % 97 == 5 or s % 200 == 9 or s % 50 == 0]      # (long ones, large trees, others)
        ptr = sums(map(len, trees))
        of = lambda t: torch.cat([t[ptr[s]:ptr[s + 1], :8] for s in some])  # noqa: E731
        host = HostCache(cache, 0)
        host.code, host.scale = [c[:, :1] for c in host.code], [c[:, :1] for c in host.scale]
        check(str(seqs), of(o), *tree_reference(host, [rows[s] for s in some], [lens[s] for s in some], [trees[s] for s in some], of(q), 1 / math.sqrt(d), window=window))
    # a cell is 128 rows of 128 channels in 32 bits; four for each workgroup that the card holds
    cells = 4 * 2 * torch.cuda.get_device_properties(0).multi_processor_count
    assert use[600] <= cells * (128 * 128 * 4 + 128 * 8) + 2 ** 20, use


def test_attend_one_nan_among_drafted_values_costs_little(h):
    """A drafted value that is NaN is looked for in the pages that some node does not see as a whole, not in a whole context."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    lens, trees = [40000, 39000], [grown(60, 8, 4), grown(50, 9, 4)]
    cache, rows = filled(10, 1, 1260, 4, 128), rows_for(lens, 1260, 5)
    table, plan, lengths, q = at.PageTable(*flat(rows)), planned(h, trees), i32(lens), randn(gen, (110, 16, 128), BF)
    run = lambda: dr.attend(h, cache, 0, table, lengths, plan, q)  # noqa: E731
    clean, before = run(), times(run)
    token = lens[0] - 1
    cache.v[0, rows[0][token // PAGE], 0, 5, token % PAGE] = 0x7F
    assert (run().isnan() != clean.isnan()).sum() == 4                  # (the last node, the four heads of key head 0, a channel)
    assert times(run) < 1.5 * before + 20
