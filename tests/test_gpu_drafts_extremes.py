"""Drafted tokens at the ends of the ranges."""
import ctypes as C
import math

import pytest
import torch

from attn_helpers import PAGE, HostCache, check, flat
from draft_helpers import keep_reference, tree_reference
from paper_2404_04541_amd import attention as at
from paper_2404_04541_amd import binding as sg
from paper_2404_04541_amd import drafts as dr
from test_gpu_drafts import filled, grown, i32, i64, planned, randn, rows_for

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
