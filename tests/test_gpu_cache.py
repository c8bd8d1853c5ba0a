"""The 8-bit paged cache: what an append leaves in it (bit for bit), attention over it against 64 bits, page tables and their copies."""
import ctypes as C
import math
import random

import pytest
import torch

from attn_helpers import MOST, PAGE, HostCache, attend_reference, check, flat, fork_reference, room_of, unflat
from paper_2404_04541_amd import attention as at
from paper_2404_04541_amd import binding as sg

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


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
    """A cache of random codes and scales; channels behind the head's are anything."""
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


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [8, 64, 72, 128])
def test_append(h, dtype, d):
    """Ragged numbers of new tokens: none, within a page, from a page's begin, over several pages; scales that stay and scales that rise."""
    heads = 3
    had = [0, 5, 64, 100, 63, 0, 130, 10]
    new = [1, 3, 200, 0, 1, 64, 62, 150]
    cache = filled(1, 2, 40, heads, d)
    gen = torch.Generator(device="cuda").manual_seed(2)
    lens = [a + b for a, b in zip(had, new)]
    rows = rows_for(lens, 40, spare=1)
    table = at.PageTable(*flat(rows))
    ptr = [0]
    for n in new:
        ptr.append(ptr[-1] + n)
    k, v = randn(gen, (ptr[-1], heads, d), dtype), randn(gen, (ptr[-1], heads, d), dtype)
    k[ptr[1]:ptr[2]] *= 40      # a scale that rises
    v[ptr[7]:] *= 1e-3
    host, other = HostCache(cache, 1), HostCache(cache, 0)
    host.append(rows, lens, ptr, k, v)
    at.append(h, cache, 1, table, i32(lens), i64(ptr), k, v)
    host.same(cache, 1, rows, lens)
    other.same(cache, 0, rows, had)


def test_append_leaves_the_rest(h):
    """Bytes behind the last token, other pages and other heads' scales stay as they are."""
    cache = filled(3, 1, 6, 2, 64)
    before = clone(cache)
    table = at.PageTable(*flat([[4, 1]]))
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = randn(gen, (1, 2, 64), BF, 1e-3), randn(gen, (1, 2, 64), BF, 1e-3)
    at.append(h, cache, 0, table, i32([70]), i64([0, 1]), k, v)
    keep = torch.ones(6, dtype=torch.bool)
    keep[1] = False
    for a, b in ((cache.k, before.k), (cache.v, before.v), (cache.k_scale, before.k_scale), (cache.v_scale, before.v_scale)):
        assert torch.equal(a[:, keep], b[:, keep])
    rest = torch.ones(PAGE, dtype=torch.bool)
    rest[5] = False
    assert torch.equal(cache.k[0, 1][:, rest], before.k[0, 1][:, rest]) and torch.equal(cache.v[0, 1][..., rest], before.v[0, 1][..., rest])


def test_append_token_by_token_reaches_one_call(h):
    """Scales after single tokens are those of one call; the entries are off by the roundings in between only."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v = randn(gen, (130, 2, 64), BF), randn(gen, (130, 2, 64), BF)
    one, many = at.PagedCache.empty(1, 4, 2, 64), at.PagedCache.empty(1, 4, 2, 64)
    table = at.PageTable(*flat([[2, 0, 3]]))
    at.append(h, one, 0, table, i32([130]), i64([0, 130]), k, v)
    for i in range(130):
        at.append(h, many, 0, table, i32([i + 1]), i64([0, 1]), k[i:i + 1], v[i:i + 1])
    assert torch.equal(one.k_scale, many.k_scale) and torch.equal(one.v_scale, many.v_scale)
    a, b = HostCache(one, 0), HostCache(many, 0)
    for x in (0, 1):
        p, q = a.tokens(x, [2, 0, 3], 130), b.tokens(x, [2, 0, 3], 130)
        # two roundings instead of one: half a step of 2^-3 each, or half of the smallest step of the page's scale
        assert ((p - q).abs() <= 2 * (2.0 ** -4 * torch.maximum(p.abs(), q.abs()) + 2.0 ** -10 * a.scale[x].max())).all()


@pytest.mark.parametrize("value, code", [(0.0, 0.0), (math.inf, MOST), (-math.inf, -MOST), (math.nan, math.nan)])
def test_append_unusual_values(h, value, code):
    cache = at.PagedCache.empty(1, 2, 1, 64)
    k = torch.full((3, 1, 64), 1.0, dtype=BF, device="cuda")
    k[1, 0, 7] = value
    at.append(h, cache, 0, at.PageTable(*flat([[1]])), i32([3]), i64([0, 3]), k, k)
    host = HostCache(cache, 0)
    for x in (0, 1):
        got = host.code[x][1, 0, 1, 7]
        assert got.isnan() if math.isnan(code) else got == code
        assert host.code[x][1, 0, 0, 0] == 256 and host.scale[x][1, 0] == 2.0 ** -8     # 1.0 fits as 256 = 2^8 and not as 512


def test_append_without_pages(h):
    """A sequence whose table lacks the pages, one shorter than its new tokens, a page that the cache does not have: nothing is written for them."""
    cache = filled(6, 1, 4, 1, 64)
    before = clone(cache)
    gen = torch.Generator(device="cuda").manual_seed(7)
    k, v = randn(gen, (30, 1, 64), BF), randn(gen, (30, 1, 64), BF)
    at.append(h, cache, 0, at.PageTable(*flat([[], [1], [9], [-1]])), i32([10, 3, 5, 5]), i64([0, 10, 20, 25, 30]), k, v)
    assert torch.equal(cache.k, before.k) and torch.equal(cache.v, before.v) and torch.equal(cache.k_scale, before.k_scale)


CASES = {
    "one": dict(lens=[1], q_len=1, heads=(1, 1), d=64),
    "ends": dict(lens=[63, 64, 65, 0, 128, 129, 2], q_len=1, heads=(4, 2), d=64),
    "chunks": dict(lens=[5000, 1, 300, 2000], q_len=1, heads=(8, 2), d=128),
    "group_of_24": dict(lens=[200, 70], q_len=1, heads=(24, 1), d=72),
    "proposed": dict(lens=[5, 66, 300], q_len=5, heads=(6, 2), d=64),
    "more_queries_than_tokens": dict(lens=[3, 0, 70], q_len=8, heads=(2, 2), d=64),
    "window": dict(lens=[1000, 64, 40], q_len=3, heads=(4, 2), d=64, window=70),
    "window_one": dict(lens=[130, 128], q_len=2, heads=(2, 1), d=64, window=1),
    "cap": dict(lens=[700, 90], q_len=2, heads=(8, 4), d=128, cap=10.0),
    "bias": dict(lens=[700, 90], q_len=1, heads=(4, 2), d=64, slopes=[0.5, 0.01, 0.0, 0.1]),
    "cap_bias": dict(lens=[333], q_len=4, heads=(4, 2), d=40, slopes=[0.5, 0.01, 0.0, 0.1], cap=6.0, window=100),
    "small_head": dict(lens=[77], q_len=1, heads=(2, 1), d=8),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
def test_attend(h, name, dtype):
    c = CASES[name]
    (heads, kv), d, lens = c["heads"], c["d"], c["lens"]
    pages = sum(-(-n // PAGE) for n in lens) + 3
    cache = filled(8, 2, pages, kv, d)
    rows = rows_for(lens, pages, 1)
    for pages_of, n in zip(rows, lens):      # behind the last token: NaN
        if n % PAGE:
            cache.k[1, pages_of[-1], :, n % PAGE:] = 0x7F
            cache.v[1, pages_of[-1], :, :, n % PAGE:] = 0xFF
    gen = torch.Generator(device="cuda").manual_seed(9)
    q = randn(gen, (len(lens), c["q_len"], heads, d), dtype, 1.5)
    slopes = torch.tensor(c["slopes"], device="cuda") if "slopes" in c else None
    o = at.attend(h, cache, 1, at.PageTable(*flat(rows)), i32(lens), q, cap=c.get("cap", 0.0), slopes=slopes, window=c.get("window", 0))
    want, bound = attend_reference(HostCache(cache, 1), rows, lens, q, 1 / math.sqrt(d), c.get("cap", 0.0), slopes, c.get("window", 0))
    check(name, o, want, bound)


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [8, 40, 56, 72, 96, 120])
def test_attend_channels_behind_the_head_anything(h, dtype, d):
    """Channels from the head's last to the room's hold NaN in every page: no score and no result shows them, before and after tokens are added."""
    cache = filled(53, 1, 12, 2, d)
    cache.k[..., d:], cache.v[..., d:, :] = 0x7F, 0xFF
    cache.k[..., d::2], cache.v[..., d::2, :] = 0xFF, 0x7F
    lens, rows = [300, 64, 1], rows_for([300, 64, 1], 12, 2)
    gen = torch.Generator(device="cuda").manual_seed(54)
    q = randn(gen, (3, 2, 4, d), dtype, 1.5)
    table = at.PageTable(*flat(rows))
    host = HostCache(cache, 0)
    check("imported", at.attend(h, cache, 0, table, i32(lens), q), *attend_reference(host, rows, lens, q, 1 / math.sqrt(d)))
    k, v = randn(gen, (5, 2, d), dtype, 4.0), randn(gen, (5, 2, d), dtype, 4.0)
    lens = [304, 64, 2]
    host.append(rows, lens, [0, 4, 4, 5], k, v)
    at.append(h, cache, 0, table, i32(lens), i64([0, 4, 4, 5]), k, v)
    host.same(cache, 0, rows, lens)
    check("appended", at.attend(h, cache, 0, table, i32(lens), q), *attend_reference(host, rows, lens, q, 1 / math.sqrt(d)))


def test_attend_behind_a_window_anything(h):
    """Pages that no query's window reaches are not looked at, nor the tokens before it in its first page."""
    cache = filled(10, 1, 8, 1, 64)
    rows, lens = [[3, 5, 0, 7, 1]], [300]
    gen = torch.Generator(device="cuda").manual_seed(11)
    q = randn(gen, (1, 1, 2, 64), BF)
    table = at.PageTable(*flat(rows))
    want = at.attend(h, cache, 0, table, i32(lens), q, window=100)
    cache.k[0, [3, 5, 0]], cache.v[0, [3, 5, 0]], cache.k_scale[0, [3, 5, 0]] = 0x7F, 0x7F, math.nan
    cache.k[0, 7, :, :8], cache.v[0, 7, :, :, :8] = 0x7F, 0x7F       # keys 192 .. 199: the window begins at 200
    assert torch.equal(at.attend(h, cache, 0, table, i32(lens), q, window=100), want)


@pytest.mark.parametrize("dtype, large, small", [(BF, 2.0 ** 30, 0.0), (BF, 2.0 ** 30, 2.0 ** -90), (BF, 2.0 ** 100, 2.0 ** -100), (F16, 3e4, 0.0), (F16, 3e4, 2.0 ** -20)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("first", [0, 4])
def test_attend_pages_of_very_different_scales(h, dtype, large, small, d, first):
    """Four pages of large values and four of zeros or tiny ones in turn, in workgroups that go over eight: what a wave has summed up of one page stays finite next to any other."""
    gen = torch.Generator(device="cuda").manual_seed(55)
    tokens, kv, heads = 6400, 8, 64
    cache, rows = at.PagedCache.empty(1, 100, kv, d), rows_for([tokens], 100, 3)
    k, v = randn(gen, (tokens, kv, d), dtype), torch.rand((tokens, kv, d), generator=gen, device="cuda") + 0.5
    page = torch.arange(tokens, device="cuda") // PAGE
    v = (v * torch.where((page + first) % 8 < 4, large, small)[:, None, None]).to(dtype)
    table = at.PageTable(*flat(rows))
    at.append(h, cache, 0, table, i32([tokens]), i64([0, tokens]), k, v)
    q = randn(gen, (1, 16, heads, d), dtype)
    o = at.attend(h, cache, 0, table, i32([tokens]), q)
    check("o", o, *attend_reference(HostCache(cache, 0), rows, [tokens], q, 1 / math.sqrt(d)))


def test_shared_and_missing_pages(h):
    """Sequences over the same pages; a table with fewer pages than its lengths, and ids that do not exist: what is there is attended to."""
    cache = filled(12, 1, 10, 2, 64)
    gen = torch.Generator(device="cuda").manual_seed(13)
    q = randn(gen, (3, 1, 4, 64), BF)
    rows = [[2, 4, 6], [2, 4, 8], [2]]
    o = at.attend(h, cache, 0, at.PageTable(*flat(rows)), i32([190, 150, 500]), q)
    want, bound = attend_reference(HostCache(cache, 0), rows, [190, 150, 64], q, 1 / 8)
    check("shared", o, want, bound)
    o = at.attend(h, cache, 0, at.PageTable(*flat([[2, 99, -5, 6]])), i32([256]), q[:1])
    host = HostCache(cache, 0)
    ks, vs = (host.tokens(x, [2, 6], 128) for x in (0, 1))
    for head in range(4):
        p = torch.softmax(q[0, 0, head].cpu().double() @ ks[:, head // 2].T / 8, 0)
        assert (o[0, 0, head].cpu().double() - p @ vs[:, head // 2]).abs().max() <= (2 * 2.0 ** -8 + 2e-4) * (p @ vs[:, head // 2].abs()).max()


def test_far_pages(h):
    """Offsets of more than 32 bits: the last pages of a cache of 5 GB."""
    heads, d, pages = 16, 128, 20000
    k = torch.empty((1, 2 * pages, heads, PAGE, d), dtype=torch.uint8, device="cuda")
    v = torch.empty((1, 2 * pages, heads, d, PAGE), dtype=torch.uint8, device="cuda")
    cache = at.PagedCache(d, k, v, *[torch.ones((1, 2 * pages, heads), device="cuda") for _ in range(2)])
    near = at.PagedCache.empty(1, 3, heads, d)
    gen = torch.Generator(device="cuda").manual_seed(14)
    kk, vv, q = randn(gen, (100, heads, d), BF), randn(gen, (100, heads, d), BF), randn(gen, (1, 1, heads, d), BF)
    far_rows, near_rows = [[2 * pages - 1, 2 * pages - 3]], [[1, 2]]
    out = []
    for c, rows in ((cache, far_rows), (near, near_rows)):
        table = at.PageTable(*flat(rows))
        at.append(h, c, 0, table, i32([100]), i64([0, 100]), kk, vv)
        out.append(at.attend(h, c, 0, table, i32([100]), q))
    assert torch.equal(*out)
    at.copy_pages(h, cache, i32([2 * pages - 1, 2 * pages - 3]), i32([2 * pages - 2, 0]))
    assert torch.equal(at.attend(h, cache, 0, at.PageTable(*flat([[2 * pages - 2, 0]])), i32([100]), q), out[0])


def test_decode_graph(h):
    """One step of serving, captured: lengths live on the GPU, so each replay is the next token."""
    stream = torch.cuda.Stream()
    handle = sg.Handle(stream=stream)
    cache, eager = at.PagedCache.empty(1, 8, 2, 64), at.PagedCache.empty(1, 8, 2, 64)
    table = at.PageTable(*flat([[1, 3, 5], [0, 2, 4]]))
    lens, ptr = i32([0, 60]), i64([0, 1, 2])
    gen = torch.Generator(device="cuda").manual_seed(15)
    k, v, q = randn(gen, (2, 2, 64), BF), randn(gen, (2, 2, 64), BF), randn(gen, (2, 1, 4, 64), BF)
    first = randn(gen, (60, 2, 64), BF)
    for c in (cache, eager):
        at.append(h, c, 0, table, i32([0, 60]), i64([0, 0, 60]), first, first)

    def step(c):
        at.append(handle, c, 0, table, lens, ptr, k, v)
        return at.attend(handle, c, 0, table, lens, q)

    torch.cuda.synchronize()
    scratch = clone(cache)
    with torch.cuda.stream(stream):
        step(scratch)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = step(cache)
    for i in range(8):
        lens += 1
        for t in (k, v, q):
            t.copy_(randn(gen, t.shape, BF))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            want = step(eager)
        stream.synchronize()
        assert torch.equal(out, want) and torch.equal(cache.k, eager.k) and torch.equal(cache.v, eager.v), i


def test_decode_graph_after_a_larger_call(h):
    """A captured step of serving, and then a batch on the same handle that needs more scratch memory."""
    stream = torch.cuda.Stream()
    handle = sg.Handle(stream=stream)
    cache = filled(60, 1, 600, 2, 64)
    table, lens = at.PageTable(*flat([list(range(40)), list(range(40, 43))])), i32([2500, 130])
    many = at.PageTable(*flat([list(range(9 * i, 9 * i + 9)) for i in range(60)]))
    many_lens = i32([570] * 60)
    gen = torch.Generator(device="cuda").manual_seed(61)
    q, large = randn(gen, (2, 1, 4, 64), BF), randn(gen, (60, 4, 4, 64), BF)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        at.attend(handle, cache, 0, table, lens, q)
    stream.synchronize()
    sizes = [t.numel() for t in handle._live.values()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = at.attend(handle, cache, 0, table, lens, q)
    with torch.cuda.stream(stream):
        at.attend(handle, cache, 0, many, many_lens, large)
        assert len(handle._live) == 2
        others = [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for n in sizes * 4]
    for _ in range(3):
        q.copy_(randn(gen, q.shape, BF))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, at.attend(h, cache, 0, table, lens, q)) and all((t == 77).all() for t in others)


# ---- tables ---------------------------------------------------------------------------------------

def made_table(rng, rows, pages, most, shared):
    lens = [rng.randint(0, most) for _ in range(rows)]
    ids = rng.sample(range(pages), pages)
    out = []
    for n in lens:
        same = out[0][:min(shared, n // PAGE, lens[0] // PAGE)] if out else []
        out.append(same + [ids.pop() for _ in range(-(-n // PAGE) - len(same))])
    return lens, out


@pytest.mark.parametrize("seed", range(8))
def test_fork(h, seed):
    rng = random.Random(seed)
    n, n_out, pages = rng.choice([(1, 1, 20), (5, 9, 300), (70, 50, 2500), (3, 200, 1500)])
    d, layers = rng.choice([40, 128]), rng.choice([1, 3])
    lens, rows = made_table(rng, n, pages, 400, rng.randint(0, 3))
    parent = [rng.randrange(-1, n) for _ in range(n_out)]
    new = [max(0, (lens[p] if p >= 0 else 0) + rng.choice([0, 1, 1, 64, -rng.randint(0, 100)])) for p in parent]
    cache = filled(20 + seed, layers, pages, 2, d)
    before = clone(cache)
    out, refs = at.fork(h, cache, at.PageTable(*flat(rows)), i32(lens), i32(parent), i32(new))
    want, copies, want_refs = fork_reference(pages, rows, lens, parent, new)
    assert unflat(out) == want and refs.tolist() == want_refs
    for part, old in ((cache.k, before.k), (cache.v, before.v), (cache.k_scale, before.k_scale), (cache.v_scale, before.v_scale)):
        for src, dst in copies:
            old[:, dst] = old[:, src]
        assert torch.equal(part, old)


def test_fork_keeps_what_sequences_hold(h):
    """Beams that part ways: each has its parent's tokens and its own, whatever the others append."""
    cache = at.PagedCache.empty(1, 40, 2, 64)
    gen = torch.Generator(device="cuda").manual_seed(30)
    lens, rows = [100, 30], [[7, 9], [11]]
    k, v = randn(gen, (130, 2, 64), BF), randn(gen, (130, 2, 64), BF)
    at.append(h, cache, 0, at.PageTable(*flat(rows)), i32(lens), i64([0, 100, 130]), k, v)
    parent, new = [0, 0, 1, 0, 1], [101, 101, 31, 65, 20]
    held = HostCache(cache, 0)
    out, _ = at.fork(h, cache, at.PageTable(*flat(rows)), i32(lens), i32(parent), i32(new))
    table = unflat(out)
    grown = [n - min(lens[p], n) for p, n in zip(parent, new)]
    ptr = [0]
    for g in grown:
        ptr.append(ptr[-1] + g)
    at.append(h, cache, 0, out, i32(new), i64(ptr), randn(gen, (ptr[-1], 2, 64), BF, 1e-3), randn(gen, (ptr[-1], 2, 64), BF, 1e-3))
    now = HostCache(cache, 0)
    for r, p in enumerate(parent):
        n = min(lens[p], new[r])
        for x in (0, 1):
            assert torch.equal(now.tokens(x, table[r], n), held.tokens(x, rows[p], n)), (r, x)


def test_fork_refusals(h):
    cache = filled(31, 1, 6, 1, 64)
    before = clone(cache)
    lens, rows = [100, 64], [[0, 1], [2]]
    table = at.PageTable(*flat(rows))

    def status(*a, **kw):
        with pytest.raises(sg.SpgemmError) as e:
            at.fork(h, cache, table, i32(a[0]), i32(a[1]), i32(a[2]), **kw)
        return e.value.status

    assert status(lens, [2], [1]) == -8 and status(lens, [-2], [1]) == -8          # no such parent
    assert status(lens, [0], [-1]) == -8                                            # no such length
    assert status([200, 64], [0], [200]) == -8                                      # a parent without its pages
    assert status(lens, [0, 0], [101, 101], entries=3) == -8                         # too little room
    assert status(lens, [0, 0, 0, 0, 0, 0], [101] * 6) == -5                         # no page left
    assert status(lens, [-1], [64 * 7]) == -5
    bad = at.PageTable(table.rowptr, i32([0, 6, 2]))
    with pytest.raises(sg.SpgemmError):
        at.fork(h, cache, bad, i32(lens), i32([0]), i32([100]))
    for a, b in ((cache.k, before.k), (cache.v, before.v)):
        assert torch.equal(a, b)
    out, refs = at.fork(h, cache, table, i32(lens), i32([]), i32([]))              # every row ends
    assert out.rows == 0 and not refs.any()


def test_fork_of_lengths_beyond_the_cache(h):
    """Lengths near 2^31 in enough rows that their pages would pass 32 bits: refused, and nothing written, whatever room the table has."""
    cache = filled(32, 1, 6, 1, 64)
    before = clone(cache)
    table, lens = at.PageTable(*flat([[0, 1], [2]])), i32([100, 64])
    most = 2 ** 31 - 1
    for rows in (1, 63, 64, 65, 1100):
        guard = torch.full((rows + 4096,), -7, dtype=torch.int32, device="cuda")
        rowptr, refs = torch.empty(rows + 1, dtype=torch.int64, device="cuda"), torch.empty(6, dtype=torch.int32, device="cuda")
        new_lens, out = i32([most] * rows), guard[4096:]
        for parent in (-1, 0):
            parents = i32([parent] * rows)
            for room in (0, 3, 8):
                nnz = C.c_int64(0)
                status = at._lib().spcache_fork(h.ptr, C.byref(cache._struct), C.byref(table.struct(cache)), lens.data_ptr(), rows, parents.data_ptr(), new_lens.data_ptr(),
                                                rowptr.data_ptr(), out.data_ptr(), min(room, rows), refs.data_ptr(), C.byref(nnz))
                assert status == -5, (rows, parent, room)
                assert (guard == -7).all()
    with pytest.raises(sg.SpgemmError) as e:                                        # a length that the cache could hold, and one that it could not
        at.fork(h, cache, table, lens, i32([0, -1]), i32([100, most]), entries=2)
    assert e.value.status == -5
    with pytest.raises(sg.SpgemmError) as e:                                        # ... and a parent that there is not
        at.fork(h, cache, table, lens, i32([5, -1]), i32([100, most]), entries=2)
    assert e.value.status == -8
    assert torch.equal(cache.k, before.k) and torch.equal(cache.v, before.v)


@pytest.mark.parametrize("seed", range(6))
def test_compact(h, seed):
    rng = random.Random(100 + seed)
    n, pages = rng.choice([(1, 5), (9, 200), (60, 3000), (4, 1025)])
    lens, rows = made_table(rng, n, pages, 300, rng.randint(0, 2))
    cache = filled(40 + seed, 2, pages, 2, 64)
    before = clone(cache)
    out, live = at.compact(h, cache, at.PageTable(*flat(rows)))
    used = sorted({p for r in rows for p in r})
    holes = [p for p in range(len(used)) if p not in set(used)]
    to = dict(zip([p for p in used if p >= len(used)], holes))
    assert live == len(used) and unflat(out) == [[to.get(p, p) for p in r] for r in rows]
    for a, b in ((cache.k, before.k), (cache.v, before.v), (cache.k_scale, before.k_scale), (cache.v_scale, before.v_scale)):
        for src, dst in to.items():
            b[:, dst] = b[:, src]
        assert torch.equal(a, b)


def test_compact_bounds(h):
    cache = filled(50, 1, 70, 1, 64)
    before = clone(cache)
    for rows in ([list(range(70))], [[]], [[0, 1, 2]]):      # all in use, none, in front already
        out, live = at.compact(h, cache, at.PageTable(*flat(rows)))
        assert unflat(out) == rows and live == len(rows[0]) and torch.equal(cache.k, before.k)
    with pytest.raises(sg.SpgemmError):
        at.compact(h, cache, at.PageTable(*flat([[1, 70]])))
    assert torch.equal(cache.k, before.k)


def test_copy(h):
    cache = filled(51, 3, 20, 2, 128)
    want = clone(cache)
    src, dst = [3, 3, 9, 40, 1], [4, 0, 19, 5, -1]      # the last two are out of range
    at.copy_pages(h, cache, i32(src), i32(dst))
    for part, old in ((cache.k, want.k), (cache.v, want.v), (cache.k_scale, want.k_scale), (cache.v_scale, want.v_scale)):
        for a, b in list(zip(src, dst))[:3]:
            old[:, b] = old[:, a]
        assert torch.equal(part, old)


def test_arguments(h):
    cache = filled(52, 1, 4, 2, 64)
    table, lens = at.PageTable(*flat([[1]])), i32([10])
    k = torch.zeros((1, 2, 64), dtype=BF, device="cuda")
    q = torch.zeros((1, 1, 4, 64), dtype=BF, device="cuda")
    for call, kind in ((lambda: at.append(h, cache, 1, table, lens, i64([0, 1]), k, k), sg.SpgemmError),
                       (lambda: at.append(h, cache, 0, table, lens, i64([0]), k, k), ValueError),
                       (lambda: at.append(h, cache, 0, table, lens, i64([0, 1]), k[:, :1], k[:, :1]), ValueError),
                       (lambda: at.append(h, cache, 0, table, lens, i64([0, 1]), k.float(), k.float()), TypeError),
                       (lambda: at.attend(h, cache, -1, table, lens, q), sg.SpgemmError),
                       (lambda: at.attend(h, cache, 0, table, lens, q[:, :, :3]), sg.SpgemmError),
                       (lambda: at.attend(h, cache, 0, table, lens.long(), q), ValueError),
                       (lambda: at.attend(h, cache, 0, table, lens, q, window=-1), sg.SpgemmError),
                       (lambda: at.attend(h, cache, 0, table, lens, q, scale=0.0), sg.SpgemmError),
                       (lambda: at.attend(h, cache, 0, table, lens, q[0]), ValueError),
                       (lambda: at.copy_pages(h, cache, i32([0]), i32([1, 2])), ValueError),
                       (lambda: at.PagedCache(128, cache.k, cache.v, cache.k_scale, cache.v_scale), ValueError)):
        with pytest.raises(kind):
            call()
