"""Attention over planned masks, forward and backward, against 64 bits on the CPU: masks, head layouts, lengths, strides, types; gradients also
against differences; what is masked may hold anything; streams, graphs, refusals that need the GPU."""
import math

import pytest
import torch

import attn_helpers
from attn_helpers import check, reference, visible
from paper_2404_04541_amd import attention as at
from paper_2404_04541_amd import binding as sg

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def h():
    return sg.Handle()


def ints(values, dtype=torch.int64):
    return torch.tensor(values, dtype=dtype, device="cuda")


def tensors(seed, dtype, tq, tk, hq, hkv, d):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda n, heads, scale: (torch.randn((n, heads, d), generator=gen, device="cuda") * scale).to(dtype)  # noqa: E731
    return make(tq, hq, 1.5), make(tk, hkv, 1.5), make(tk, hkv, 1.0), make(tq, hq, 1.0)


def plan_of(h, tq, tk, q_ptr=None, k_ptr=None, prefix=None, causal=True, window=0, tiles=None):
    return at.symbolic(h, tq, tk, q_ptr=ints(q_ptr) if q_ptr else None, k_ptr=ints(k_ptr) if k_ptr else None, prefix=ints(prefix) if prefix else None, causal=causal,
                       window=window, tiles=(ints(tiles[0]), ints(tiles[1], torch.int32)) if tiles else None)


def run(h, q, k, v, d_o, mask, cap=0.0, slopes=None, scale=None):
    """All results against the reference; returns them."""
    plan = plan_of(h, q.shape[0], k.shape[0], **mask)
    o, lse = at.forward(h, plan, q, k, v, scale=scale, cap=cap, slopes=slopes)
    dq, dk, dv = at.backward(h, plan, q, k, v, o, lse, d_o, scale=scale, cap=cap, slopes=slopes)
    seen, diag = visible(q.shape[0], k.shape[0], **mask)
    want = reference(q, k, v, d_o, seen, diag, scale or 1 / math.sqrt(q.shape[2]), cap, slopes)
    got = {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    for name, (value, bound) in want.items():
        check(name, got[name], value, bound)
    return got


MASKS = {
    "one": (1, 1, {}),
    "two": (2, 2, {}),
    "one_query": (1, 200, {}),
    "one_key": (200, 1, {}),
    "all": (65, 130, {"causal": False}),
    "causal": (300, 300, {}),
    "more_keys": (70, 301, {}),
    "more_queries": (301, 70, {}),                                                       # rows before the first key see nothing
    "window": (300, 333, {"window": 50}),
    "window_one": (130, 130, {"window": 1}),
    "window_past_only": (100, 100, {"causal": False, "window": 7}),
    "prefix": (200, 200, {"q_ptr": [0, 90, 200], "k_ptr": [0, 90, 200], "prefix": [40, 110]}),
    "prefix_window": (150, 150, {"q_ptr": [0, 150], "k_ptr": [0, 150], "prefix": [100], "window": 30}),
    "documents": (300, 300, {"q_ptr": [0, 1, 1, 64, 65, 200, 300], "k_ptr": [0, 1, 1, 64, 65, 200, 300]}),
    "no_keys": (100, 60, {"q_ptr": [0, 40, 70, 100], "k_ptr": [0, 30, 30, 60]}),           # the second document has none
    "no_queries": (60, 200, {"q_ptr": [0, 30, 30, 60], "k_ptr": [0, 30, 160, 200]}),
    "outside": (200, 260, {"q_ptr": [10, 100, 150], "k_ptr": [20, 130, 200]}),             # tokens before the first and behind the last document
    "pattern": (400, 500, {"tiles": ([0, 2, 2, 5, 6], [1, 0, 3, 0, 3, 1])}),              # unordered, repeated, an empty row
    "pattern_documents": (260, 260, {"q_ptr": [0, 130, 260], "k_ptr": [0, 130, 260], "tiles": ([0, 1, 3, 5], [0, 0, 1, 2, 1])}),
    "pattern_empty": (130, 130, {"tiles": ([0, 0, 0], [])}),
}


@pytest.mark.parametrize("name", MASKS)
@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
def test_masks(h, name, dtype):
    tq, tk, mask = MASKS[name]
    got = run(h, *tensors(1, dtype, tq, tk, 2, 1, 64), mask)
    seen, _ = visible(tq, tk, **mask)
    empty = ~seen.any(1)
    assert (got["o"].cpu()[empty] == 0).all() and (got["dq"].cpu()[empty] == 0).all() and (got["lse"].cpu()[:, empty] == -math.inf).all()


@pytest.mark.parametrize("d", [8, 40, 64, 72, 128])
@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (8, 1), (16, 16)])
def test_heads(h, d, heads):
    run(h, *tensors(2, BF, 150, 190, *heads, d), {"q_ptr": [0, 40, 150], "k_ptr": [0, 60, 190]})


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap, bias", [(5.0, False), (30.0, True), (0.0, True)])
def test_scores(h, dtype, d, cap, bias):
    slopes = torch.tensor([0.5, 0.03, 0.0, -0.01], device="cuda") if bias else None
    run(h, *tensors(3, dtype, 200, 260, 4, 2, d), {"q_ptr": [0, 70, 200], "k_ptr": [0, 100, 260]}, cap=cap, slopes=slopes, scale=0.3)


def test_long_rows(h):
    """Many tiles a row, both buffers, maxima that grow late."""
    q, k, v, d_o = tensors(4, BF, 130, 2900, 2, 2, 128)
    k[2500:] *= 3
    run(h, q, k, v, d_o, {})
    run(h, q, k, v, d_o, {"causal": False, "tiles": ([0, 4, 7], [0, 5, 6, 22, 3, 4, 21])})


@pytest.mark.parametrize("tq, tk", [(1024, 1024), (1025, 1024), (1024, 1025), (1, 1025), (1030, 1)])
def test_around_a_small_plan(h, tq, tk):
    """Masks of at most 1024 queries and keys are planned by one workgroup."""
    run(h, *tensors(41, BF, tq, tk, 2, 1, 64), {"q_ptr": [0, tq // 3, tq], "k_ptr": [0, tk // 2, tk], "window": 500})


@pytest.mark.parametrize("tq, tk", [(33100, 90), (262200, 70), (90, 16500), (70, 131200)])
def test_many_tiles_in_order(h, tq, tk):
    """Tiles are ordered by their work: up to 256 of them by counting, more by sorting, whose works LDS holds or does not.  Documents of a few thousand tokens, so that
    sums stay as short as the bounds take them to be."""
    docs = min(tq, tk) // 2
    cut = lambda n: [int(n * (i / docs) ** 1.2) for i in range(docs + 1)]  # noqa: E731
    run(h, *tensors(42, BF, tq, tk, 1, 1, 8), {"q_ptr": cut(tq), "k_ptr": cut(tk), "causal": False})


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap, bias", [(0.0, False), (20.0, False), (100.0, False), (20.0, True), (0.0, True)])
def test_rows_in_pieces(h, d, cap, bias):
    """Few workgroups and long rows (and columns, and heads that share them): their work is cut into pieces and joined."""
    slopes = torch.tensor([0.02, 0.001, 0.0, 0.1], device="cuda") if bias else None
    run(h, *tensors(23, BF, 90, 2300, 4, 2, d), {}, cap=cap, slopes=slopes)
    run(h, *tensors(24, BF, 1500, 70, 4, 1, d), {"causal": False}, cap=cap, slopes=slopes)
    run(h, *tensors(25, F16, 700, 700, 4, 2, d), {"window": 600, "tiles": ([0, 1, 3, 5, 7, 9, 12], [0, 0, 1, 0, 2, 1, 3, 0, 4, 0, 2, 5])}, cap=cap, slopes=slopes)


@pytest.mark.parametrize("cap", [1.0, 30.0, 50.0, 52.0, 60.0])
def test_scores_at_the_cap(h, cap):
    """Rows whose scores are all at the cap, all at its negative, or both: no power over- or underflows on the way."""
    q, k, v, _ = tensors(26, BF, 96, 200, 1, 1, 64)
    one = torch.ones(64, dtype=BF, device="cuda")
    q[:32], q[32:64], k[:] = one, -one, one * 8
    k[100:, :, :] = -8 * one
    q[64:] = 4 * one
    plan = plan_of(h, 96, 200, causal=False)
    o, lse = at.forward(h, plan, q, k, v, scale=4.0, cap=cap)
    seen, diag = visible(96, 200, causal=False)
    want = reference(q, k, v, None, seen, diag, 4.0, cap)
    check("o", o, *want["o"])
    check("lse", lse, *want["lse"])
    mask = {"q_ptr": [0, 96], "k_ptr": [0, 100]}          # only keys at one end: every score of rows 32 to 63 is -cap
    plan = plan_of(h, 96, 200, **mask, causal=False)
    o, lse = at.forward(h, plan, q, k, v, scale=4.0, cap=cap)
    seen, diag = visible(96, 200, **mask, causal=False)
    want = reference(q, k, v, None, seen, diag, 4.0, cap)
    check("o", o, *want["o"])
    check("lse", lse, *want["lse"])


def test_views(h):
    """One tensor of queries, keys and values; heads before tokens; gradients come in plain layout."""
    d, dtype = 64, BF
    gen = torch.Generator(device="cuda").manual_seed(5)
    packed = torch.randn((150, 8, d), generator=gen, device="cuda").to(dtype)
    q, k, v = packed[:, :4], packed[:, 4:6], packed[:, 6:]
    d_o = torch.randn((4, 150, d), generator=gen, device="cuda").to(dtype).transpose(0, 1)
    a = run(h, q, k, v, d_o, {})
    b = run(h, q.contiguous(), k.contiguous(), v.contiguous(), d_o.contiguous(), {})
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_same_bits_again(h):
    x = tensors(6, BF, 700, 700, 8, 2, 128)
    mask = {"q_ptr": [0, 300, 700], "k_ptr": [0, 300, 700]}
    plan = plan_of(h, 700, 700, **mask)
    first = None
    for _ in range(3):
        o, lse = at.forward(h, plan, *x[:3], cap=20.0)
        res = (o, lse) + at.backward(h, plan, *x[:3], o, lse, x[3], cap=20.0)
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, res))
        first = res


def test_outside_documents_anything(h):
    """Tokens of no document hold NaN and infinities: nobody's result shows them, and they get no gradient."""
    mask = {"q_ptr": [10, 100, 150], "k_ptr": [20, 130, 200]}
    q, k, v, d_o = tensors(7, BF, 200, 260, 4, 2, 64)
    clean = run(h, q, k, v, d_o, mask)
    for t, a, b in ((q, 10, 150), (d_o, 10, 150), (k, 20, 200), (v, 20, 200)):
        t[:a] = math.nan
        t[b:] = math.inf
    plan = plan_of(h, 200, 260, **mask)
    o, lse = at.forward(h, plan, q, k, v)
    got = {"o": o, "lse": lse, **dict(zip(("dq", "dk", "dv"), at.backward(h, plan, q, k, v, o, lse, d_o)))}
    for n in clean:
        assert torch.equal(clean[n], got[n]), n


def test_visible_nan_is_seen(h):
    q, k, v, _ = tensors(8, BF, 64, 64, 1, 1, 64)
    v[40, 0, 3] = math.nan
    o, _ = at.forward(h, plan_of(h, 64, 64), q, k, v)
    assert o[40:, 0, 3].isnan().all()


def test_large_scores(h):
    """Scores of thousands: the running maximum keeps every power finite, and rows become choices."""
    q, k, v, _ = tensors(9, F16, 100, 100, 2, 2, 64)
    plan = plan_of(h, 100, 100)
    o, lse = at.forward(h, plan, q, k, v, scale=400.0)
    best = (q.double().transpose(0, 1) @ k.double().transpose(0, 1).transpose(1, 2) * 400).masked_fill(~torch.tril(torch.ones(100, 100, dtype=torch.bool, device="cuda")), -math.inf)
    assert torch.isfinite(o).all() and torch.allclose(lse.double(), torch.logsumexp(best, -1), rtol=1e-5)


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("peak", [63, 60, 31, 4])
def test_maxima_that_rise_with_every_tile(h, dtype, d, peak):
    """Of every whole tile of 64 keys one, at its end or elsewhere, has a score that is 32 above the one of the tile before: with that maximum a power would be 2^46."""
    q, k, v, d_o = tensors(27, dtype, 160, 576, 2, 1, d)
    q *= 0.5
    k *= 0.5
    q[:, :, 0], k[:, :, 0] = 8, 0
    for tile in range(9):
        k[64 * tile + peak, :, 0] = 4 * tile
    x = (q, k, v, d_o)
    first = run(h, *x, {"causal": False}, scale=1.0)
    for _ in range(3):
        again = run(h, *x, {"causal": False}, scale=1.0)
        assert all(torch.equal(first[n], again[n]) for n in first)


def test_gradients_against_differences(h):
    """Central differences of the definition in 64 bits, at entries all over the tensors."""
    mask, cap, scale = {"q_ptr": [0, 20, 50], "k_ptr": [0, 25, 60], "window": 30}, 8.0, 0.4
    slopes = torch.tensor([0.2, 0.0, 0.05, 0.4], device="cuda")
    x = tensors(10, F16, 50, 60, 4, 2, 16)
    got = run(h, *x, mask, cap=cap, slopes=slopes, scale=scale)
    seen, diag = visible(50, 60, **mask)
    bounds = reference(*x, seen, diag, scale, cap, slopes)
    host = [t.cpu().double() for t in x]

    def loss(parts):
        total = 0.0
        for head in range(4):
            q, k, v, g = parts[0][:, head], parts[1][:, head // 2], parts[2][:, head // 2], parts[3][:, head]
            raw = q @ k.T * scale
            s = cap * torch.tanh(raw / cap) - float(slopes[head]) * (diag[:, None] - torch.arange(60)).abs()
            p = torch.nan_to_num(torch.softmax(s.masked_fill(~seen, -math.inf), 1), 0.0)
            total = total + (p @ v * g).sum()
        return float(total)

    rng = torch.Generator().manual_seed(0)
    for which, name in enumerate(("dq", "dk", "dv")):
        for _ in range(12):
            at_ = tuple(int(torch.randint(n, (1,), generator=rng)) for n in host[which].shape)
            step, values = 1e-5, []
            for sign in (1, -1):
                moved = [t.clone() for t in host]
                moved[which][at_] += sign * step
                values.append(loss(moved))
            slope = (values[0] - values[1]) / (2 * step)
            assert abs(float(got[name][at_]) - slope) <= 1.01 * float(bounds[name][1][at_]) + 1e-6, (name, at_)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap, bias", [(0.0, False), (30.0, False), (0.0, True), (30.0, True)])
@pytest.mark.parametrize("size", [2.0 ** -18, 2.0 ** -10, 1.0])
def test_small_gradients_in_float16(h, monkeypatch, size, d, cap, bias):
    """The digits of a score's gradient do not depend on how large d_o is: it is scaled, by a power of two for each row or key, before it becomes an operand.
    The scale is 2^15, or what brings the largest of a row or key below 2^15: those here are below 2^7, so that half of float16's smallest
    step, 2^-25, stands for at most 2^-33, and for 2^-40 where they are below 1.  (Scores lie within 8 of each other: no probability of the forward
    pass is below float16's normal range.)  Queries and keys are small and the factor of the scores is large, so that the gradients are not."""
    slopes = torch.tensor([0.002, 0.001, 0.0, 0.003], device="cuda") if bias else None
    gen = torch.Generator(device="cuda").manual_seed(28)
    part = lambda n, heads: torch.randn((n, heads, d), generator=gen, device="cuda").clamp(-2.5, 2.5)  # noqa: E731
    scale = 2.0 ** 19 / d ** 0.5
    monkeypatch.setitem(attn_helpers.TINY, F16, 2.0 ** -33 if size == 1.0 else 2.0 ** -40)
    for tq, tk, mask in ((200, 1000, {"causal": False}), (700, 700, {"q_ptr": [0, 200, 700], "k_ptr": [0, 200, 700]})):
        q, k, v, d_o = part(tq, 4) * 2.0 ** -10, part(tk, 2) * 2.0 ** -10, part(tk, 2), part(tq, 4) * size
        run(h, *(t.to(F16) for t in (q, k, v, d_o)), mask, cap=cap, slopes=slopes, scale=scale)


def test_probabilities_of_long_rows_in_float16(h, monkeypatch):
    """Rows of 196 608 equal scores: each probability is 85.3 of float16's smallest steps, and keeps its digits as an operand of the values' gradient, where it is
    2^15 times as large.  (In the forward pass they are 1 before the division.)"""
    monkeypatch.setitem(attn_helpers.TINY, F16, 2.0 ** -40)
    q, k, v, d_o = tensors(29, F16, 64, 3 << 16, 1, 1, 8)
    run(h, torch.zeros_like(q), k, v, d_o.abs() * 1024, {"causal": False})


@pytest.mark.parametrize("cap", [0.0, 3000.0])
def test_large_gradients_in_float16(h, cap):
    """Scores' gradients beyond float16's largest number, between inputs and gradients that it holds."""
    q, k, v, d_o = tensors(30, F16, 300, 400, 4, 2, 64)
    run(h, q * 16, k * 16, v * 256, d_o * 256, {"q_ptr": [0, 100, 300], "k_ptr": [0, 150, 400]}, scale=2.0 ** -12, cap=cap)


def test_autograd(h):
    q, k, v, d_o = (t.requires_grad_() for t in tensors(11, BF, 90, 90, 4, 2, 64))
    plan = plan_of(h, 90, 90)
    (at.attention(h, plan, q, k, v, cap=10.0) * d_o.detach()).sum().backward()
    o, lse = at.forward(h, plan, q.detach(), k.detach(), v.detach(), cap=10.0)
    want = at.backward(h, plan, q.detach(), k.detach(), v.detach(), o, lse, d_o.detach(), cap=10.0)
    assert all(torch.equal(a.grad, b) for a, b in zip((q, k, v), want))


def test_stream_of_its_own():
    stream = torch.cuda.Stream()
    x = tensors(12, BF, 200, 200, 4, 2, 64)
    torch.cuda.synchronize()
    handle = sg.Handle(stream=stream)
    with torch.cuda.stream(stream):
        run(handle, *x, {"q_ptr": [0, 80, 200], "k_ptr": [0, 80, 200]})
    stream.synchronize()


def test_results_belong_to_the_stream():
    """With another stream current, a result that is dropped at once is not the next tensor of that stream: the work may still be writing it."""
    handle = sg.Handle(stream=torch.cuda.Stream())
    q, k, v, d_o = tensors(14, BF, 300, 300, 4, 4, 64)
    q_ptr = ints([0, 300])
    torch.cuda.synchronize()
    plan = at.symbolic(handle, 300, 300, q_ptr=q_ptr, k_ptr=q_ptr)
    o, lse = at.forward(handle, plan, q, k, v)
    grads = at.backward(handle, plan, q, k, v, o, lse, d_o)
    handle.stream.synchronize()
    mine = {t.data_ptr() for t in (plan.memory, o, lse, *grads)}
    sizes = [t.numel() * t.element_size() for t in (plan.memory, o, lse, *grads)]
    del plan, o, lse, grads
    assert not mine & {t.data_ptr() for t in [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]}


def test_graph(h):
    """Captured once, replayed on new inputs with the program's own work between: every replay is the eager result."""
    stream = torch.cuda.Stream()
    handle = sg.Handle(stream=stream)
    q_ptr = ints([0, 100, 260])
    x = list(tensors(13, BF, 260, 260, 4, 2, 64))

    def step():
        plan = at.symbolic(handle, 260, 260, q_ptr=q_ptr, k_ptr=q_ptr, check=False)
        o, lse = at.forward(handle, plan, *x[:3])
        return (o, lse) + at.backward(handle, plan, *x[:3], o, lse, x[3])

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = step()
    for seed in range(14, 18):
        for t, new in zip(x, tensors(seed, BF, 260, 260, 4, 2, 64)):
            t.copy_(new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            want = step()
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed


def test_graph_after_a_larger_call():
    """A graph keeps its scratch memory when a later call on the handle needs more: a replay gives the eager result, and writes nothing that belongs to others."""
    stream = torch.cuda.Stream()
    handle, other = sg.Handle(stream=stream), sg.Handle(stream=stream)
    q_ptr, large_ptr = ints([0, 100, 260]), ints([0, 3000])
    x = list(tensors(31, BF, 260, 260, 4, 2, 64))
    large = tensors(32, BF, 3000, 3000, 4, 2, 64)

    def step(which, x, ptr):
        n = x[0].shape[0]
        plan = at.symbolic(which, n, n, q_ptr=ptr, k_ptr=ptr, check=False)
        o, lse = at.forward(which, plan, *x[:3])
        return (o, lse) + at.backward(which, plan, *x[:3], o, lse, x[3])

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(handle, x, q_ptr)
    stream.synchronize()
    before = dict(handle._live)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = step(handle, x, q_ptr)
    sizes = [t.numel() for t in handle._live.values()]
    with torch.cuda.stream(stream):
        first = step(handle, large, large_ptr)
        assert all(p in handle._live for p in before)                          # kept, and a block of at least twice the size beside it
        assert len(handle._live) == len(before) + 1 and max(t.numel() for t in handle._live.values()) >= 2 * max(sizes)
        others = [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for n in sizes * 8]
    for seed in range(33, 36):
        for t, new in zip(x, tensors(seed, BF, 260, 260, 4, 2, 64)):
            t.copy_(new)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
            again = step(handle, large, large_ptr)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            want = step(other, x, q_ptr)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed
        assert all(torch.equal(a, b) for a, b in zip(first, again)) and all((t == 77).all() for t in others)
    live = handle._live
    handle.close()
    assert not live


def test_scratch_without_graphs_is_replaced():
    """Where no graph has it, a block that is too small goes when a larger one comes."""
    handle = sg.Handle()
    for n in (260, 3000):
        x = tensors(34, BF, n, n, 4, 2, 64)
        plan = plan_of(handle, n, n)
        o, lse = at.forward(handle, plan, *x[:3])
        at.backward(handle, plan, *x[:3], o, lse, x[3])
        assert len(handle._live) == 1


def test_documents_are_checked(h):
    good = dict(q_ptr=ints([0, 50, 100]), k_ptr=ints([0, 50, 100]))
    at.symbolic(h, 100, 100, **good)
    for bad in (dict(good, q_ptr=ints([0, 60, 50])), dict(good, k_ptr=ints([0, 50, 101])), dict(good, q_ptr=ints([-1, 50, 100])), dict(good, prefix=ints([1, -1])),
                dict(good, tiles=(ints([0, 1]), ints([1], torch.int32))), dict(good, tiles=(ints([0, 2]), ints([0], torch.int32)))):
        with pytest.raises(sg.SpgemmError) as e:
            at.symbolic(h, 100, 100, **bad)
        assert e.value.status == -8


def test_a_large_pattern_is_checked(h):
    """Beyond 1024 tokens, where a plan's launches are others: 9 x 9 tiles."""
    rows = list(range(10))
    at.symbolic(h, 1100, 1100, tiles=(ints(rows), ints([8, 0, 1, 2, 3, 4, 5, 6, 7], torch.int32)))
    for ptr, cols in ((rows, [0, 1, 2, 3, 9, 5, 6, 7, 8]), (rows, [0, 1, 2, 3, 4, 5, 6, 7, -1]), (rows[:-1] + [10], list(range(9))), ([0, 2, 1] + rows[3:], list(range(9)))):
        with pytest.raises(sg.SpgemmError) as e:
            at.symbolic(h, 1100, 1100, tiles=(ints(ptr), ints(cols, torch.int32)))
        assert e.value.status == -8


def test_unchecked_documents_are_cut(h):
    """Pointers that leave the tensors, not looked at by the host: every access stays inside, rows see what exists."""
    q, k, v, _ = tensors(19, BF, 100, 100, 1, 1, 64)
    plan = at.symbolic(h, 100, 100, q_ptr=ints([0, 50, 5000]), k_ptr=ints([0, 50, 7000]), check=False)
    o, _ = at.forward(h, plan, q, k, v)
    want, _ = at.forward(h, plan_of(h, 100, 100, [0, 50, 100], [0, 50, 100]), q, k, v)
    assert torch.equal(o, want)


def test_arguments(h):
    q, k, v, d_o = tensors(20, BF, 64, 64, 4, 2, 64)
    plan = plan_of(h, 64, 64)
    bad = torch.zeros((64, 4, 65), dtype=BF, device="cuda")[:, :, 1:]
    odd = torch.zeros((64, 4, 68), dtype=BF, device="cuda")[:, :, :64]
    for args, kind in (((q[:63], k, v), ValueError), ((q.float(), k, v), TypeError), ((q, k.half(), v), TypeError), ((q, k, v[:, :, :32]), ValueError),
                       ((q.transpose(1, 2), k, v), ValueError), ((bad, k, v), sg.SpgemmError), ((odd, k, v), sg.SpgemmError), ((q[:, :3], k, v), sg.SpgemmError)):
        with pytest.raises(kind):
            at.forward(h, plan, *args)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(cap=-1.0), dict(cap=math.inf), dict(scale=math.nan), dict(cap=1e-39)):
        with pytest.raises(sg.SpgemmError):
            at.forward(h, plan, q, k, v, **kw)
    with pytest.raises(ValueError):
        at.forward(h, plan, q, k, v, slopes=torch.zeros(3, device="cuda"))


def test_nothing_to_do(h):
    q, k, v, d_o = tensors(21, BF, 0, 10, 2, 1, 64)
    plan = plan_of(h, 0, 10)
    o, lse = at.forward(h, plan, q, k, v)
    dq, dk, dv = at.backward(h, plan, q, k, v, o, lse, d_o)
    assert o.numel() == 0 and (dk == 0).all() and (dv == 0).all()
    q, k, v, d_o = tensors(22, BF, 10, 0, 2, 1, 64)
    plan = plan_of(h, 10, 0)
    o, lse = at.forward(h, plan, q, k, v)
    dq, dk, dv = at.backward(h, plan, q, k, v, o, lse, d_o)
    assert (o == 0).all() and (lse == -math.inf).all() and (dq == 0).all() and dk.numel() == 0
