"""Host-side checks of include/spattn.h that need no GPU: symbols, struct layouts, and refusals that come before the first HIP call."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "spattn.h")
INVALID_ARG, DIM_MISMATCH, UNSUPPORTED = -1, -2, -4


@pytest.fixture(scope="module")
def at():
    from paper_2404_04541_amd import attention, binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2404_04541_amd.build import build_library
        build_library()
    return attention


@pytest.fixture()
def h(at):
    lib, handle = at._lib(), C.c_void_p()
    assert lib.spgemm_create(C.byref(handle), None, None) == 0
    yield handle
    lib.spgemm_destroy(handle)


def test_every_declared_symbol_is_exported(at):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b((?:spattn|spcache)_[a-z_]+)\s*\(", text)))
    assert names == sorted(at.EXPORTED)
    for n in names:
        assert hasattr(at._lib(), n), n


def test_constants_and_layouts_match_the_header(at):
    text = open(HEADER).read()
    assert int(re.search(r"#define SPATTN_TILE (\d+)", text).group(1)) == at.TILE
    assert int(re.search(r"#define SPCACHE_PAGE (\d+)", text).group(1)) == at.PAGE
    assert re.search(r"SPATTN_F16 = (\d), SPATTN_BF16 = (\d)", text).groups() == (str(at.F16), str(at.BF16))
    assert C.sizeof(at.TensorStruct) == 24
    assert C.sizeof(at.MaskStruct) == 3 * 8 + 3 * 8 + 8 + 8 + 8          # sizes, pointers, causal (padded), window, pattern
    assert C.sizeof(at.ArgsStruct) == 2 * 8 + 4 * 4 + 2 * 4 + 8 + 3 * 24
    assert C.sizeof(at.CacheStruct) == 2 * 8 + 2 * 4 + 4 * 8


def mask(at, **kw):
    base = dict(q_len=100, k_len=200, docs=0, q_ptr=None, k_ptr=None, prefix=None, causal=1, window=0, tiles=None)
    return at.MaskStruct(*(base | kw).values())


def test_masks_are_refused(at, h):
    from paper_2404_04541_amd import binding as sg
    lib = at._lib()
    pattern = lambda *a: C.pointer(sg.CsrStruct(*a))  # noqa: E731
    for m, status in ((mask(at, q_len=-1), INVALID_ARG), (mask(at, window=-1), INVALID_ARG), (mask(at, causal=2), INVALID_ARG), (mask(at, k_len=1 << 30), UNSUPPORTED),
                      (mask(at, docs=2), INVALID_ARG), (mask(at, q_ptr=64, k_ptr=64), INVALID_ARG), (mask(at, tiles=pattern(2, 2, 1, 64, 64, None, 0)), DIM_MISMATCH),
                      (mask(at, tiles=pattern(1, 2, 1, None, 64, None, 0)), INVALID_ARG), (mask(at, tiles=pattern(1, 2, 1, 64, None, None, 0)), INVALID_ARG)):
        assert lib.spattn_symbolic(h, C.byref(m), C.c_void_p(256), 1 << 30, None) == status
        assert lib.spattn_plan_bytes(C.byref(m)) == 0 and lib.spgemm_last_error(h)
    good = mask(at, tiles=pattern(1, 2, 1, 64, 64, None, 0))
    need = lib.spattn_plan_bytes(C.byref(good))
    assert need > lib.spattn_plan_bytes(C.byref(mask(at))) > 100 * 16
    assert lib.spattn_symbolic(h, None, C.c_void_p(256), need, None) == INVALID_ARG
    assert lib.spattn_symbolic(h, C.byref(good), None, need, None) == INVALID_ARG
    assert lib.spattn_symbolic(h, C.byref(good), C.c_void_p(256), need - 1, None) == INVALID_ARG
    assert lib.spattn_symbolic(h, C.byref(good), C.c_void_p(128), need, None) == INVALID_ARG
    assert lib.spattn_symbolic(None, C.byref(good), C.c_void_p(256), need, None) == INVALID_ARG


def args(at, **kw):
    t = at.TensorStruct(1024, 512, 64)
    base = dict(mask=C.pointer(mask(at)), plan_mem=256, dtype=1, heads=8, kv_heads=2, head_dim=64, scale=0.1, cap=0.0, slopes=None, q=t, k=t, v=t)
    return at.ArgsStruct(*(base | kw).values())


def test_passes_are_refused(at, h):
    lib, t = at._lib(), at.TensorStruct(1024, 512, 64)
    cases = [(dict(plan_mem=None), INVALID_ARG), (dict(dtype=2), INVALID_ARG), (dict(heads=7), INVALID_ARG), (dict(kv_heads=0), INVALID_ARG),
             (dict(heads=1 << 17, kv_heads=1 << 17), UNSUPPORTED), (dict(head_dim=0), INVALID_ARG), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED),
             (dict(scale=0.0), INVALID_ARG), (dict(scale=float("nan")), INVALID_ARG), (dict(cap=-1.0), INVALID_ARG), (dict(cap=float("inf")), INVALID_ARG),
             (dict(q=at.TensorStruct(None, 512, 64)), INVALID_ARG), (dict(k=at.TensorStruct(1032, 512, 64)), UNSUPPORTED),
             (dict(v=at.TensorStruct(1024, 516, 64)), UNSUPPORTED), (dict(k=at.TensorStruct(1024, -8, 64)), INVALID_ARG),
             (dict(k=at.TensorStruct(1024, 1 << 23, 64)), UNSUPPORTED)]
    for kw, status in cases:
        a = args(at, **kw)
        assert lib.spattn_forward(h, C.byref(a), t, C.c_void_p(64)) == status, kw
        assert lib.spattn_backward(h, C.byref(a), t, C.c_void_p(64), t, t, t, t) == status, kw
    a = args(at)
    assert lib.spattn_forward(h, None, t, C.c_void_p(64)) == INVALID_ARG
    assert lib.spattn_forward(h, C.byref(a), t, None) == INVALID_ARG
    assert lib.spattn_forward(h, C.byref(a), at.TensorStruct(None, 0, 0), C.c_void_p(64)) == INVALID_ARG
    assert lib.spattn_backward(h, C.byref(a), t, None, t, t, t, t) == INVALID_ARG
    assert lib.spattn_backward(h, C.byref(a), t, C.c_void_p(64), t, t, at.TensorStruct(1030, 512, 64), t) == UNSUPPORTED


def test_cache_calls_are_refused(at, h):
    from paper_2404_04541_amd import binding as sg
    lib, t = at._lib(), at.TensorStruct(1024, 512, 64)
    cache = lambda **kw: C.byref(at.CacheStruct(*(dict(layers=1, pages=4, kv_heads=2, head_dim=64, k=64, v=64, k_scale=64, v_scale=64) | kw).values()))  # noqa: E731
    table = lambda rows=1, cols=4, nnz=1, ptr=64, col=64: C.byref(sg.CsrStruct(rows, cols, nnz, ptr, col, None, 0))  # noqa: E731
    p = C.c_void_p(64)
    append = lambda c, tab, lens=p, new=p, layer=0, tokens=1, dtype=1, k=t: lib.spcache_append(h, c, layer, tab, lens, new, tokens, dtype, k, t)  # noqa: E731
    for c, status in ((None, INVALID_ARG), (cache(layers=0), INVALID_ARG), (cache(head_dim=100), UNSUPPORTED), (cache(pages=1 << 24), UNSUPPORTED),
                      (cache(k=None), INVALID_ARG), (cache(v=72), UNSUPPORTED)):
        assert append(c, table()) == status
        assert lib.spcache_copy(h, c, 1, p, p) == status
        assert lib.spcache_compact(h, c, table(), p, None) == status
    for tab, status in ((None, INVALID_ARG), (table(rows=-1), INVALID_ARG), (table(ptr=None), INVALID_ARG), (table(col=None), INVALID_ARG), (table(cols=5), DIM_MISMATCH)):
        assert append(cache(), tab) == status
        assert lib.spcache_attend(h, cache(), 0, tab, p, 1, 4, 1, 0.1, 0.0, None, 0, t, t) == status
        assert lib.spcache_fork(h, cache(), tab, p, 1, p, p, p, p, 1, p, None) == status
        assert lib.spcache_compact(h, cache(), tab, p, None) == status
    assert append(cache(), table(), lens=None) == INVALID_ARG
    assert append(cache(), table(), new=None) == INVALID_ARG
    assert append(cache(), table(), layer=1) == INVALID_ARG
    assert append(cache(), table(), tokens=-1) == INVALID_ARG
    assert append(cache(), table(), dtype=5) == INVALID_ARG
    assert append(cache(), table(), k=at.TensorStruct(1032, 512, 64)) == UNSUPPORTED
    attend = lambda q_len=1, heads=4, scale=0.1, window=0, o=t: lib.spcache_attend(h, cache(), 0, table(), p, q_len, heads, 1, scale, 0.0, None, window, t, o)  # noqa: E731
    assert attend(q_len=-1) == attend(heads=3) == attend(scale=0.0) == attend(window=-1) == attend(o=at.TensorStruct(None, 0, 0)) == INVALID_ARG
    assert attend(q_len=1 << 30) == attend(q_len=1 << 20) == UNSUPPORTED
    fork = lambda n=1, parent=p, ptr=p, pages=p, room=1, refs=p: lib.spcache_fork(h, cache(), table(), p, n, parent, p, ptr, pages, room, refs, None)  # noqa: E731
    assert fork(n=-1) == fork(parent=None) == fork(ptr=None) == fork(pages=None) == fork(room=-1) == fork(refs=None) == INVALID_ARG
    assert lib.spcache_compact(h, cache(), table(), None, None) == INVALID_ARG
    assert lib.spcache_copy(h, cache(), -1, p, p) == lib.spcache_copy(h, cache(), 1, None, p) == INVALID_ARG
    assert lib.spcache_copy(None, cache(), 1, p, p) == INVALID_ARG
