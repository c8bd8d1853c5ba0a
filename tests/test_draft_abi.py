"""Host-side checks of include/spdraft.h that need no GPU: symbols, struct layouts, and refusals that come before the first HIP call."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "spdraft.h")
INVALID_ARG, DIM_MISMATCH, UNSUPPORTED = -1, -2, -4


@pytest.fixture(scope="module")
def dr():
    from paper_2404_04541_amd import binding, drafts
    if not os.path.exists(binding.LIB_PATH):
        from paper_2404_04541_amd.build import build_library
        build_library()
    return drafts


@pytest.fixture()
def h(dr):
    lib, handle = dr._lib(), C.c_void_p()
    assert lib.spgemm_create(C.byref(handle), None, None) == 0
    yield handle
    lib.spgemm_destroy(handle)


def test_every_declared_symbol_is_exported(dr):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(spdraft_[a-z_]+)\s*\(", text)))
    assert names == sorted(dr.EXPORTED)
    for n in names:
        assert hasattr(dr._lib(), n), n


def test_constants_and_layouts_match_the_header(dr):
    text = open(HEADER).read()
    assert int(re.search(r"#define SPDRAFT_MOST (\d+)", text).group(1)) == dr.MOST
    assert int(re.search(r"#define SPDRAFT_F32 (\d+)", text).group(1)) == dr.F32
    assert C.sizeof(dr.TreesStruct) == 5 * 8 and C.sizeof(dr.RowsStruct) == 2 * 8


def trees(dr, **kw):
    return dr.TreesStruct(*(dict(rows=2, tokens=10, ptr=64, parent=64, most=8) | kw).values())


BAD_TREES = [(dict(rows=-1), INVALID_ARG), (dict(tokens=-1), INVALID_ARG), (dict(tokens=1 << 24), UNSUPPORTED), (dict(rows=1 << 24), UNSUPPORTED), (dict(most=0), INVALID_ARG),
             (dict(most=257), UNSUPPORTED), (dict(ptr=None), INVALID_ARG)]


def test_trees_are_refused(dr, h):
    lib = dr._lib()
    for kw, status in BAD_TREES:
        t = trees(dr, **kw)
        assert lib.spdraft_symbolic(h, C.byref(t), C.c_void_p(256), 1 << 30, None) == status, kw
        assert lib.spdraft_plan_bytes(C.byref(t)) == 0 and lib.spgemm_last_error(h)
    t = trees(dr)
    need = lib.spdraft_plan_bytes(C.byref(t))
    assert lib.spdraft_plan_bytes(C.byref(trees(dr, most=256, tokens=1000))) > need >= 10 * 24
    assert lib.spdraft_symbolic(h, None, C.c_void_p(256), need, None) == INVALID_ARG
    assert lib.spdraft_symbolic(h, C.byref(t), None, need, None) == INVALID_ARG
    assert lib.spdraft_symbolic(h, C.byref(t), C.c_void_p(256), need - 1, None) == INVALID_ARG
    assert lib.spdraft_symbolic(h, C.byref(t), C.c_void_p(128), need, None) == INVALID_ARG
    assert lib.spdraft_symbolic(h, C.byref(trees(dr, parent=None)), C.c_void_p(256), need, None) == INVALID_ARG
    assert lib.spdraft_symbolic(None, C.byref(t), C.c_void_p(256), need, None) == INVALID_ARG


@pytest.fixture()
def parts(dr):
    from paper_2404_04541_amd import attention as at
    from paper_2404_04541_amd import binding as sg
    cache = lambda **kw: C.byref(at.CacheStruct(*(dict(layers=1, pages=4, kv_heads=2, head_dim=64, k=64, v=64, k_scale=64, v_scale=64) | kw).values()))  # noqa: E731
    table = lambda rows=2, cols=4, nnz=1, ptr=64, col=64: C.byref(sg.CsrStruct(rows, cols, nnz, ptr, col, None, 0))  # noqa: E731
    return cache, table, at.TensorStruct


def test_attend_is_refused(dr, h, parts):
    cache, table, tensor = parts
    lib, p, good = dr._lib(), C.c_void_p(256), tensor(1024, 512, 64)

    def attend(c=None, tab=None, lens=p, layer=0, t=None, plan=p, heads=4, dtype=1, scale=0.1, cap=0.0, window=0, q=good, o=good):
        return lib.spdraft_attend(h, c or cache(), layer, tab or table(), lens, C.byref(t or trees(dr)), plan, heads, dtype, scale, cap, None, window, q, o)

    for kw, status in BAD_TREES:
        assert attend(t=trees(dr, **kw)) == status
    for kw, status in ((dict(c=cache(layers=0)), INVALID_ARG), (dict(c=cache(head_dim=100)), UNSUPPORTED), (dict(tab=table(ptr=None)), INVALID_ARG), (dict(tab=table(cols=5)), DIM_MISMATCH),
                       (dict(tab=table(rows=3)), DIM_MISMATCH), (dict(lens=None), INVALID_ARG), (dict(layer=1), INVALID_ARG), (dict(plan=None), INVALID_ARG), (dict(heads=3), INVALID_ARG),
                       (dict(dtype=2), INVALID_ARG), (dict(scale=0.0), INVALID_ARG), (dict(cap=-1.0), INVALID_ARG), (dict(window=-1), INVALID_ARG),
                       (dict(q=tensor(None, 512, 64)), INVALID_ARG), (dict(o=tensor(1032, 512, 64)), UNSUPPORTED), (dict(t=trees(dr, tokens=(1 << 24) - 1)), UNSUPPORTED)):
        assert attend(**kw) == status, kw
    assert lib.spdraft_attend(h, None, 0, table(), p, C.byref(trees(dr)), p, 4, 1, 0.1, 0.0, None, 0, good, good) == INVALID_ARG
    assert lib.spdraft_attend(None, cache(), 0, table(), p, C.byref(trees(dr)), p, 4, 1, 0.1, 0.0, None, 0, good, good) == INVALID_ARG


def test_verify_is_refused(dr, h):
    lib, p = dr._lib(), C.c_void_p(256)

    def verify(t=None, plan=p, vocab=100, dtype=2, target=(64, 100), draft=(64, 100), ids=p, u=p, path=p, kept=p, following=p):
        return lib.spdraft_verify(h, C.byref(t or trees(dr)), plan, vocab, dtype, dr.RowsStruct(*target), dr.RowsStruct(*draft), ids, u, path, kept, following)

    for kw, status in BAD_TREES:
        assert verify(t=trees(dr, **kw)) == status
    for kw, status in ((dict(plan=None), INVALID_ARG), (dict(vocab=0), INVALID_ARG), (dict(vocab=(1 << 24) + 1), UNSUPPORTED), (dict(dtype=3), INVALID_ARG),
                       (dict(target=(None, 100)), INVALID_ARG), (dict(target=(64, -1)), INVALID_ARG), (dict(draft=(64, -1)), INVALID_ARG), (dict(target=(66, 100)), INVALID_ARG),
                       (dict(dtype=1, draft=(65, 100)), INVALID_ARG), (dict(ids=None), INVALID_ARG), (dict(u=None), INVALID_ARG), (dict(path=None), INVALID_ARG),
                       (dict(kept=None), INVALID_ARG), (dict(following=None), INVALID_ARG), (dict(t=trees(dr, tokens=(1 << 22))), UNSUPPORTED)):
        assert verify(**kw) == status, kw
    assert verify(t=trees(dr, rows=0)) == 0


def test_keep_is_refused(dr, h, parts):
    cache, table, _ = parts
    lib, p, other = dr._lib(), C.c_void_p(256), C.c_void_p(512)

    def keep(c=None, tab=None, lens=p, t=None, path=p, kept=p, out=other):
        return lib.spdraft_keep(h, c or cache(), tab or table(), lens, C.byref(t or trees(dr)), path, kept, out)

    for kw, status in BAD_TREES:
        assert keep(t=trees(dr, **kw)) == status
    for kw, status in ((dict(c=cache(k=None)), INVALID_ARG), (dict(tab=table(rows=1)), DIM_MISMATCH), (dict(tab=table(cols=3)), DIM_MISMATCH), (dict(lens=None), INVALID_ARG),
                       (dict(path=None), INVALID_ARG), (dict(kept=None), INVALID_ARG), (dict(out=None), INVALID_ARG), (dict(out=p), INVALID_ARG), (dict(c=cache(layers=40000)), UNSUPPORTED),
                       (dict(t=trees(dr, rows=1 << 23), tab=table(rows=1 << 23)), UNSUPPORTED)):
        assert keep(**kw) == status, kw
    assert keep(t=trees(dr, rows=0, tokens=0), tab=table(rows=0)) == 0


def test_keep_into_its_inputs_is_refused(dr, h, parts):
    """Every workgroup of a sequence reads its length, its path and how much of it stays, and one writes the new length: that may lie in none of them."""
    cache, table, _ = parts
    lib, at = dr._lib(), dict(lens=1024, path=2048, kept=4096)

    def keep(out):
        return lib.spdraft_keep(h, cache(), table(), C.c_void_p(at["lens"]), C.byref(trees(dr)), C.c_void_p(at["path"]), C.c_void_p(at["kept"]), C.c_void_p(out))

    for name, size in (("lens", 8), ("path", 40), ("kept", 8)):
        for out in range(at[name] - 4, at[name] + size, 4):
            assert keep(out) == INVALID_ARG, (name, out)


def test_read_is_refused(dr, h, parts):
    cache, table, tensor = parts
    lib, p, good = dr._lib(), C.c_void_p(256), tensor(1024, 512, 64)

    def read(c=None, tab=None, lens=p, layer=0, ptr=p, tokens=4, dtype=1, k=good, v=good):
        return lib.spcache_read(h, c or cache(), layer, tab or table(), lens, ptr, tokens, dtype, k, v)

    for kw, status in ((dict(c=cache(head_dim=100)), UNSUPPORTED), (dict(tab=table(cols=5)), DIM_MISMATCH), (dict(lens=None), INVALID_ARG), (dict(layer=-1), INVALID_ARG),
                       (dict(ptr=None), INVALID_ARG), (dict(tokens=-1), INVALID_ARG), (dict(tokens=1 << 30), UNSUPPORTED), (dict(dtype=2), INVALID_ARG),
                       (dict(k=tensor(None, 512, 64)), INVALID_ARG), (dict(v=tensor(1024, 516, 64)), UNSUPPORTED), (dict(tab=table(rows=1 << 24)), UNSUPPORTED)):
        assert read(**kw) == status, kw
    assert read(tokens=0) == 0
