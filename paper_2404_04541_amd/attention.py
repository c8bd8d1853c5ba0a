"""Thin Python binding of the C ABI in include/spattn.h (argument marshalling only), and one autograd function over it.

Tensors of tokens are [tokens, heads, head_dim] with a contiguous last dimension; the other strides are the tensor's own.  Results come
in fresh tensors, allocated on the handle's stream where it has one of its own; where another stream is current, ordering the two is the caller's.  Like everything in `binding`, nothing here computes: without the built library these calls raise.
"""
from __future__ import annotations

import ctypes as C
import math
from dataclasses import dataclass
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as sg

F16, BF16 = 0, 1
TILE = 128
PAGE = 64

EXPORTED = ("spattn_plan_bytes", "spattn_symbolic", "spattn_forward", "spattn_backward", "spcache_append", "spcache_read", "spcache_attend",
            "spcache_fork", "spcache_compact", "spcache_copy")


class TensorStruct(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class MaskStruct(C.Structure):
    _fields_ = [("q_len", C.c_int64), ("k_len", C.c_int64), ("docs", C.c_int64), ("q_ptr", C.c_void_p), ("k_ptr", C.c_void_p),
                ("prefix", C.c_void_p), ("causal", C.c_int32), ("window", C.c_int64), ("tiles", C.POINTER(sg.CsrStruct))]


class ArgsStruct(C.Structure):
    _fields_ = [("mask", C.POINTER(MaskStruct)), ("plan_mem", C.c_void_p), ("dtype", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("scale", C.c_float), ("cap", C.c_float), ("slopes", C.c_void_p), ("q", TensorStruct), ("k", TensorStruct),
                ("v", TensorStruct)]


class CacheStruct(C.Structure):
    _fields_ = [("layers", C.c_int64), ("pages", C.c_int64), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


_ready = None


def _lib():
    global _ready
    lib = sg.load_library()
    if _ready is lib:
        return lib
    P, V, I, T = C.POINTER, C.c_void_p, C.c_int64, TensorStruct
    lib.spattn_plan_bytes.argtypes = [P(MaskStruct)]
    lib.spattn_symbolic.argtypes = [V, P(MaskStruct), V, C.c_size_t, P(C.c_int32)]
    lib.spattn_forward.argtypes = [V, P(ArgsStruct), T, V]
    lib.spattn_backward.argtypes = [V, P(ArgsStruct), T, V, T, T, T, T]
    lib.spcache_append.argtypes = [V, P(CacheStruct), I, P(sg.CsrStruct), V, V, I, C.c_int32, T, T]
    lib.spcache_read.argtypes = [V, P(CacheStruct), I, P(sg.CsrStruct), V, V, I, C.c_int32, T, T]
    lib.spcache_attend.argtypes = [V, P(CacheStruct), I, P(sg.CsrStruct), V, I, C.c_int32, C.c_int32, C.c_float, C.c_float, V, I, T, T]
    lib.spcache_fork.argtypes = [V, P(CacheStruct), P(sg.CsrStruct), V, I, V, V, V, V, I, V, P(C.c_int64)]
    lib.spcache_compact.argtypes = [V, P(CacheStruct), P(sg.CsrStruct), V, P(C.c_int64)]
    lib.spcache_copy.argtypes = [V, P(CacheStruct), I, V, V]
    for name in EXPORTED:
        getattr(lib, name).restype = C.c_size_t if name == "spattn_plan_bytes" else C.c_int
    _ready = lib
    return lib


def _dtype(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float16:
        return F16
    raise TypeError(f"attention takes float16 or bfloat16, not {t.dtype}")


def _tensor(t: torch.Tensor, name: str, tokens: Optional[int] = None, like: Optional[torch.Tensor] = None) -> TensorStruct:
    """[tokens, heads, head_dim] as the library sees it."""
    shape, strides = t.shape, t.stride()
    if len(shape) != 3 or (strides[2] != 1 and t.numel()):
        raise ValueError(f"{name}: [tokens, heads, head_dim] with a contiguous last dimension is wanted")
    if not t.is_cuda:
        raise ValueError(f"{name}: not on a GPU")
    if tokens is not None and shape[0] != tokens:
        raise ValueError(f"{name}: {shape[0]} tokens, not {tokens}")
    if like is not None and t.dtype != like.dtype:
        raise TypeError(f"{name}: {t.dtype}, not {like.dtype}")
    return TensorStruct(t.data_ptr() or None, strides[0] if shape[0] > 1 else 0, strides[1] if shape[1] > 1 else 0)


def _like(t: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of its shape (in a third of the time that naming shape, type and device takes)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _results(handle: sg.Handle, make):
    """make(), on the handle's stream, so that its memory goes to nobody else before the work is done."""
    if handle.stream is None:
        return make()
    with torch.cuda.stream(handle.stream):
        return make()


def _result(t: torch.Tensor) -> TensorStruct:
    """A fresh contiguous tensor of this module's own."""
    strides = t.stride()
    return TensorStruct(t.data_ptr() or None, strides[0], strides[1])


def _array(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, n: Optional[int] = None) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor on the GPU is wanted")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name}: {t.numel()} elements, not {n}")
    return t.data_ptr() or None


def _slopes(slopes: Optional[torch.Tensor], heads: int) -> Optional[int]:
    return _array(slopes, "slopes", torch.float32, heads)


@dataclass
class Plan:
    """The structure of a mask in device memory (spattn_symbolic); usable for any tensors of its sizes."""
    q_len: int
    k_len: int
    mask: MaskStruct
    memory: torch.Tensor


def symbolic(handle: sg.Handle, q_len: int, k_len: int, q_ptr: Optional[torch.Tensor] = None, k_ptr: Optional[torch.Tensor] = None,
             prefix: Optional[torch.Tensor] = None, causal: bool = True, window: int = 0, tiles=None, check: bool = True) -> Plan:
    """The mask of packed documents (int64 row pointers; without them one document of everything).

    tiles: the pattern, a DeviceCSR (its values are not read) or (rowptr int64, colidx int32).  check: wait, and raise where the documents or the
    pattern are out of range; without it they are cut to what exists, and the call only enqueues."""
    lib = _lib()
    docs = 0
    if (q_ptr is None) != (k_ptr is None):
        raise ValueError("q_ptr and k_ptr come together")
    if q_ptr is not None:
        docs = q_ptr.numel() - 1
        if docs < 1:
            raise ValueError("q_ptr: no documents")
    m = MaskStruct(int(q_len), int(k_len), docs, _array(q_ptr, "q_ptr", torch.int64), _array(k_ptr, "k_ptr", torch.int64, docs + 1 if docs else None),
                   _array(prefix, "prefix", torch.int64, max(docs, 1)), int(bool(causal)), int(window), None)
    held = None
    if tiles is not None:
        rowptr, colidx = (tiles.rowptr, tiles.colidx) if hasattr(tiles, "rowptr") else tiles
        held = sg.CsrStruct(rowptr.numel() - 1, getattr(tiles, "cols", -(-int(k_len) // TILE)), colidx.numel(), _array(rowptr, "pattern rowptr", torch.int64),
                            _array(colidx, "pattern colidx", torch.int32), None, 0)
        m.tiles = C.pointer(held)
    nbytes = lib.spattn_plan_bytes(C.byref(m))
    nbytes = max(nbytes, 1)
    memory = _results(handle, lambda: torch.empty(nbytes, dtype=torch.uint8, device="cuda") if q_ptr is None else q_ptr.new_empty(nbytes, dtype=torch.uint8))
    checked = C.c_int32(0)
    handle._check(lib.spattn_symbolic(handle.ptr, C.byref(m), memory.data_ptr(), nbytes, C.byref(checked) if check else None))
    m.q_ptr = m.k_ptr = None          # (what follows needs the sizes only)
    m.prefix, m.docs = None, 0
    return Plan(int(q_len), int(k_len), m, memory)


def _args(plan: Plan, q, k, v, scale, cap, slopes) -> ArgsStruct:
    heads, kv_heads, d = q.shape[1], k.shape[1], q.shape[2]
    if k.shape[2] != d or v.shape[1:] != k.shape[1:]:
        raise ValueError("q, k and v: heads and head_dim do not fit")
    return ArgsStruct(C.pointer(plan.mask), plan.memory.data_ptr(), _dtype(q), heads, kv_heads, d, 1.0 / math.sqrt(d) if scale is None else float(scale),
                      float(cap), _slopes(slopes, heads), _tensor(q, "q", plan.q_len), _tensor(k, "k", plan.k_len, q), _tensor(v, "v", plan.k_len, q))


def forward(handle: sg.Handle, plan: Plan, q, k, v, scale: Optional[float] = None, cap: float = 0.0, slopes: Optional[torch.Tensor] = None):
    """-> (o [q_len, heads, head_dim], lse float32 [heads, q_len]).  scale: 1 / sqrt(head_dim) unless given."""
    lib = _lib()
    a = _args(plan, q, k, v, scale, cap, slopes)
    o, lse = _results(handle, lambda: (_like(q), q.new_empty((q.shape[1], plan.q_len), dtype=torch.float32)))
    handle._check(lib.spattn_forward(handle.ptr, C.byref(a), _result(o), lse.data_ptr() or None))
    return o, lse


def backward(handle: sg.Handle, plan: Plan, q, k, v, o, lse, d_o, scale: Optional[float] = None, cap: float = 0.0, slopes: Optional[torch.Tensor] = None):
    """-> (dq, dk, dv): gradients of (o * d_o).sum() from forward's results."""
    lib = _lib()
    a = _args(plan, q, k, v, scale, cap, slopes)
    if o.shape != q.shape or d_o.shape != q.shape:
        raise ValueError("o and d_o have q's shape")
    dq, dk, dv = _results(handle, lambda: (_like(q), _like(k), _like(v)))
    handle._check(lib.spattn_backward(handle.ptr, C.byref(a), _tensor(o, "o", plan.q_len, q), _array(lse, "lse", torch.float32, q.shape[1] * plan.q_len),
                                      _tensor(d_o, "d_o", plan.q_len, q), _result(dq), _result(dk), _result(dv)))
    return dq, dk, dv


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, handle, plan, scale, cap, slopes):
        o, lse = forward(handle, plan, q, k, v, scale, cap, slopes)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.rest = (handle, plan, scale, cap, slopes)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, d_o):
        q, k, v, o, lse = ctx.saved_tensors
        handle, plan, scale, cap, slopes = ctx.rest
        return backward(handle, plan, q, k, v, o, lse, d_o.contiguous(), scale, cap, slopes) + (None,) * 5


def attention(handle: sg.Handle, plan: Plan, q, k, v, scale: Optional[float] = None, cap: float = 0.0, slopes: Optional[torch.Tensor] = None):
    """forward's o, differentiable once in q, k and v (not in slopes); second derivatives raise.  The handle's stream has to be the current one, forward and backward."""
    return _Attention.apply(q, k, v, handle, plan, scale, cap, slopes)


# ---- cache -----------------------------------------------------------------------------------------

class PagedCache:
    """Keys [layers, pages, kv_heads, 64, room] and values [layers, pages, kv_heads, room, 64] in 8 bits (uint8 tensors of e4m3), and their scales
    [layers, pages, kv_heads]; room is 64 for a head_dim of at most 64, else 128."""

    def __init__(self, head_dim: int, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        room = 64 if head_dim <= 64 else 128
        shape = k.shape
        if len(shape) != 5 or shape[3:] != (PAGE, room) or v.shape != (*shape[:3], room, PAGE):
            raise ValueError("cache: keys are [layers, pages, kv_heads, 64, room], values [layers, pages, kv_heads, room, 64]")
        if k_scale.shape != shape[:3] or v_scale.shape != shape[:3]:
            raise ValueError("cache: scales are [layers, pages, kv_heads]")
        self.head_dim, self.k, self.v, self.k_scale, self.v_scale = int(head_dim), k, v, k_scale, v_scale
        self.layers, self.pages, self.kv_heads = shape[:3]
        self._struct = CacheStruct(self.layers, self.pages, self.kv_heads, self.head_dim, _array(k, "cache keys", torch.uint8), _array(v, "cache values", torch.uint8),
                                   _array(k_scale, "cache scales", torch.float32), _array(v_scale, "cache scales", torch.float32))

    @classmethod
    def empty(cls, layers: int, pages: int, kv_heads: int, head_dim: int, device="cuda") -> "PagedCache":
        room = 64 if head_dim <= 64 else 128
        k = torch.zeros((layers, pages, kv_heads, PAGE, room), dtype=torch.uint8, device=device)
        v = torch.zeros((layers, pages, kv_heads, room, PAGE), dtype=torch.uint8, device=device)
        scale = [torch.ones((layers, pages, kv_heads), dtype=torch.float32, device=device) for _ in range(2)]
        return cls(head_dim, k, v, *scale)


class PageTable:
    """Row s lists the pages of sequence s: pages[rowptr[s] : rowptr[s + 1]] (int64, int32).  The tensors stay the table's for its life."""

    def __init__(self, rowptr: torch.Tensor, pages: torch.Tensor):
        self.rowptr, self.pages, self.rows = rowptr, pages, rowptr.numel() - 1
        self._struct = sg.CsrStruct(self.rows, 0, pages.numel(), _array(rowptr, "table rowptr", torch.int64), _array(pages, "table pages", torch.int32), None, 0)

    def struct(self, cache: PagedCache) -> sg.CsrStruct:
        self._struct.cols = cache.pages
        return self._struct


def append(handle: sg.Handle, cache: PagedCache, layer: int, table: PageTable, lens: torch.Tensor, new_ptr: torch.Tensor, k, v) -> None:
    """Rows new_ptr[s] .. new_ptr[s + 1] - 1 of k and v become the last tokens of sequence s, whose lens[s] (int32) counts them already."""
    lib = _lib()
    if tuple(k.shape[1:]) != (cache.kv_heads, cache.head_dim) or v.shape != k.shape:
        raise ValueError("k and v: [tokens, kv_heads, head_dim] of the cache is wanted")
    handle._check(lib.spcache_append(handle.ptr, C.byref(cache._struct), int(layer), C.byref(table.struct(cache)), _array(lens, "lens", torch.int32, table.rows),
                                     _array(new_ptr, "new_ptr", torch.int64, table.rows + 1), k.shape[0], _dtype(k), _tensor(k, "k"), _tensor(v, "v", None, k)))


def read(handle: sg.Handle, cache: PagedCache, layer: int, table: PageTable, lens: torch.Tensor, ptr: torch.Tensor, tokens: int, dtype: torch.dtype = torch.bfloat16):
    """-> (k, v) [tokens, kv_heads, head_dim]: rows ptr[s] .. ptr[s + 1] - 1 (int64) are the last tokens of sequence s, back from 8 bits: what `forward` takes, with k_ptr = ptr.

    tokens: how many rows there are, ptr's last element.  Rows of tokens that a sequence does not have, or whose page its table lacks, are zero."""
    lib = _lib()
    if tokens < 0:
        raise ValueError("tokens: a negative number")
    rows = _array(ptr, "ptr", torch.int64, table.rows + 1)
    k = _results(handle, lambda: cache.k.new_empty((int(tokens), cache.kv_heads, cache.head_dim), dtype=dtype))
    v = _results(handle, lambda: torch.empty_like(k))
    handle._check(lib.spcache_read(handle.ptr, C.byref(cache._struct), int(layer), C.byref(table.struct(cache)), _array(lens, "lens", torch.int32, table.rows), rows,
                                   int(tokens), _dtype(k), _result(k), _result(v)))
    return k, v


def attend(handle: sg.Handle, cache: PagedCache, layer: int, table: PageTable, lens: torch.Tensor, q, scale: Optional[float] = None, cap: float = 0.0,
           slopes: Optional[torch.Tensor] = None, window: int = 0):
    """-> o like q [sequences, q_len, heads, head_dim]: the last q_len tokens of every sequence over its cache."""
    lib = _lib()
    if q.dim() != 4 or q.shape[0] != table.rows or q.shape[3] != cache.head_dim:
        raise ValueError("q: [sequences, q_len, heads, head_dim] is wanted")
    n, q_len, heads, d = q.shape
    per_sequence, per_token, per_head, per_channel = q.stride()
    if (n > 1 and q_len > 1 and per_sequence != q_len * per_token) or (per_channel != 1 and q.numel()):
        raise ValueError("q: tokens of all sequences at one stride and a contiguous last dimension are wanted")
    if not q.is_cuda:
        raise ValueError("q: not on a GPU")
    o = _results(handle, lambda: _like(q))
    rows = TensorStruct(q.data_ptr() or None, (per_sequence if q_len == 1 else per_token) if n * q_len > 1 else 0, per_head if heads > 1 else 0)
    handle._check(lib.spcache_attend(handle.ptr, C.byref(cache._struct), int(layer), C.byref(table.struct(cache)), _array(lens, "lens", torch.int32, n), q_len, heads,
                                     _dtype(q), 1.0 / math.sqrt(d) if scale is None else float(scale), float(cap), _slopes(slopes, heads), int(window),
                                     rows, TensorStruct(o.data_ptr() or None, heads * d, d)))
    return o


def fork(handle: sg.Handle, cache: PagedCache, table: PageTable, lens: torch.Tensor, parent: torch.Tensor, new_lens: torch.Tensor, entries: Optional[int] = None,
         check: bool = True):
    """The table's next step: row r continues row parent[r] (-1: none) and has new_lens[r] tokens (both int32) -> (PageTable, refs int32 [pages]).

    entries: how many pages the new table has, where the caller knows (sum of ceil(new_lens / 64)).  check: wait, and raise where the step cannot be
    made; without it the call only enqueues."""
    lib = _lib()
    n = parent.numel()
    if entries is None:
        entries = int(((new_lens.clamp(min=0).to(torch.int64) + PAGE - 1) // PAGE).sum())
    rowptr, pages, refs = _results(handle, lambda: (parent.new_empty(n + 1, dtype=torch.int64), parent.new_empty(int(entries), dtype=torch.int32),
                                                    parent.new_empty(cache.pages, dtype=torch.int32)))
    nnz = C.c_int64(0)
    handle._check(lib.spcache_fork(handle.ptr, C.byref(cache._struct), C.byref(table.struct(cache)), _array(lens, "lens", torch.int32, table.rows), n,
                                   _array(parent, "parent", torch.int32), _array(new_lens, "new_lens", torch.int32, n), rowptr.data_ptr(),
                                   pages.data_ptr() if entries else None, int(entries), refs.data_ptr() if cache.pages else None, C.byref(nnz) if check else None))
    return PageTable(rowptr, pages[:nnz.value] if check else pages), refs


def compact(handle: sg.Handle, cache: PagedCache, table: PageTable, check: bool = True):
    """The pages in use to the front of the cache -> (PageTable, how many pages are in use; None without check)."""
    lib = _lib()
    pages = _results(handle, lambda: _like(table.pages))
    live = C.c_int64(0)
    handle._check(lib.spcache_compact(handle.ptr, C.byref(cache._struct), C.byref(table.struct(cache)), pages.data_ptr() if pages.numel() else None,
                                      C.byref(live) if check else None))
    return PageTable(table.rowptr, pages), int(live.value) if check else None


def copy_pages(handle: sg.Handle, cache: PagedCache, src: torch.Tensor, dst: torch.Tensor) -> None:
    """Page dst[i] becomes a copy of page src[i] (int32), in all layers; destinations distinct, and none of them a source."""
    lib = _lib()
    handle._check(lib.spcache_copy(handle.ptr, C.byref(cache._struct), src.numel(), _array(src, "src", torch.int32), _array(dst, "dst", torch.int32, src.numel())))
