"""Thin Python binding of the C ABI in include/spdraft.h (argument marshalling only): trees of drafted tokens over the paged cache of `attention`.

A step of serving: `symbolic` once; `attention.append` and `attend` in every layer; `verify`; `keep`.  Tensors of a tree's nodes are packed, [tokens, ...], sequence after sequence.
Results come in fresh tensors, allocated on the handle's stream where it has one of its own; where another stream is current, ordering the two is the caller's.  Like everything in
`binding`, nothing here computes: without the built library these calls raise.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

import torch

from . import attention as at
from . import binding as sg

MOST = 256
F32 = 2

EXPORTED = ("spdraft_plan_bytes", "spdraft_symbolic", "spdraft_attend", "spdraft_verify", "spdraft_keep")


class TreesStruct(C.Structure):
    _fields_ = [("rows", C.c_int64), ("tokens", C.c_int64), ("ptr", C.c_void_p), ("parent", C.c_void_p), ("most", C.c_int32)]


class RowsStruct(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64)]


_ready = None


def _lib():
    global _ready
    lib = at._lib()
    if _ready is lib:
        return lib
    P, V, I, T = C.POINTER, C.c_void_p, C.c_int64, at.TensorStruct
    lib.spdraft_plan_bytes.argtypes = [P(TreesStruct)]
    lib.spdraft_symbolic.argtypes = [V, P(TreesStruct), V, C.c_size_t, P(C.c_int32)]
    lib.spdraft_attend.argtypes = [V, P(at.CacheStruct), I, P(sg.CsrStruct), V, P(TreesStruct), V, C.c_int32, C.c_int32, C.c_float, C.c_float, V, I, T, T]
    lib.spdraft_verify.argtypes = [V, P(TreesStruct), V, I, C.c_int32, RowsStruct, RowsStruct, V, V, V, V, V]
    lib.spdraft_keep.argtypes = [V, P(at.CacheStruct), P(sg.CsrStruct), V, P(TreesStruct), V, V, V]
    for name in EXPORTED:
        getattr(lib, name).restype = C.c_size_t if name == "spdraft_plan_bytes" else C.c_int
    _ready = lib
    return lib


class Trees:
    """The structure of a batch's trees in device memory (spdraft_symbolic).  ptr stays the trees' for their life."""

    def __init__(self, struct: TreesStruct, ptr: torch.Tensor, memory: torch.Tensor):
        self.rows, self.tokens, self.most = int(struct.rows), int(struct.tokens), int(struct.most)
        self.ptr, self.memory, self._struct = ptr, memory, struct


def symbolic(handle: sg.Handle, ptr: torch.Tensor, parent: torch.Tensor, most: int, check: bool = True) -> Trees:
    """Nodes ptr[s] .. ptr[s + 1] - 1 (int64) are the tree of sequence s; node i of a tree continues its node parent[i] < i (int32), -1 the context alone.

    most: no tree has more nodes (at most 256).  check: wait, and raise where ptr, a tree's size or a parent is wrong; without it such a parent counts as -1, and the
    call only enqueues."""
    lib = _lib()
    if ptr.numel() < 1:
        raise ValueError("ptr: rows + 1 elements are wanted")
    t = TreesStruct(ptr.numel() - 1, parent.numel(), at._array(ptr, "ptr", torch.int64), _array(parent, "parent", torch.int32, ptr), int(most))
    nbytes = max(lib.spdraft_plan_bytes(C.byref(t)), 1)
    memory = at._results(handle, lambda: ptr.new_empty(nbytes, dtype=torch.uint8))
    handle._check(lib.spdraft_symbolic(handle.ptr, C.byref(t), memory.data_ptr(), nbytes, C.byref(C.c_int32(0)) if check else None))
    t.parent = None            # (what follows needs the plan only)
    return Trees(t, ptr, memory)


def _array(t: torch.Tensor, name: str, dtype: torch.dtype, like: torch.Tensor, n: Optional[int] = None) -> Optional[int]:
    if t.device != like.device:
        raise ValueError(f"{name}: on {t.device}, not on {like.device}")
    if t.dtype is not dtype or not t.is_contiguous() or (n is not None and t.numel() != n):
        return at._array(t, name, dtype, n)      # (which says what is wrong)
    return t.data_ptr() or None


def attend(handle: sg.Handle, cache: at.PagedCache, layer: int, table: at.PageTable, lens: torch.Tensor, trees: Trees, q, scale: Optional[float] = None, cap: float = 0.0,
           slopes: Optional[torch.Tensor] = None, window: int = 0):
    """-> o like q [tokens, heads, head_dim]: every node of the trees over its sequence's context, its ancestors and itself.  The nodes' keys and values are the last tokens of their
    sequence in the cache (`attention.append` with new_ptr = the trees' ptr); lens counts them."""
    lib = _lib()
    if q.dim() != 3 or q.shape[0] != trees.tokens or q.shape[2] != cache.head_dim:
        raise ValueError("q: [tokens, heads, head_dim] of the trees and the cache is wanted")
    if q.device != trees.ptr.device or cache.k.device != q.device:
        raise ValueError(f"q: on {q.device}, the trees on {trees.ptr.device}, the cache on {cache.k.device}")
    heads, d = q.shape[1], q.shape[2]
    rows = at._tensor(q, "q")
    o = at._results(handle, lambda: at._like(q))
    handle._check(lib.spdraft_attend(handle.ptr, C.byref(cache._struct), int(layer), C.byref(table.struct(cache)), _array(lens, "lens", torch.int32, q, table.rows),
                                     C.byref(trees._struct), trees.memory.data_ptr(), heads, at._dtype(q), 1.0 / math.sqrt(d) if scale is None else float(scale), float(cap),
                                     at._slopes(slopes, heads), int(window), rows, at._result(o)))
    return o


def _rows(t: Optional[torch.Tensor], name: str, trees: Trees) -> RowsStruct:
    if t is None:
        return RowsStruct(None, 0)
    if t.dim() != 2 or t.shape[0] != trees.tokens or (t.stride(1) != 1 and t.shape[1] > 1 and t.numel()):
        raise ValueError(f"{name}: [tokens, vocab] with a contiguous last dimension is wanted")
    if not t.is_cuda or t.device != trees.ptr.device:
        raise ValueError(f"{name}: on {t.device}, the trees on {trees.ptr.device}")
    return RowsStruct(t.data_ptr() or None, t.stride(0) if t.shape[0] > 1 else 0)


def verify(handle: sg.Handle, trees: Trees, ids: torch.Tensor, u: torch.Tensor, target: torch.Tensor, draft: Optional[torch.Tensor] = None):
    """-> (path int32 [tokens], kept int32 [rows], next int32 [rows]): the nodes of every tree that stay (their numbers in the tree, in order, -1 behind them), how many, and
    the token that follows.

    ids (int32) are the nodes' tokens, node 0 of a tree the one that the step before ended with; u (float32, from 0 to below 1) random numbers, one a node.  Row i of target [tokens, vocab]
    holds the target's probabilities behind node i, row i of draft those that its children were drawn from, one after the other, without replacement; without draft the
    children count as chosen, not drawn.  Both float32, bfloat16 or float16."""
    lib = _lib()
    if draft is not None and (draft.shape != target.shape or draft.dtype != target.dtype):
        raise ValueError("draft has target's shape and type")
    t, d = _rows(target, "target", trees), _rows(draft, "draft", trees)
    dtype = F32 if target.dtype == torch.float32 else at._dtype(target)
    if draft is not None and d.data is None and trees.tokens:
        raise ValueError("draft: no elements")
    ids_ptr, u_ptr = _array(ids, "ids", torch.int32, trees.ptr, trees.tokens), _array(u, "u", torch.float32, trees.ptr, trees.tokens)
    path, kept, token = at._results(handle, lambda: (ids.new_empty(trees.tokens), ids.new_empty(trees.rows), ids.new_empty(trees.rows)))
    handle._check(lib.spdraft_verify(handle.ptr, C.byref(trees._struct), trees.memory.data_ptr(), target.shape[1], dtype, t, d, ids_ptr, u_ptr, path.data_ptr() or None,
                                     kept.data_ptr() or None, token.data_ptr() or None))
    return path, kept, token


def keep(handle: sg.Handle, cache: at.PagedCache, table: at.PageTable, lens: torch.Tensor, trees: Trees, path: torch.Tensor, kept: torch.Tensor) -> torch.Tensor:
    """In all layers, token path[ptr[s] + i] of the tree of s becomes its token i, i < kept[s] -> the new lens (int32): the context's tokens and kept ones.  Pages that hold a tree's nodes
    belong to its sequence alone."""
    lib = _lib()
    at_lens = _array(lens, "lens", torch.int32, trees.ptr, table.rows)
    if cache.k.device != lens.device:
        raise ValueError(f"cache: on {cache.k.device}, not on {lens.device}")
    ways, counts = _array(path, "path", torch.int32, trees.ptr, trees.tokens), _array(kept, "kept", torch.int32, trees.ptr, trees.rows)
    out = at._results(handle, lambda: at._like(lens))
    handle._check(lib.spdraft_keep(handle.ptr, C.byref(cache._struct), C.byref(table.struct(cache)), at_lens, C.byref(trees._struct), ways, counts, out.data_ptr() or None))
    return out
