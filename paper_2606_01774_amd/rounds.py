"""The softmax half of a serving round: attention of a block of nodes over a paged cache,
verification of drafted tokens, and the pages of the cache.

Bindings of the C entry points of the same names (``include/bdgdn.h``), re-exported by the
package.  Like the others they only marshal arguments.  A pool of keys or values is a tensor
``[n_pages, page, h_kv, d]`` with contiguous heads' elements and otherwise any strides of a
multiple of 16 bytes; the tables of a cache are a ``CacheTables``.
"""
from __future__ import annotations

import ctypes
import functools
import math
from typing import NamedTuple

import torch

from . import _DT, _F32, _I32, _check, _dev, _p, _stream, load_library

BDGDN_MASK_FULL = 0
BDGDN_MASK_CAUSAL = 1
BDGDN_MASK_BITS = 2
BDGDN_CACHE_DONE = 0
BDGDN_CACHE_NO_PAGES = 1
BDGDN_CACHE_NO_ROOM = 2
BDGDN_CACHE_BAD_SLOT = 3
BDGDN_CACHE_BAD_KEEP = 4

_MASKS = {"full": BDGDN_MASK_FULL, "causal": BDGDN_MASK_CAUSAL}


class CacheDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page", "n_slots", "max_pages", "h_kv", "d", "dtype")] + [
        (n, ctypes.c_int64) for n in ("page_stride", "token_stride", "head_stride")]


class AttnDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_req", "nodes", "h_q", "h_kv", "d")] + [("scale", ctypes.c_float)] + [
        (n, ctypes.c_int32) for n in ("dtype", "out_dtype", "mask")] + [
        (n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride")]


class VerifyDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_req", "nodes", "vocab", "dtype")] + [
        (n, ctypes.c_int64) for n in ("target_req_stride", "target_row_stride", "draft_req_stride", "draft_row_stride",
                                      "noise_stride")]


class _Tables(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("page_table", "seq_len", "refcount", "free_bits")]


class CacheTables(NamedTuple):
    """The tables of a cache on the device, all int32: page_table [n_slots, max_pages], seq_len
    [n_slots], refcount [n_pages], free_bits [(n_pages + 31) // 32]."""
    page_table: torch.Tensor
    seq_len: torch.Tensor
    refcount: torch.Tensor
    free_bits: torch.Tensor


def make_cache_tables(n_slots, max_pages, n_pages, device="cuda") -> CacheTables:
    """The tables of an empty cache."""
    bits = [-1] * (n_pages // 32)
    if n_pages % 32:
        last = (1 << n_pages % 32) - 1
        bits.append(last - (1 << 32) if last >= 1 << 31 else last)
    return CacheTables(torch.full((n_slots, max_pages), -1, dtype=_I32, device=device),
                       torch.zeros(n_slots, dtype=_I32, device=device),
                       torch.zeros(n_pages, dtype=_I32, device=device),
                       torch.tensor(bits, dtype=_I32).to(device))


def bind(lib):
    """Argument types of the entry points of this module."""
    P, I, L, Z, R = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.POINTER
    for name, res, args in (
            ("bdgdn_tree_attn_workspace", Z, [R(AttnDesc), R(CacheDesc)]),
            ("bdgdn_tree_attn", ctypes.c_int, [R(AttnDesc), R(CacheDesc)] + [P] * 13 + [Z, P]),
            ("bdgdn_tree_mask", ctypes.c_int, [I, I, P, P, P, P]),
            ("bdgdn_verify_workspace", Z, [R(VerifyDesc)]),
            ("bdgdn_verify", ctypes.c_int, [R(VerifyDesc)] + [P] * 13 + [Z, P]),
            ("bdgdn_cache_workspace", Z, [R(CacheDesc), I, I]),
            ("bdgdn_cache_append", ctypes.c_int, [R(CacheDesc), R(_Tables), P, P, I, I, I, L] + [P] * 5 + [Z, P]),
            ("bdgdn_cache_fork", ctypes.c_int, [R(CacheDesc), R(_Tables), I, P, P, P, P]),
            ("bdgdn_cache_compact", ctypes.c_int, [R(CacheDesc), R(_Tables), P, I, I, I] + [P] * 5 + [Z, P]),
            ("bdgdn_cache_truncate", ctypes.c_int, [R(CacheDesc), R(_Tables), I, P, P, P])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args


# ------------------------------------------------------------------ marshalling
@functools.lru_cache(maxsize=512)
def _cache_desc(n_slots, max_pages, shape, strides, dtype):
    n_pages, page, h_kv, d = shape
    return CacheDesc(n_pages, page, n_slots, max_pages, h_kv, d, _DT.get(dtype, -1), *strides)


@functools.lru_cache(maxsize=512)
def _table_desc(n_slots, max_pages, n_pages, page):
    return CacheDesc(n_pages, page, n_slots, max_pages)


def _pool(t, name):
    """A pool's geometry, (shape, strides without the last), after its checks."""
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or t.dim() != 4:
        raise ValueError(f"{name} must be a device tensor [n_pages, page, h_kv, d]")
    strides = t.stride()
    if strides[3] != 1:
        raise ValueError(f"the elements of a head of {name} must be contiguous")
    return tuple(t.shape), strides[:3]


def _rows(t, name, dtype):
    """The stride between the nodes' rows of [R, N, h, d], which may be a part of longer rows."""
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or t.dim() != 4:
        raise ValueError(f"{name} must be a device tensor [R, N, heads, d]")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.is_contiguous():
        return 0
    R, N, h, d = t.shape
    s = t.stride()
    row = s[1] if N > 1 else s[0]
    if s[3] != 1 or (h > 1 and s[2] != d) or (R > 1 and s[0] != N * row):
        raise ValueError(f"{name} must have contiguous heads and one stride between its rows")
    return row if R * N > 1 else 0


def _tables(tables):
    table, seq_len, refcount, bits = tables
    out = _Tables(_p(table, "page_table", _I32), _p(seq_len, "seq_len", _I32), _p(refcount, "refcount", _I32),
                  _p(bits, "free_bits", _I32))
    if table.dim() != 2 or seq_len.numel() != table.shape[0] or bits.numel() != (refcount.numel() + 31) // 32:
        raise ValueError("the cache's tables do not fit each other")
    return out


def _vector(t, name, n, dtype=_I32):
    if t is not None and t.numel() != n:
        raise ValueError(f"{name} must have {n} elements")
    return _p(t, name, dtype)


def _workspace(workspace, need, device):
    """(workspace, its address, its size), allocated where none is given."""
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, _p(workspace, "workspace"), workspace.numel() * workspace.element_size()


# ------------------------------------------------------------------ attention
@functools.lru_cache(maxsize=512)
def _attn_plan(R, N, h_q, h_kv, d, scale, dtype, out_dtype, mask, strides, cache):
    desc = AttnDesc(R, N, h_q, h_kv, d, scale, _DT.get(dtype, -1), _DT.get(out_dtype, -1), mask, *strides)
    c = _cache_desc(*cache)
    return desc, c, int(load_library().bdgdn_tree_attn_workspace(ctypes.byref(desc), ctypes.byref(c)))


def bdgdn_tree_attn_workspace(desc: AttnDesc, cache: CacheDesc) -> int:
    return int(load_library().bdgdn_tree_attn_workspace(ctypes.byref(desc), ctypes.byref(cache)))


def bdgdn_tree_attn(q, k, v, k_pages, v_pages, page_table, seq_len, *, mask="full", count=None, slot=None,
                    scale=None, o=None, lse=None, want_lse=False, out_dtype=None, workspace=None, stream=None):
    """Attention of N <= 64 new nodes per request (q [R, N, h_q, d], k, v [R, N, h_kv, d]) over
    the cached tokens of slot[r] and over the nodes that the mask lets them see: "full",
    "causal", or int64 words [R, N] (bit j of word n: node n sees node j; bdgdn_tree_mask makes
    a tree's).  scale is 1/sqrt(d) unless given, out_dtype q's.  Returns (o, lse or None)."""
    lib = load_library()
    dt = q.dtype
    strides = (_rows(q, "q", dt), _rows(k, "k", dt), _rows(v, "v", dt))
    (R, N, h_q, d), h_kv = q.shape, k.shape[2]
    if k.shape != (R, N, h_kv, d) or v.shape != k.shape:
        raise ValueError("k and v must be [R, N, h_kv, d] for q's R, N and d")
    shape, pool_strides = _pool(k_pages, "k_pages")
    if _pool(v_pages, "v_pages") != (shape, pool_strides) or k_pages.dtype != dt or v_pages.dtype != dt:
        raise ValueError("k_pages and v_pages must be alike and of q's type")
    if page_table.dim() != 2 or seq_len.numel() != page_table.shape[0]:
        raise ValueError("page_table must be [n_slots, max_pages] and seq_len [n_slots]")
    kind = BDGDN_MASK_BITS if isinstance(mask, torch.Tensor) else _MASKS.get(mask)
    if kind is None:
        raise ValueError(f"unknown mask {mask!r}")
    bits = _vector(mask, "mask", R * N, torch.int64) if kind == BDGDN_MASK_BITS else None
    out_dtype = o.dtype if o is not None else dt if out_dtype is None else out_dtype
    desc, cache, need = _attn_plan(R, N, h_q, h_kv, d, 1.0 / math.sqrt(d) if scale is None else float(scale), dt,
                                   out_dtype, kind, strides, (*page_table.shape, shape, pool_strides, dt))
    if o is None:
        o = torch.empty(R, N, h_q, d, dtype=out_dtype, device=q.device)
    elif o.shape != q.shape:
        raise ValueError("o must have q's shape")
    if lse is None and want_lse:
        lse = torch.empty(R, N, h_q, dtype=_F32, device=q.device)
    workspace, pw, size = _workspace(workspace, need, q.device)
    st = lib.bdgdn_tree_attn(desc, cache, q.data_ptr(), k.data_ptr(), v.data_ptr(), k_pages.data_ptr(),
                             v_pages.data_ptr(), _p(page_table, "page_table", _I32), _p(seq_len, "seq_len", _I32),
                             _vector(slot, "slot", R), _vector(count, "count", R), bits, _p(o, "o", out_dtype),
                             _vector(lse, "lse", R * N * h_q, _F32), pw, size, _stream(stream))
    _check(st, "bdgdn_tree_attn")
    return o, lse


def bdgdn_tree_mask(parent, *, mask=None, depth=None, want_depth=False, stream=None):
    """Mask words (int64 [R, N]) of drafted trees from parent [R, N] int32: a node sees itself
    and its ancestors.  With want_depth (or depth given) returns (mask, depth)."""
    lib = load_library()
    if parent.dim() != 2:
        raise ValueError("parent must be [R, N]")
    pp = _p(parent, "parent", _I32)
    R, N = parent.shape
    if mask is None:
        mask = torch.empty(R, N, dtype=torch.int64, device=parent.device)
    if depth is None and want_depth:
        depth = torch.empty_like(parent)
    st = lib.bdgdn_tree_mask(R, N, pp, _vector(mask, "mask", R * N, torch.int64), _vector(depth, "depth", R * N),
                             _stream(stream))
    _check(st, "bdgdn_tree_mask")
    return mask if depth is None else (mask, depth)


# ------------------------------------------------------------------ verification
@functools.lru_cache(maxsize=512)
def _verify_plan(R, N, V, dtype, strides):
    desc = VerifyDesc(R, N, V, _DT.get(dtype, -1), *strides)
    return desc, int(load_library().bdgdn_verify_workspace(ctypes.byref(desc)))


def bdgdn_verify_workspace(desc: VerifyDesc) -> int:
    return int(load_library().bdgdn_verify_workspace(ctypes.byref(desc)))


def _logits(t, name):
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be a device tensor [R, N, V] with contiguous rows")
    return t.stride()[:2]


def bdgdn_verify(target, token, u, noise, *, draft=None, parent=None, count=None, temperature=None, n_accept=None,
                 n_path=None, want_n_path=False, path=None, next_token=None, workspace=None, stream=None):
    """Verification of drafted tokens: target [R, N, V] logits after each node, token [R, N]
    int32, u [R, N] fp32 in [0, 1), noise [R, V] fp32 exponential; draft [R, N or N - 1, V]
    logits of the target's type that a node's children were drawn from (None: certain
    proposals), parent [R, N] int32 (None: chains), temperature [R] fp32 (None: 1; <= 0 greedy).
    Returns (n_accept [R], path [R, N], next_token [R]), with want_n_path (or n_path given)
    (n_accept, path, next_token, n_path), all int32."""
    lib = load_library()
    t_strides = _logits(target, "target")
    R, N, V = target.shape
    d_strides = (0, 0)
    if draft is not None:
        d_strides = _logits(draft, "draft")
        if draft.dtype != target.dtype or draft.shape[0] != R or draft.shape[1] not in (N, N - 1) or draft.shape[2] != V:
            raise ValueError("draft must be [R, N or N - 1, V] of the target's type")
        if draft.shape[1] == 0:
            draft = None
    if noise.dim() != 2 or noise.shape != (R, V) or noise.dtype != _F32 or noise.device.type != "cuda" or (
            V > 1 and noise.stride(1) != 1):
        raise ValueError("noise must be a device tensor [R, V] of fp32 with contiguous rows")
    desc, need = _verify_plan(R, N, V, target.dtype, (*t_strides, *d_strides, noise.stride(0)))
    dev = target.device
    if n_accept is None:
        n_accept = torch.empty(R, dtype=_I32, device=dev)
    if path is None:
        path = torch.empty(R, N, dtype=_I32, device=dev)
    if next_token is None:
        next_token = torch.empty(R, dtype=_I32, device=dev)
    if n_path is None and want_n_path:
        n_path = torch.empty(R, dtype=_I32, device=dev)
    workspace, pw, size = _workspace(workspace, need, dev)
    st = lib.bdgdn_verify(desc, target.data_ptr(), None if draft is None else draft.data_ptr(),
                          _vector(token, "token", R * N), _vector(parent, "parent", R * N), _vector(count, "count", R),
                          _vector(temperature, "temperature", R, _F32), _vector(u, "u", R * N, _F32), noise.data_ptr(),
                          _vector(n_accept, "n_accept", R), _vector(n_path, "n_path", R), _vector(path, "path", R * N),
                          _vector(next_token, "next_token", R), pw, size, _stream(stream))
    _check(st, "bdgdn_verify")
    return (n_accept, path, next_token) if n_path is None else (n_accept, path, next_token, n_path)


# ------------------------------------------------------------------ the cache's pages
def bdgdn_cache_workspace(cache: CacheDesc, num_req: int, rows_max: int) -> int:
    return int(load_library().bdgdn_cache_workspace(ctypes.byref(cache), num_req, rows_max))


@functools.lru_cache(maxsize=512)
def _cache_bytes(cache, num_req, rows_max):
    return bdgdn_cache_workspace(_cache_desc(*cache), num_req, rows_max)


def _pool_list(tables, pools):
    """(descriptor's key, host array of the pools' addresses) of alike pools."""
    if not pools:
        raise ValueError("a cache has at least one pool")
    first = _pool(pools[0], "pools[0]")
    dt = pools[0].dtype
    for i, t in enumerate(pools):
        if _pool(t, f"pools[{i}]") != first or t.dtype != dt:
            raise ValueError("the pools of a cache must be alike")
    if first[0][0] != tables.refcount.numel():
        raise ValueError("the pools must have as many pages as refcount")
    return ((*tables.page_table.shape, *first, dt),
            (ctypes.c_void_p * len(pools))(*[t.data_ptr() for t in pools]))


def bdgdn_cache_append(tables, pools, rows, slot, count, *, path=None, status=None, workspace=None, stream=None):
    """Rows rows[i][r, path[r, j]], j < count[r], of every pool i behind the sequences in
    slot[r].  rows: one [R, N, h_kv, d] per pool; path [R, N] int32 or None (rows in order).
    Returns status [R] (BDGDN_CACHE_DONE or why a sequence was left as it was)."""
    lib = load_library()
    key, ptrs = _pool_list(tables, pools)
    if len(rows) != len(pools):
        raise ValueError("rows must hold one tensor per pool")
    stride, shape = _rows(rows[0], "rows[0]", pools[0].dtype), rows[0].shape
    for i, t in enumerate(rows):
        if _rows(t, f"rows[{i}]", pools[0].dtype) != stride or t.shape != shape:
            raise ValueError("the rows of all pools must be alike")
    R, N = shape[:2]
    if shape[2:] != pools[0].shape[2:]:
        raise ValueError("rows must be [R, N, h_kv, d] for the pools' h_kv and d")
    if status is None:
        status = torch.empty(R, dtype=_I32, device=slot.device)
    workspace, pw, size = _workspace(workspace, _cache_bytes(key, R, N), slot.device)
    st = lib.bdgdn_cache_append(_cache_desc(*key), _tables(tables), ptrs,
                                (ctypes.c_void_p * len(rows))(*[t.data_ptr() for t in rows]), len(pools), R, N, stride,
                                _vector(slot, "slot", R), _vector(path, "path", R * N), _vector(count, "count", R),
                                _vector(status, "status", R), pw, size, _stream(stream))
    _check(st, "bdgdn_cache_append")
    return status


def bdgdn_cache_fork(tables, src, dst, *, page, status=None, stream=None):
    """Slots dst[i] (empty) share the sequences of src[i].  Returns status."""
    lib = load_library()
    n = src.numel()
    if status is None:
        status = torch.empty(n, dtype=_I32, device=src.device)
    st = lib.bdgdn_cache_fork(_table_desc(*tables.page_table.shape, tables.refcount.numel(), int(page)), _tables(tables), n,
                              _p(src, "src", _I32), _vector(dst, "dst", n), _vector(status, "status", n), _stream(stream))
    _check(st, "bdgdn_cache_fork")
    return status


def bdgdn_cache_compact(tables, pools, slot, keep, count, *, status=None, workspace=None, stream=None):
    """Keeps positions keep[r, :count[r]] (rising) of the sequences in slot[r].  Returns status."""
    lib = load_library()
    key, ptrs = _pool_list(tables, pools)
    if keep.dim() != 2:
        raise ValueError("keep must be [R, M]")
    R, M = keep.shape
    if status is None:
        status = torch.empty(R, dtype=_I32, device=slot.device)
    workspace, pw, size = _workspace(workspace, _cache_bytes(key, R, M), slot.device)
    st = lib.bdgdn_cache_compact(_cache_desc(*key), _tables(tables), ptrs, len(pools), R, M, _vector(slot, "slot", R),
                                 _p(keep, "keep", _I32), _vector(count, "count", R), _vector(status, "status", R), pw,
                                 size, _stream(stream))
    _check(st, "bdgdn_cache_compact")
    return status


def bdgdn_cache_truncate(tables, slot, length=None, *, page, stream=None):
    """Shortens the sequences in slot[r] to length[r] tokens (None: frees the slots)."""
    lib = load_library()
    n = slot.numel()
    st = lib.bdgdn_cache_truncate(_table_desc(*tables.page_table.shape, tables.refcount.numel(), int(page)), _tables(tables),
                                  n, _p(slot, "slot", _I32), _vector(length, "length", n), _stream(stream))
    _check(st, "bdgdn_cache_truncate")
