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

from . import _DT, _F32, _I32, _Tensor, _check, _p, _stream, load_library

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


class _CacheTables(NamedTuple):
    page_table: torch.Tensor
    seq_len: torch.Tensor
    refcount: torch.Tensor
    free_bits: torch.Tensor


class CacheTables(_CacheTables):
    """The tables of a cache on the device, all int32: page_table [n_slots, max_pages], seq_len
    [n_slots], refcount [n_pages], free_bits [(n_pages + 31) // 32].  Beside these four it may know
    the tokens of a page (``page``, else None); calls with another page are then refused."""
    page = None

    def __new__(cls, page_table, seq_len, refcount, free_bits, page=None):
        if page is not None and int(page) < 1:
            raise ValueError(f"page must be a number of tokens, got {page}")
        self = super().__new__(cls, page_table, seq_len, refcount, free_bits)
        self.page = None if page is None else int(page)
        return self

    def _replace(self, **kw):
        page = kw.pop("page", self.page)
        return CacheTables(*super()._replace(**kw), page=page)


def make_cache_tables(n_slots, max_pages, n_pages, device="cuda", page=None) -> CacheTables:
    """The tables of an empty cache; page is what the calls hold its pools' pages to."""
    bits = [-1] * (n_pages // 32)
    if n_pages % 32:
        last = (1 << n_pages % 32) - 1
        bits.append(last - (1 << 32) if last >= 1 << 31 else last)
    return CacheTables(torch.full((n_slots, max_pages), -1, dtype=_I32, device=device),
                       torch.zeros(n_slots, dtype=_I32, device=device),
                       torch.zeros(n_pages, dtype=_I32, device=device),
                       torch.tensor(bits, dtype=_I32).to(device), page)


def _page_of(tables, page):
    """Tokens of a page, from what the caller or the pools say (or None) and what the tables know."""
    known = getattr(tables, "page", None)
    if page is None:
        if known is None:
            raise ValueError("page must be given for tables that do not know it")
        return known
    if known is not None and page != known:
        raise ValueError(f"these are tables of pages of {known} tokens, not of {page}")
    return int(page)


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
# A serving round makes these calls once a layer, so they cost what their marshalling does: what
# follows from shapes, strides and types alone is worked out once for each set of them, and a
# call reads its tensors' attributes and passes plain integers.
@functools.lru_cache(maxsize=512)
def _cache_desc(n_slots, max_pages, shape, strides, dtype):
    n_pages, page, h_kv, d = shape
    return CacheDesc(n_pages, page, n_slots, max_pages, h_kv, d, _DT.get(dtype, -1), *strides[:3])


@functools.lru_cache(maxsize=512)
def _table_desc(n_slots, max_pages, n_pages, page):
    return CacheDesc(n_pages, page, n_slots, max_pages)


def _check_pool(shape, strides, name):
    if len(shape) != 4:
        raise ValueError(f"{name} must be [n_pages, page, h_kv, d]")
    if strides[3] != 1:
        raise ValueError(f"the elements of a head of {name} must be contiguous")


def _row_stride(shape, strides, name):
    """Elements between the nodes' rows of [R, N, h, d], which may be a part of longer rows; 0
    for contiguous ones, which is why rows that share memory (an expanded tensor's) are refused."""
    if len(shape) != 4:
        raise ValueError(f"{name} must be [R, N, heads, d]")
    R, N, h, d = shape
    if R * N == 0:
        return 0
    row = strides[1] if N > 1 else strides[0] if R > 1 else h * d
    if (d > 1 and strides[3] != 1) or (h > 1 and strides[2] != d) or (R > 1 and N > 1 and strides[0] != N * row) or row < h * d:
        raise ValueError(f"{name} must have contiguous heads and one stride between its rows, which share no memory")
    return 0 if row == h * d else row


def _device(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")


def _alike(ts, name):
    """The addresses of device tensors of one shape, stride and type."""
    first = ts[0]
    _device(first, f"{name}[0]")
    shape, strides, dt = first.shape, first.stride(), first.dtype
    for i, t in enumerate(ts):
        if not (type(t) is _Tensor and t.is_cuda and t.dtype is dt and t.shape == shape and t.stride() == strides):
            _device(t, f"{name}[{i}]")
            if t.dtype is not dt or t.shape != shape or t.stride() != strides:
                raise ValueError(f"{name}[{i}] must be like {name}[0]")
    return (ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts])


def _tables(tables):
    table, seq_len, refcount, bits = tables
    out = _Tables(_p(table, "page_table", _I32), _p(seq_len, "seq_len", _I32), _p(refcount, "refcount", _I32),
                  _p(bits, "free_bits", _I32))
    if table.dim() != 2 or seq_len.numel() != table.shape[0] or bits.numel() != (refcount.numel() + 31) // 32:
        raise ValueError("the cache's tables do not fit each other")
    return out


def _vector(t, name, n, dtype=_I32):
    if t is None:
        return None
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} elements")
    return _p(t, name, dtype)


def _empty(shape, dtype, device, stream):
    """Memory of the stream that the call runs on: another stream's could be handed out again, or
    still be in use there, while this one's kernels work on it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _scratch(workspace, need, device, stream):
    """(workspace, its size), allocated where none is given."""
    if workspace is None:
        return _empty(need, torch.uint8, device, stream), need
    _p(workspace, "workspace")
    return workspace, workspace.numel() * workspace.element_size()


# ------------------------------------------------------------------ attention
@functools.lru_cache(maxsize=512)
def _attn_plan(q, sq, k, sk, v, sv, kp, skp, vp, svp, table, slots, scale, dtype, out_dtype, mask):
    """Everything that follows from shapes, strides and types: both descriptors and the bytes of
    workspace."""
    rows = [_row_stride(*x) for x in ((q, sq, "q"), (k, sk, "k"), (v, sv, "v"))]
    (R, N, h_q, d), h_kv = q, k[2]
    if tuple(k) != (R, N, h_kv, d) or v != k:
        raise ValueError("k and v must be [R, N, h_kv, d] for q's R, N and d")
    _check_pool(kp, skp, "k_pages")
    if vp != kp or svp != skp:
        raise ValueError("k_pages and v_pages must be alike")
    if len(table) != 2 or slots != table[0]:
        raise ValueError("page_table must be [n_slots, max_pages] and seq_len [n_slots]")
    if mask is None:
        raise ValueError("unknown mask")
    desc = AttnDesc(R, N, h_q, h_kv, d, 1.0 / math.sqrt(d) if scale is None else scale, _DT.get(dtype, -1),
                    _DT.get(out_dtype, -1), mask, *rows)
    cache = _cache_desc(table[0], table[1], tuple(kp), skp, dtype)
    return desc, cache, int(load_library().bdgdn_tree_attn_workspace(ctypes.byref(desc), ctypes.byref(cache)))


def bdgdn_tree_attn_workspace(desc: AttnDesc, cache: CacheDesc) -> int:
    return int(load_library().bdgdn_tree_attn_workspace(ctypes.byref(desc), ctypes.byref(cache)))


def bdgdn_tree_attn(q, k, v, k_pages, v_pages, page_table, seq_len, *, mask="full", count=None, slot=None,
                    scale=None, o=None, lse=None, want_lse=False, out_dtype=None, workspace=None, stream=None):
    """Attention of N <= 64 new nodes per request (q [R, N, h_q, d], k, v [R, N, h_kv, d]) over
    the cached tokens of slot[r] and over the nodes that the mask lets them see: "full",
    "causal", or int64 words [R, N] (bit j of word n: node n sees node j; bdgdn_tree_mask makes
    a tree's).  scale is 1/sqrt(d) unless given, out_dtype q's.  Returns (o, lse or None)."""
    lib = load_library()
    for t, name in ((q, "q"), (k, "k"), (v, "v"), (k_pages, "k_pages"), (v_pages, "v_pages")):
        if not (type(t) is _Tensor and t.is_cuda):
            _device(t, name)
    dt = q.dtype
    if k.dtype is not dt or v.dtype is not dt or k_pages.dtype is not dt or v_pages.dtype is not dt:
        raise ValueError(f"k, v, k_pages and v_pages must be of q's type, {dt}")
    shape = q.shape
    words = isinstance(mask, _Tensor)
    out_dtype = o.dtype if o is not None else dt if out_dtype is None else out_dtype
    desc, cache, need = _attn_plan(shape, q.stride(), k.shape, k.stride(), v.shape, v.stride(), k_pages.shape,
                                   k_pages.stride(), v_pages.shape, v_pages.stride(), page_table.shape, seq_len.numel(),
                                   None if scale is None else float(scale), dt, out_dtype,
                                   BDGDN_MASK_BITS if words else _MASKS.get(mask))
    R, N, h_q, _ = shape
    device = q.device
    if o is None:
        o = _empty(shape, out_dtype, device, stream)
        po = o.data_ptr()
    else:
        if o.shape != shape:
            raise ValueError("o must have q's shape")
        po = _p(o, "o", out_dtype)
    if lse is None and want_lse:
        lse = _empty((R, N, h_q), _F32, device, stream)
    workspace, size = _scratch(workspace, need, device, stream)
    st = lib.bdgdn_tree_attn(desc, cache, q.data_ptr(), k.data_ptr(), v.data_ptr(), k_pages.data_ptr(),
                             v_pages.data_ptr(), _p(page_table, "page_table", _I32), _p(seq_len, "seq_len", _I32),
                             _vector(slot, "slot", R), _vector(count, "count", R),
                             _vector(mask, "mask", R * N, torch.int64) if words else None, po,
                             _vector(lse, "lse", R * N * h_q, _F32), workspace.data_ptr(), size, _stream(stream))
    _check(st, "bdgdn_tree_attn")
    return o, lse


def bdgdn_tree_mask(parent, *, mask=None, depth=None, want_depth=False, stream=None):
    """Mask words (int64 [R, N]) of drafted trees from parent [R, N] int32: a node sees itself
    and its ancestors.  With want_depth (or depth given) returns (mask, depth)."""
    lib = load_library()
    pp = _p(parent, "parent", _I32)
    if parent.dim() != 2:
        raise ValueError("parent must be [R, N]")
    R, N = parent.shape
    if mask is None:
        mask = _empty((R, N), torch.int64, parent.device, stream)
    if depth is None and want_depth:
        depth = _empty(parent.shape, _I32, parent.device, stream)
    st = lib.bdgdn_tree_mask(R, N, pp, _vector(mask, "mask", R * N, torch.int64), _vector(depth, "depth", R * N),
                             _stream(stream))
    _check(st, "bdgdn_tree_mask")
    return mask if depth is None else (mask, depth)


# ------------------------------------------------------------------ verification
@functools.lru_cache(maxsize=512)
def _verify_plan(target, st, draft, sd, noise, sn, dtype):
    for shape, strides, name in ((target, st, "target"), (draft, sd, "draft")):
        if shape is not None and (len(shape) != 3 or (shape[2] > 1 and strides[2] != 1)):
            raise ValueError(f"{name} must be [R, N, V] with contiguous rows")
    R, N, V = target
    if draft is not None and (draft[0] != R or draft[1] not in (N, N - 1) or draft[2] != V):
        raise ValueError("draft must be [R, N or N - 1, V] for target's R, N and V")
    if tuple(noise) != (R, V) or (V > 1 and sn[1] != 1):
        raise ValueError("noise must be [R, V] with contiguous rows")
    desc = VerifyDesc(R, N, V, _DT.get(dtype, -1), st[0], st[1], *((0, 0) if draft is None else sd[:2]), sn[0])
    return desc, int(load_library().bdgdn_verify_workspace(ctypes.byref(desc)))


def bdgdn_verify_workspace(desc: VerifyDesc) -> int:
    return int(load_library().bdgdn_verify_workspace(ctypes.byref(desc)))


def bdgdn_verify(target, token, u, noise, *, draft=None, parent=None, count=None, temperature=None, n_accept=None,
                 n_path=None, want_n_path=False, path=None, next_token=None, workspace=None, stream=None):
    """Verification of drafted tokens: target [R, N, V] logits after each node, token [R, N]
    int32, u [R, N] fp32 in [0, 1), noise [R, V] fp32 exponential; draft [R, N or N - 1, V]
    logits of the target's type that a node's children were drawn from (None: certain
    proposals), parent [R, N] int32 (None: chains), temperature [R] fp32 (None: 1; <= 0 greedy).
    Returns (n_accept [R], path [R, N], next_token [R]), with want_n_path (or n_path given)
    (n_accept, path, next_token, n_path), all int32."""
    lib = load_library()
    _device(target, "target")
    _device(noise, "noise")
    dt = target.dtype
    if noise.dtype is not _F32:
        raise ValueError(f"noise must be {_F32}, got {noise.dtype}")
    if draft is not None:
        _device(draft, "draft")
        if draft.dtype is not dt:
            raise ValueError(f"draft must be of target's type, {dt}")
    desc, need = _verify_plan(target.shape, target.stride(), None if draft is None else draft.shape,
                              None if draft is None else draft.stride(), noise.shape, noise.stride(), dt)
    R, N, V = target.shape
    if draft is not None and draft.shape[1] == 0:
        draft = None
    dev = target.device
    if n_accept is None:
        n_accept = _empty(R, _I32, dev, stream)
    if path is None:
        path = _empty((R, N), _I32, dev, stream)
    if next_token is None:
        next_token = _empty(R, _I32, dev, stream)
    if n_path is None and want_n_path:
        n_path = _empty(R, _I32, dev, stream)
    workspace, size = _scratch(workspace, need, dev, stream)
    st = lib.bdgdn_verify(desc, target.data_ptr(), None if draft is None else draft.data_ptr(),
                          _vector(token, "token", R * N), _vector(parent, "parent", R * N), _vector(count, "count", R),
                          _vector(temperature, "temperature", R, _F32), _vector(u, "u", R * N, _F32), noise.data_ptr(),
                          _vector(n_accept, "n_accept", R), _vector(n_path, "n_path", R), _vector(path, "path", R * N),
                          _vector(next_token, "next_token", R), workspace.data_ptr(), size, _stream(stream))
    _check(st, "bdgdn_verify")
    return (n_accept, path, next_token) if n_path is None else (n_accept, path, next_token, n_path)


# ------------------------------------------------------------------ the cache's pages
def bdgdn_cache_workspace(cache: CacheDesc, num_req: int, rows_max: int) -> int:
    return int(load_library().bdgdn_cache_workspace(ctypes.byref(cache), num_req, rows_max))


@functools.lru_cache(maxsize=512)
def _pools_plan(table, n_pages, shape, strides, dtype, R, M, rows, row_strides):
    """(descriptor, bytes of workspace, stride between rows) of calls that move M rows at most
    for each of R requests; rows are the new ones' shape (append)."""
    _check_pool(shape, strides, "pools[0]")
    if shape[0] != n_pages:
        raise ValueError("the pools must have as many pages as refcount")
    if rows is not None and tuple(rows[2:]) != tuple(shape[2:]):
        raise ValueError("rows must be [R, N, h_kv, d] for the pools' h_kv and d")
    stride = 0 if rows is None else _row_stride(rows, row_strides, "rows[0]")
    desc = _cache_desc(table[0], table[1], tuple(shape), strides, dtype)
    return desc, bdgdn_cache_workspace(desc, R, M), stride


def bdgdn_cache_append(tables, pools, rows, slot, count, *, path=None, status=None, workspace=None, stream=None):
    """Rows rows[i][r, path[r, j]], j < count[r], of every pool i behind the sequences in
    slot[r].  rows: one [R, N, h_kv, d] per pool; path [R, N] int32 or None (rows in order).
    Returns status [R] (BDGDN_CACHE_DONE or why a sequence was left as it was)."""
    lib = load_library()
    n = len(pools)
    if n == 0 or len(rows) != n:
        raise ValueError("a cache has at least one pool, and rows one tensor per pool")
    pool_ptrs, row_ptrs, p0, r0 = _alike(pools, "pools"), _alike(rows, "rows"), pools[0], rows[0]
    if r0.dtype is not p0.dtype or r0.dim() != 4:
        raise ValueError("rows must be [R, N, h_kv, d] of the pools' type")
    R, N = r0.shape[:2]
    desc, need, stride = _pools_plan(tables[0].shape, tables[2].numel(), p0.shape, p0.stride(), p0.dtype, R, N, r0.shape,
                                     r0.stride())
    _page_of(tables, p0.shape[1])
    device = p0.device
    if status is None:
        status = _empty(R, _I32, device, stream)
    workspace, size = _scratch(workspace, need, device, stream)
    st = lib.bdgdn_cache_append(desc, _tables(tables), pool_ptrs, row_ptrs, n, R, N, stride, _vector(slot, "slot", R),
                                _vector(path, "path", R * N), _vector(count, "count", R), _vector(status, "status", R),
                                workspace.data_ptr(), size, _stream(stream))
    _check(st, "bdgdn_cache_append")
    return status


def bdgdn_cache_fork(tables, src, dst, *, page=None, status=None, stream=None):
    """Slots dst[i] (empty) share the sequences of src[i].  page: tokens of a page, for tables that do
    not know it.  Returns status."""
    lib = load_library()
    page = _page_of(tables, page)
    n = src.numel()
    if status is None:
        status = _empty(n, _I32, src.device, stream)
    st = lib.bdgdn_cache_fork(_table_desc(*tables.page_table.shape, tables.refcount.numel(), page), _tables(tables), n,
                              _p(src, "src", _I32), _vector(dst, "dst", n), _vector(status, "status", n), _stream(stream))
    _check(st, "bdgdn_cache_fork")
    return status


def bdgdn_cache_compact(tables, pools, slot, keep, count, *, status=None, workspace=None, stream=None):
    """Keeps positions keep[r, :count[r]] (rising) of the sequences in slot[r].  Returns status."""
    lib = load_library()
    if len(pools) == 0:
        raise ValueError("a cache has at least one pool")
    ptrs, p0 = _alike(pools, "pools"), pools[0]
    pk = _p(keep, "keep", _I32)
    if keep.dim() != 2:
        raise ValueError("keep must be [R, M]")
    R, M = keep.shape
    desc, need, _ = _pools_plan(tables[0].shape, tables[2].numel(), p0.shape, p0.stride(), p0.dtype, R, M, None, None)
    _page_of(tables, p0.shape[1])
    if status is None:
        status = _empty(R, _I32, p0.device, stream)
    workspace, size = _scratch(workspace, need, p0.device, stream)
    st = lib.bdgdn_cache_compact(desc, _tables(tables), ptrs, len(pools), R, M, _vector(slot, "slot", R), pk,
                                 _vector(count, "count", R), _vector(status, "status", R), workspace.data_ptr(), size,
                                 _stream(stream))
    _check(st, "bdgdn_cache_compact")
    return status


def bdgdn_cache_truncate(tables, slot, length=None, *, page=None, stream=None):
    """Shortens the sequences in slot[r] to length[r] tokens (None: frees the slots).  page as for
    bdgdn_cache_fork."""
    lib = load_library()
    page = _page_of(tables, page)
    n = slot.numel()
    st = lib.bdgdn_cache_truncate(_table_desc(*tables.page_table.shape, tables.refcount.numel(), page), _tables(tables),
                                  n, _p(slot, "slot", _I32), _vector(length, "length", n), _stream(stream))
    _check(st, "bdgdn_cache_truncate")
