"""What a hybrid layer does around its mixers, and with the logits before verification: rotary
positions, norms with gate, scale and residual, projections in 8-bit integers, penalties, biases
and grammar masks.

Bindings of the C entry points of the same names (``include/bdgdn.h``), re-exported by the
package.  Like the others they only marshal arguments.  Rows have contiguous elements and otherwise
any strides, so tensors may be parts of one projection's rows; outputs that are not given are
contiguous.  All tensors of a call, and ``stream``, are on the current device.
"""
from __future__ import annotations

import ctypes
import functools
import math

import torch

from . import _DT, _F32, _I32, _Tensor, _check, _p, _raw_stream, _stream, load_library
from .rounds import _empty, _scratch, _vector

BDGDN_ROPE_HALF = 0
BDGDN_ROPE_PAIRS = 1
BDGDN_ROPE_PLAIN = 0
BDGDN_ROPE_LINEAR = 1
BDGDN_ROPE_NTK = 2
BDGDN_ROPE_PARTS = 3
BDGDN_ACT_SIGMOID = 2
BDGDN_HISTORY_PROMPT = 1 << 30

_LAYOUTS = {"half": BDGDN_ROPE_HALF, "pairs": BDGDN_ROPE_PAIRS}
_SCALINGS = {None: BDGDN_ROPE_PLAIN, "none": BDGDN_ROPE_PLAIN, "linear": BDGDN_ROPE_LINEAR, "ntk": BDGDN_ROPE_NTK,
             "parts": BDGDN_ROPE_PARTS}
_ACTS = {None: 0, "none": 0, "silu": 1, "sigmoid": BDGDN_ACT_SIGMOID}
_I64, _I8 = torch.int64, torch.int8
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _fields(ctype, *names):
    return [(n, ctype) for n in names]


class RopeFreq(ctypes.Structure):
    _fields_ = _fields(ctypes.c_int32, "rot", "scaling") + _fields(ctypes.c_double, "base", "factor", "original", "slow", "fast")


class Heads(ctypes.Structure):
    _fields_ = _fields(ctypes.c_int64, "req", "row", "head")


class RopeDesc(ctypes.Structure):
    _fields_ = (_fields(ctypes.c_int32, "num_req", "nodes", "h_q", "h_k", "d", "rot", "layout", "dtype", "inverse", "n_slots")
                + _fields(ctypes.c_float, "scale") + _fields(Heads, "q", "k", "q_out", "k_out"))


class Rows(ctypes.Structure):
    _fields_ = _fields(ctypes.c_int64, "outer", "inner")


class NormDesc(ctypes.Structure):
    _fields_ = (_fields(ctypes.c_int32, "outer", "inner", "d", "x_dtype", "r_dtype", "dtype", "post", "pre", "act")
                + _fields(ctypes.c_float, "scale", "eps")
                + _fields(Rows, "x", "z", "r", "r_out", "y", "dx", "dz", "dr", "dr_out", "dy"))


class LogitsDesc(ctypes.Structure):
    _fields_ = (_fields(ctypes.c_int32, "num_req", "nodes", "vocab", "dtype", "out_dtype", "n_slots", "n_bias")
                + _fields(ctypes.c_int64, "req_stride", "row_stride", "out_req_stride", "out_row_stride",
                          "history_stride", "allow_req_stride", "allow_row_stride"))


class QuantDesc(ctypes.Structure):
    _fields_ = _fields(ctypes.c_int32, "rows", "cols", "width", "dtype") + _fields(ctypes.c_int64, "x_stride", "q_stride")


class QuantMatmulDesc(ctypes.Structure):
    _fields_ = _fields(ctypes.c_int32, "m", "n", "k", "out_dtype") + _fields(ctypes.c_int64, "a_stride", "w_stride", "out_stride")


def bind(lib):
    """Argument types of the entry points of this module."""
    P, I, L, Z, R = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.POINTER
    for name, res, args in (
            ("bdgdn_rope_freqs", ctypes.c_int, [R(RopeFreq), P]),
            ("bdgdn_rope", ctypes.c_int, [R(RopeDesc)] + [P] * 10),
            ("bdgdn_norm_fwd", ctypes.c_int, [R(NormDesc)] + [P] * 9),
            ("bdgdn_norm_bwd_workspace", Z, [R(NormDesc)]),
            ("bdgdn_norm_bwd", ctypes.c_int, [R(NormDesc)] + [P] * 15 + [Z, P]),
            ("bdgdn_logits", ctypes.c_int, [R(LogitsDesc)] + [P] * 14),
            ("bdgdn_history_add", ctypes.c_int, [I, I, I, I, L] + [P] * 5 + [I, P]),
            ("bdgdn_quant_rows", ctypes.c_int, [R(QuantDesc)] + [P] * 4),
            ("bdgdn_quant_matmul_workspace", Z, [R(QuantMatmulDesc)]),
            ("bdgdn_quant_matmul", ctypes.c_int, [R(QuantMatmulDesc)] + [P] * 7 + [Z, P])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args


# ------------------------------------------------------------------ marshalling
def _here(stream, names, *tensors, need=1):
    """The tensors are on the device that the call runs on, the first `need` of them given; its raw stream.  (A
    small call costs what its marshalling does: what is usual is one comparison a tensor.)"""
    at = _current_device()
    if stream is not None and stream.device_index != at:
        raise ValueError(f"the stream is on device {stream.device_index}, the call runs on device {at}")
    for i in range(need):
        if tensors[i] is None:
            raise ValueError(f"{names.split()[i]} must be a device tensor")
    for t in tensors:
        if t is not None and not (isinstance(t, _Tensor) and t.is_cuda and t.get_device() == at):
            name = names.split()[[i for i, u in enumerate(tensors) if u is t][0]]
            if not isinstance(t, _Tensor) or not t.is_cuda:
                raise ValueError(f"{name} must be a device tensor")
            raise ValueError(f"{name} is on device {t.get_device()}, the call runs on device {at}")
    return _stream(stream) if stream is not None or _raw_stream is None else _raw_stream(at)


def _current_device():
    return _get_device() if torch.cuda.is_initialized() else torch.cuda.current_device()


def _fresh(like, dtype, stream):
    """A contiguous tensor of another's shape."""
    if stream is None and like.dtype is dtype:   # (half the time of torch.empty)
        return torch.empty_like(like, memory_format=torch.contiguous_format)
    return _empty(like.shape, dtype, like.device, stream)


def _like(t, name, shape, dtype):
    if t is not None and (t.shape != shape or t.dtype is not dtype):
        raise ValueError(f"{name} must be {tuple(shape)} of {dtype}, got {tuple(t.shape)} of {t.dtype}")


def _at(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------ rotary positions
def make_rope_turns(rot, base=10000.0, *, scaling=None, factor=1.0, original=None, slow=1.0, fast=32.0, device="cuda"):
    """(turns, scale) for bdgdn_rope: the turns a position of rot / 2 pairs, as 64-bit fractions
    (int64 [rot / 2]), and what the rotated elements are multiplied with.  scaling: None, "linear"
    (positions divided by factor), "ntk" (the base grows with factor) or "parts" (only pairs that turn
    less than fast times over `original` positions are slowed down, those of fewer than slow turns by
    the whole factor; scale is 0.1 log(factor) + 1, else 1)."""
    if scaling not in _SCALINGS:
        raise ValueError(f"unknown scaling {scaling!r}")
    if scaling == "parts" and original is None:
        raise ValueError("scaling by parts needs the original number of positions")
    desc = RopeFreq(int(rot), _SCALINGS[scaling], base, factor, 0.0 if original is None else original, slow, fast)
    turns = torch.empty(max(int(rot) // 2, 1), dtype=_I64)
    _check(load_library().bdgdn_rope_freqs(ctypes.byref(desc), turns.data_ptr()), "bdgdn_rope_freqs")
    return turns.to(device), 0.1 * math.log(factor) + 1 if scaling == "parts" and factor > 1 else 1.0


@functools.lru_cache(maxsize=512)
def _rope_plan(q, sq, k, sk, qo, sqo, ko, sko, dtype, rot, layout, inverse, scale, n_slots):
    if len(q) != 4 or (k is not None and (len(k) != 4 or k[:2] != q[:2] or k[3] != q[3])):
        raise ValueError("q must be [R, N, h_q, d] and k [R, N, h_k, d] for q's R, N and d")
    if layout is None:
        raise ValueError("unknown layout")
    (R, N, h_q, d), h_k = q, 0 if k is None else k[2]
    strides = []
    for shape, s, heads in ((q, sq, h_q), (k, sk, h_k), (qo, sqo, h_q), (ko, sko, h_k)):
        if shape is None:   # not there, or a contiguous output to come
            s = (N * heads * d, heads * d, d, 1)
        elif d > 1 and s[3] != 1:
            raise ValueError("the elements of a head must be contiguous")
        strides.append(Heads(*s[:3]))
    return RopeDesc(R, N, h_q, h_k, d, rot, layout, _DT.get(dtype, -1), int(inverse), n_slots, scale, *strides)


def bdgdn_rope(q, turns, k=None, *, pos=None, seq_len=None, slot=None, count=None, layout="half", scale=1.0, inverse=False,
               q_out=None, k_out=None, stream=None):
    """Rotary positions: the first 2 * len(turns) elements of every head of q [R, N, h_q, d] and k
    [R, N, h_k, d] (or None) turn by position seq_len[slot[r]] + pos[r, n] (pos [R, N] int32, None: n;
    seq_len [n_slots] int32, None: 0).  turns and scale: make_rope_turns.  layout "half" or "pairs";
    inverse turns back (the gradient).  q_out and k_out may be q and k; rows n >= count[r] are left
    out.  Returns q_out, or (q_out, k_out)."""
    lib = load_library()
    here = _here(stream, "q turns k pos seq_len slot count q_out k_out",
                 q, turns, k, pos, seq_len, slot, count, q_out, k_out, need=2)
    dt, shape = q.dtype, q.shape
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    if k is not None and k.dtype is not dt:
        raise ValueError(f"k must be of q's type, {dt}")
    _like(q_out, "q_out", shape, dt)
    _like(k_out, "k_out", None if k is None else k.shape, dt)
    desc = _rope_plan(shape, q.stride(), *((None, None) if k is None else (k.shape, k.stride())),
                      *((None, None) if q_out is None else (shape, q_out.stride())),
                      *((None, None) if k_out is None else (k.shape, k_out.stride())), dt, 2 * turns.numel(),
                      _LAYOUTS.get(layout), bool(inverse), float(scale), 0 if seq_len is None else seq_len.numel())
    R, N = shape[:2]
    if q_out is None:
        q_out = _fresh(q, dt, stream)
    if k_out is None and k is not None:
        k_out = _fresh(k, dt, stream)
    if k is not None and k.shape[2] == 0:
        k, pk, pko = None, None, None
    else:
        pk, pko = _at(k), _at(k_out)
    st = lib.bdgdn_rope(desc, q.data_ptr(), pk, _p(turns, "turns", _I64), _vector(pos, "pos", R * N),
                        _p(seq_len, "seq_len", _I32), _vector(slot, "slot", R), _vector(count, "count", R),
                        q_out.data_ptr(), pko, here)
    _check(st, "bdgdn_rope")
    return q_out if k_out is None else (q_out, k_out)


# ------------------------------------------------------------------ norms
def _row_strides(shape, s, name):
    if s is None:
        return Rows(shape[-1] if len(shape) == 2 else shape[1] * shape[2], shape[-1])
    if shape[-1] > 1 and s[-1] != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    return Rows(s[0], s[1] if len(shape) == 3 else shape[-1])


@functools.lru_cache(maxsize=512)
def _norm_plan(shape, strides, types, post, pre, act, scale, eps):
    """The descriptor, and its bytes of workspace for the backward; strides in the order of Rows fields, None for
    contiguous or absent tensors."""
    if len(shape) not in (2, 3):
        raise ValueError("x must be [rows, d] or [tokens, heads, d]")
    if act is None:
        raise ValueError("unknown act")
    names = ("x", "z", "r", "r_out", "y", "dx", "dz", "dr", "dr_out", "dy")
    desc = NormDesc(shape[0], 1 if len(shape) == 2 else shape[1], shape[-1], *(_DT.get(t, -1) for t in types), int(post),
                    int(pre), act, scale, eps, *(_row_strides(shape, s, n) for s, n in zip(strides, names)))
    return desc, int(load_library().bdgdn_norm_bwd_workspace(ctypes.byref(desc)))


def _strides(*ts):
    return tuple(None if t is None else t.stride() for t in ts)


def _weights(d, **ws):
    return [_vector(w, name, d, _F32) for name, w in ws.items()]


def bdgdn_norm_fwd(x, *, z=None, r=None, w_post=None, w_pre=None, layer_scale=None, post=False, pre=False, act="silu",
                   scale=1.0, eps=1e-6, r_out=None, y=None, out_dtype=None, stream=None):
    """The norms around a mixer with its gate, scale and residual: n = x / rms(x) * w_post (post), u =
    n act(z), r' = r + scale layer_scale u, y = r' / rms(r') * w_pre (pre).  x, z, r are [rows, d]
    or [tokens, heads, d]; weights [d] fp32 or None for ones; act "silu", "sigmoid" or "none".  y has
    out_dtype (z's type, or else x's).  Returns (y, r'), None for r' where there is neither r nor r_out."""
    lib = load_library()
    here = _here(stream, "x z r w_post w_pre layer_scale r_out y",
                 x, z, r, w_post, w_pre, layer_scale, r_out, y)
    shape = x.shape
    dt = z.dtype if z is not None else y.dtype if y is not None else x.dtype if out_dtype is None else out_dtype
    if out_dtype is not None and out_dtype is not dt:
        raise ValueError(f"y has the type of z, {dt}")
    rt = r.dtype if r is not None else r_out.dtype if r_out is not None else x.dtype
    for t, name, kind in ((z, "z", dt), (r, "r", rt), (r_out, "r_out", rt), (y, "y", dt)):
        _like(t, name, shape, kind)
    desc, _ = _norm_plan(shape, _strides(x, z, r, r_out, y, None, None, None, None, None), (x.dtype, rt, dt), bool(post),
                         bool(pre), _ACTS.get(act), float(scale), float(eps))
    if y is None:
        y = _fresh(x if x.dtype is dt else z if z is not None else x, dt, stream)
    if r_out is None and r is not None:
        r_out = _fresh(r, rt, stream)
    st = lib.bdgdn_norm_fwd(desc, x.data_ptr(), _at(z), _at(r),
                            *_weights(shape[-1], w_post=w_post, w_pre=w_pre, layer_scale=layer_scale), _at(r_out),
                            y.data_ptr(), here)
    _check(st, "bdgdn_norm_fwd")
    return y, r_out


def bdgdn_norm_bwd_workspace(desc: NormDesc) -> int:
    return int(load_library().bdgdn_norm_bwd_workspace(ctypes.byref(desc)))


def bdgdn_norm_bwd(x, dy, *, z=None, r_out=None, dr_out=None, w_post=None, w_pre=None, layer_scale=None, post=False,
                   pre=False, act="silu", scale=1.0, eps=1e-6, dx=None, dz=None, dr=None, dw_post=None, dw_pre=None,
                   dlayer_scale=None, workspace=None, stream=None):
    """The backward of bdgdn_norm_fwd for upstream gradients dy of y and dr_out of r' (either may be
    None).  r_out is the forward's r', to be given where it took a residual.  Returns (dx, dz, dr,
    dw_post, dw_pre, dlayer_scale); dr where r_out or dr_out is given, the weights' where they are."""
    lib = load_library()
    here = _here(stream, "x dy z r_out dr_out w_post w_pre layer_scale dx dz dr dw_post dw_pre dlayer_scale workspace",
                 x, dy, z, r_out, dr_out, w_post, w_pre, layer_scale, dx, dz, dr, dw_post, dw_pre, dlayer_scale, workspace)
    shape, d = x.shape, x.shape[-1]
    rt = r_out.dtype if r_out is not None else dr_out.dtype if dr_out is not None else dr.dtype if dr is not None else x.dtype
    # (without z and dy nothing is of y's type: bf16 goes with all others)
    dt = z.dtype if z is not None else dy.dtype if dy is not None else x.dtype if x.dtype is rt else torch.bfloat16
    for t, name, kind in ((dy, "dy", dt), (z, "z", dt), (r_out, "r_out", rt), (dr_out, "dr_out", rt), (dx, "dx", x.dtype),
                          (dz, "dz", dt), (dr, "dr", rt)):
        _like(t, name, shape, kind)
    for w, g, name in ((w_post, dw_post, "w_post"), (w_pre, dw_pre, "w_pre"), (layer_scale, dlayer_scale, "layer_scale")):
        if g is not None and w is None:
            raise ValueError(f"d{name} without {name}")
    desc, need = _norm_plan(shape, _strides(x, z, None, r_out, None, dx, dz, dr, dr_out, dy), (x.dtype, rt, dt), bool(post),
                            bool(pre), _ACTS.get(act), float(scale), float(eps))
    dev = x.device
    if dx is None:
        dx = _fresh(x, x.dtype, stream)
    if dz is None and z is not None:
        dz = _fresh(z, dt, stream)
    if dr is None and (r_out is not None or dr_out is not None):
        dr = _fresh(r_out if r_out is not None else dr_out, rt, stream)
    if dw_post is None and w_post is not None and post:
        dw_post = _fresh(w_post, _F32, stream)
    if dw_pre is None and w_pre is not None and pre:
        dw_pre = _fresh(w_pre, _F32, stream)
    if dlayer_scale is None and layer_scale is not None:
        dlayer_scale = _fresh(layer_scale, _F32, stream)
    workspace, size = _scratch(workspace, need, dev, stream)
    st = lib.bdgdn_norm_bwd(desc, x.data_ptr(), _at(z), _at(r_out),
                            *_weights(d, w_post=w_post, w_pre=w_pre, layer_scale=layer_scale), _at(dy), _at(dr_out),
                            dx.data_ptr(), _at(dz), _at(dr),
                            *_weights(d, dw_post=dw_post, dw_pre=dw_pre, dlayer_scale=dlayer_scale),
                            workspace.data_ptr(), size, here)
    _check(st, "bdgdn_norm_bwd")
    return dx, dz, dr, dw_post, dw_pre, dlayer_scale


# ------------------------------------------------------------------ logits
@functools.lru_cache(maxsize=512)
def _logits_plan(shape, s, out, so, dtype, out_dtype, history, sh, allow, sa, n_bias):
    if len(shape) != 3 or (shape[2] > 1 and s[2] != 1) or (so is not None and shape[2] > 1 and so[2] != 1):
        raise ValueError("logits and out must be [R, N, V] with contiguous rows")
    R, N, V = shape
    if out is not None and out != shape:
        raise ValueError("out must have the shape of logits")
    so = (N * V, V) if so is None else so
    slots = 0
    if history is not None:
        if len(history) != 2 or history[1] != V or (V > 1 and sh[1] != 1):
            raise ValueError("history must be [n_slots, V] with contiguous rows")
        slots = history[0]
    ar = an = 0
    if allow is not None:
        words = (V + 31) // 32
        if len(allow) != 3 or allow[0] not in (1, R) or allow[1] not in (1, N) or allow[2] != words or (words > 1 and sa[2] != 1):
            raise ValueError("allow must be [R or 1, N or 1, (V + 31) // 32] with contiguous rows")
        ar, an = (0 if allow[0] == 1 else sa[0]), (0 if allow[1] == 1 else sa[1])
    return LogitsDesc(R, N, V, _DT.get(dtype, -1), _DT.get(out_dtype, -1), slots, n_bias, s[0], s[1], so[0], so[1],
                      0 if history is None else sh[0], ar, an)


def bdgdn_logits(logits, *, token=None, mask=None, count=None, history=None, slot=None, repetition=None, presence=None,
                 frequency=None, bias_token=None, bias=None, allow=None, out=None, out_dtype=None, stream=None):
    """Penalties for repeated tokens, biases and grammar masks on the logits [R, N, V] after each node.
    token [R, N] int32 and mask [R, N] int64 (bdgdn_tree_mask; None: chains) say what the block's nodes
    add to history [n_slots, V] int32 (bdgdn_history_add); repetition, presence, frequency [R] fp32;
    bias_token, bias [R, K] int32 and fp32; allow int32 words [R or 1, N or 1, (V + 31) // 32], bit
    t % 32 of word t // 32 set where token t is allowed.  out may be logits.  Returns out (out_dtype:
    that of logits)."""
    lib = load_library()
    here = _here(stream, "logits token mask count history slot repetition presence frequency bias_token bias allow out",
                 logits, token, mask, count, history, slot, repetition, presence, frequency, bias_token, bias, allow, out)
    dt, shape = logits.dtype, logits.shape
    if out is not None:
        if out_dtype is not None and out_dtype is not out.dtype:
            raise ValueError(f"out is of {out.dtype}, not {out_dtype}")
        out_dtype = out.dtype
    elif out_dtype is None:
        out_dtype = dt
    for t, name in ((history, "history"), (allow, "allow")):
        if t is not None and t.dtype is not _I32:
            raise ValueError(f"{name} must be {_I32}, got {t.dtype}")
    if (bias is None) != (bias_token is None) or (bias is not None and (bias.dim() != 2 or bias.shape != bias_token.shape
                                                                        or bias.shape[0] != shape[0])):
        raise ValueError("bias_token and bias must both be [R, K]")
    desc = _logits_plan(shape, logits.stride(), *((None, None) if out is None else (out.shape, out.stride())), dt, out_dtype,
                        *((None, None) if history is None else (history.shape, history.stride())),
                        *((None, None) if allow is None else (allow.shape, allow.stride())),
                        0 if bias is None else bias.shape[1])
    R, N, _ = shape
    if out is None:
        out = _fresh(logits, out_dtype, stream)
    if bias is not None and bias.numel() == 0:
        bias = bias_token = None
    n = 0 if bias is None else bias.numel()
    st = lib.bdgdn_logits(desc, logits.data_ptr(), _at(history), _vector(slot, "slot", R), _vector(token, "token", R * N),
                          _vector(mask, "mask", R * N, _I64), _vector(count, "count", R),
                          _vector(repetition, "repetition", R, _F32), _vector(presence, "presence", R, _F32),
                          _vector(frequency, "frequency", R, _F32), _vector(bias_token, "bias_token", n),
                          _vector(bias, "bias", n, _F32), _at(allow), out.data_ptr(), here)
    _check(st, "bdgdn_logits")
    return out


def bdgdn_history_add(history, token, *, slot=None, path=None, count=None, prompt=False, stream=None):
    """Adds token[r, path[r, j]], j < count[r], to row slot[r] of history [n_slots, V] int32 (path None:
    in order; count None: all): one more occurrence each or, with prompt, the mark of a prompt's token
    (BDGDN_HISTORY_PROMPT)."""
    lib = load_library()
    here = _here(stream, "history token slot path count",
                 history, token, slot, path, count, need=2)
    if history.dim() != 2 or history.dtype is not _I32 or (history.shape[1] > 1 and history.stride(1) != 1):
        raise ValueError("history must be [n_slots, V] int32 with contiguous rows")
    if token.dim() != 2:
        raise ValueError("token must be [R, N]")
    R, N = token.shape
    st = lib.bdgdn_history_add(R, N, history.shape[1], history.shape[0], history.stride(0), history.data_ptr(),
                               _vector(slot, "slot", R), _p(token, "token", _I32), _vector(path, "path", R * N),
                               _vector(count, "count", R), int(bool(prompt)), here)
    _check(st, "bdgdn_history_add")


# ------------------------------------------------------------------ 8-bit products
@functools.lru_cache(maxsize=512)
def _quant_plan(shape, s, dtype, width, q_stride):
    if len(shape) != 2 or (shape[1] > 1 and s[1] != 1):
        raise ValueError("x must be [rows, columns] with contiguous rows")
    return QuantDesc(shape[0], shape[1], width, _DT.get(dtype, -1), s[0], q_stride)


def bdgdn_quant_rows(x, *, q=None, scale=None, stream=None):
    """8-bit integers and a scale for each row of x [rows, columns]: scale = max |x| (1 / 127), q =
    x / scale rounded to the nearest integer, in fp32.  q is int8 [rows, columns filled up with zeros to a multiple of
    128].  Returns (q, scale)."""
    lib = load_library()
    here = _here(stream, "x q scale",
                 x, q, scale)
    if x.dim() != 2:
        raise ValueError("x must be [rows, columns]")
    rows, width = x.shape[0], (x.shape[1] + 127) // 128 * 128
    if q is None:
        q = _empty((rows, width), _I8, x.device, stream)
    else:
        _like(q, "q", (rows, width), _I8)
        if q.stride(1) != 1:
            raise ValueError("the rows of q must be contiguous")
    if scale is None:
        scale = _empty(rows, _F32, x.device, stream)
    desc = _quant_plan(x.shape, x.stride(), x.dtype, width, q.stride(0))
    st = lib.bdgdn_quant_rows(desc, x.data_ptr(), q.data_ptr(), _vector(scale, "scale", rows, _F32), here)
    _check(st, "bdgdn_quant_rows")
    return q, scale


@functools.lru_cache(maxsize=512)
def _matmul_plan(a, sa, w, sw, out_dtype, so):
    if len(a) != 2 or len(w) != 2 or a[1] != w[1] or sa[1] != 1 or sw[1] != 1:
        raise ValueError("a and w must be [m, k] and [n, k] with contiguous rows")
    desc = QuantMatmulDesc(a[0], w[0], a[1], _DT.get(out_dtype, -1), sa[0], sw[0], w[0] if so is None else so[0])
    return desc, bdgdn_quant_matmul_workspace(desc)


def bdgdn_quant_matmul_workspace(desc: QuantMatmulDesc) -> int:
    return int(load_library().bdgdn_quant_matmul_workspace(ctypes.byref(desc)))


def bdgdn_quant_matmul(a, a_scale, w, w_scale, *, bias=None, out=None, out_dtype=torch.bfloat16, workspace=None, stream=None):
    """The product [m, n] of rows of 8-bit integers a [m, k] and w [n, k] (bdgdn_quant_rows; k a multiple
    of 128) with scales a_scale [m] for each token and w_scale [n] for each channel: a_scale[i]
    w_scale[j] sum_k a[i, k] w[j, k] + bias[j], exact in its integer sums."""
    lib = load_library()
    here = _here(stream, "a a_scale w w_scale bias out workspace",
                 a, a_scale, w, w_scale, bias, out, workspace, need=4)
    if a.dtype is not _I8 or w.dtype is not _I8:
        raise ValueError(f"a and w must be {_I8}")
    if out is not None:
        out_dtype = out.dtype
    desc, need = _matmul_plan(a.shape, a.stride(), w.shape, w.stride(), out_dtype, None if out is None else out.stride())
    m, n = a.shape[0], w.shape[0]
    if out is None:
        out = _empty((m, n), out_dtype, a.device, stream)
    else:
        _like(out, "out", (m, n), out_dtype)
        if n > 1 and out.stride(1) != 1:
            raise ValueError("the rows of out must be contiguous")
    if need:
        workspace, size = _scratch(workspace, need, a.device, stream)
    else:
        size = 0
    st = lib.bdgdn_quant_matmul(desc, a.data_ptr(), _vector(a_scale, "a_scale", m, _F32), w.data_ptr(),
                                _vector(w_scale, "w_scale", n, _F32), _vector(bias, "bias", n, _F32), out.data_ptr(),
                                _at(workspace) if need else None, size, here)
    _check(st, "bdgdn_quant_matmul")
    return out
