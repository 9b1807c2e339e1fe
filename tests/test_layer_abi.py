"""Host-side validation of the entry points around a hybrid layer's mixers (no GPU is touched: every
call here fails validation, or has nothing to do), and the frequencies, which the host computes."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2606_01774_amd as bd
from paper_2606_01774_amd import layers

FAKE = 0x1000   # never dereferenced: validation fails first
INV, UNS, WS, OK = bd.BDGDN_ERR_INVALID_ARG, bd.BDGDN_ERR_UNSUPPORTED, bd.BDGDN_ERR_WORKSPACE, bd.BDGDN_OK


# ------------------------------------------------------------------ rotary positions
def turns(rot, scaling=bd.BDGDN_ROPE_PLAIN, base=10000.0, factor=1.0, original=0.0, slow=1.0, fast=32.0):
    out = np.zeros(max(rot, 2), dtype=np.uint64)
    st = bd.load_library().bdgdn_rope_freqs(layers.RopeFreq(rot, scaling, base, factor, original, slow, fast), out.ctypes.data)
    return st, out[:max(rot, 0) // 2]


@pytest.mark.parametrize("kw,status", [
    (dict(rot=0), INV), (dict(rot=7), INV), (dict(rot=-4), INV), (dict(rot=8, base=0.5), INV), (dict(rot=8, base=math.nan), INV),
    (dict(rot=8, base=math.inf), INV), (dict(rot=8, factor=0.0), INV), (dict(rot=8, factor=math.nan), INV), (dict(rot=8, scaling=4), INV),
    (dict(rot=8, scaling=-1), INV), (dict(rot=8, scaling=3), INV), (dict(rot=8, scaling=3, original=64, slow=2, fast=2), INV),
    (dict(rot=8, scaling=3, original=64, slow=-1), INV), (dict(rot=2, scaling=2, factor=2.0), INV),
    (dict(rot=8, scaling=3, original=64), OK), (dict(rot=2), OK), (dict(rot=8, base=1.0), OK),
])
def test_frequencies_that_are_refused(kw, status):
    assert turns(**kw)[0] == status


@pytest.mark.parametrize("rot", [2, 10, 64, 128])
@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 8.0), ("linear", 0.01), ("ntk", 4.0), ("parts", 16.0)])
def test_frequencies(rot, scaling, factor):
    """Turns a position in units of 2^-64, from the formulas in extended precision (64 bits: a
    unit or two of the largest ones)."""
    if scaling == "ntk" and rot == 2:
        return
    kind = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}[scaling]
    st, got = turns(rot, kind, 500000.0, factor, 4096.0, 2.0, 20.0)
    assert st == OK
    L = np.longdouble
    base = L(500000) * (L(factor) ** (L(rot) / (rot - 2)) if scaling == "ntk" else 1)
    pi = L("3.14159265358979323846264338327950288")
    for i in range(rot // 2):
        w = base ** (L(-2 * i) / rot)
        if scaling == "linear":
            w = w / L(factor)
        if scaling == "parts":
            keep = min(max((4096 * w / (2 * pi) - 2) / 18, L(0)), L(1))
            w = w * keep + w / factor * (1 - keep)
        part = Fraction(*(w / (2 * pi)).as_integer_ratio()) % 1 * (1 << 64)
        assert abs(int(got[i]) - part) <= 16 * max(1, float(w)), i
    host, scale = bd.make_rope_turns(rot, 500000.0, scaling=scaling, factor=factor, original=4096, slow=2, fast=20, device="cpu")
    assert host.tolist() == got.view(np.int64).tolist()
    assert scale == (0.1 * math.log(factor) + 1 if scaling == "parts" else 1.0)


def test_rope_turns_arguments():
    with pytest.raises(ValueError, match="unknown scaling"):
        bd.make_rope_turns(8, scaling="cubic", device="cpu")
    with pytest.raises(ValueError, match="original"):
        bd.make_rope_turns(8, scaling="parts", factor=2.0, device="cpu")
    with pytest.raises(bd.BdgdnError):
        bd.make_rope_turns(7, device="cpu")


def _rope(**kw):
    whole = layers.Heads(40 * 64 * 5, 40 * 64, 64)
    d = dict(num_req=2, nodes=5, h_q=8, h_k=2, d=64, rot=32, layout=0, dtype=bd.BDGDN_BF16, inverse=0, n_slots=4, scale=1.0,
             q=whole, k=whole, q_out=whole, k_out=whole)
    d.update(kw)
    return layers.RopeDesc(**d)


def _call_rope(desc, **ptr):
    p = dict(q=FAKE, k=FAKE, turns=FAKE, pos=None, len=None, slot=None, count=None, qo=FAKE, ko=FAKE)
    p.update(ptr)
    return bd.load_library().bdgdn_rope(desc, *p.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(num_req=-1), INV), (dict(nodes=-1), INV), (dict(h_q=0), INV), (dict(h_k=-1), INV), (dict(rot=0), INV), (dict(rot=7), INV),
    (dict(rot=66), INV), (dict(scale=math.inf), INV), (dict(scale=math.nan), INV), (dict(layout=2), INV), (dict(inverse=2), INV),
    (dict(dtype=3), UNS), (dict(d=4098), UNS), (dict(h_q=70000), UNS), (dict(num_req=1 << 16, nodes=1 << 15), UNS),
    (dict(q=layers.Heads(-1, 2560, 64)), INV), (dict(k=layers.Heads(0, 2560, -64)), INV),
    (dict(q=layers.Heads(1 << 50, 2560, 64)), INV),
    (dict(q_out=layers.Heads(12800, 2560, 63)), INV), (dict(q_out=layers.Heads(12800, 500, 64)), INV),
    (dict(q_out=layers.Heads(0, 2560, 64)), INV), (dict(k_out=layers.Heads(12800, 0, 64)), INV),
])
def test_rope_rejects_bad_descriptors(kw, status):
    assert _call_rope(_rope(**kw)) == status


@pytest.mark.parametrize("ptr", [dict(q=None), dict(k=None), dict(turns=None), dict(qo=None), dict(ko=None), dict(q=0x1001),
                                 dict(ko=0x1001), dict(turns=0x1004)])
def test_rope_rejects_bad_pointers(ptr):
    assert _call_rope(_rope(), **ptr) == INV


def test_rope_slots_and_places():
    assert _call_rope(_rope(h_k=0)) == INV                              # k without heads
    assert _call_rope(_rope(n_slots=1), len=FAKE) == INV                # two requests, one sequence, no slots
    assert _call_rope(_rope(n_slots=0), len=FAKE, slot=FAKE) == INV
    other = layers.Heads(12800, 2560, 128)
    assert _call_rope(_rope(q_out=other), qo=FAKE) == INV               # in place with other strides
    assert _call_rope(_rope(k_out=other), qo=0x2000, ko=FAKE) == INV
    assert _call_rope(_rope(num_req=0), q=None) == OK and _call_rope(_rope(nodes=0), q=None) == OK


# ------------------------------------------------------------------ norms
def _norm(**kw):
    d = dict(outer=6, inner=1, d=64, x_dtype=bd.BDGDN_BF16, r_dtype=bd.BDGDN_F32, dtype=bd.BDGDN_BF16, post=1, pre=1, act=1,
             scale=1.0, eps=1e-6)
    d.update({n: layers.Rows(64, 64) for n in ("x", "z", "r", "r_out", "y", "dx", "dz", "dr", "dr_out", "dy")})
    d.update(kw)
    return layers.NormDesc(**d)


def _fwd(desc, **ptr):
    p = dict(x=FAKE, z=FAKE, r=0x2000, w_post=FAKE, w_pre=FAKE, ls=FAKE, r_out=0x3000, y=0x4000)
    p.update(ptr)
    return bd.load_library().bdgdn_norm_fwd(desc, *p.values(), None)


def _bwd(desc, size=1 << 40, **ptr):
    p = dict(x=FAKE, z=FAKE, r_out=FAKE, w_post=FAKE, w_pre=FAKE, ls=FAKE, dy=FAKE, dr_out=0x2000, dx=0x3000, dz=0x4000,
             dr=0x5000, dw_post=FAKE, dw_pre=FAKE, dls=FAKE, ws=FAKE)
    p.update(ptr)
    return bd.load_library().bdgdn_norm_bwd(desc, *p.values(), size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(outer=-1), INV), (dict(inner=-1), INV), (dict(d=0), INV), (dict(d=16385), UNS), (dict(outer=1 << 16, inner=1 << 15), UNS),
    (dict(post=2), INV), (dict(pre=-1), INV), (dict(act=3), INV), (dict(act=-1), INV), (dict(scale=math.inf), INV),
    (dict(eps=-1e-6), INV), (dict(eps=math.nan), INV), (dict(x_dtype=2), UNS), (dict(r_dtype=-1), UNS), (dict(dtype=7), UNS),
    (dict(dtype=bd.BDGDN_F32), UNS), (dict(dtype=bd.BDGDN_F32, x_dtype=bd.BDGDN_F32, r_dtype=bd.BDGDN_BF16), UNS),
])
def test_norms_reject_bad_descriptors(kw, status):
    assert _fwd(_norm(**kw)) == status and _bwd(_norm(**kw)) == status and bd.bdgdn_norm_bwd_workspace(_norm(**kw)) == 0


def test_norms_reject_bad_rows_and_pointers():
    for name in ("x", "z", "r", "r_out", "y"):
        assert _fwd(_norm(**{name: layers.Rows(-64, 64)})) == INV, name
    for name in ("r_out", "y"):
        assert _fwd(_norm(**{name: layers.Rows(63, 64)})) == INV and _fwd(_norm(**{name: layers.Rows(0, 64)})) == INV, name
        assert _fwd(_norm(inner=2, **{name: layers.Rows(100, 64)})) == INV, name
    for name in ("dx", "dz", "dr"):
        assert _bwd(_norm(**{name: layers.Rows(63, 64)})) == INV, name
    for name in ("x", "dy", "dr_out"):
        assert _bwd(_norm(**{name: layers.Rows(1 << 50, 64)})) == INV, name
    assert _fwd(_norm(), x=None) == INV and _fwd(_norm(), r_out=None, y=None) == INV
    for name, at in (("x", 0x1001), ("z", 0x1001), ("r", 0x2002), ("y", 0x4001), ("r_out", 0x3002), ("w_post", 0x1002), ("ls", 0x1001)):
        assert _fwd(_norm(), **{name: at}) == INV, name
    assert _fwd(_norm(r=layers.Rows(128, 64)), r=0x3000) == INV         # in place with other strides
    assert _bwd(_norm(dr_out=layers.Rows(128, 64)), dr_out=0x5000) == INV
    assert _bwd(_norm(), x=None) == INV and _bwd(_norm(), dy=None, dr_out=None) == INV and _bwd(_norm(), z=None) == INV
    assert _bwd(_norm(post=0)) == INV and _bwd(_norm(pre=0)) == INV     # sums of weights that are not there
    none = dict(dx=None, dz=None, dr=None, dw_post=None, dw_pre=None, dls=None)
    assert _bwd(_norm(), **none) == INV
    for name, at in (("dx", 0x3001), ("dw_pre", 0x1002), ("dls", 0x1001), ("ws", 0x1040)):
        assert _bwd(_norm(), **{name: at}) == INV, name
    need = bd.bdgdn_norm_bwd_workspace(_norm())
    assert need > 0 and _bwd(_norm(), size=need - 1) == WS and _bwd(_norm(), ws=None) == WS
    assert _fwd(_norm(outer=0), x=None, y=None) == OK
    assert _bwd(_norm(inner=0), **dict(none, ws=None), x=None, dy=None) == OK
    assert bd.bdgdn_norm_bwd_workspace(_norm(outer=0)) == 0


# ------------------------------------------------------------------ logits
def _logits(**kw):
    d = dict(num_req=2, nodes=4, vocab=100, dtype=bd.BDGDN_BF16, out_dtype=bd.BDGDN_BF16, n_slots=3, n_bias=5, req_stride=400,
             row_stride=100, out_req_stride=400, out_row_stride=100, history_stride=100, allow_req_stride=16, allow_row_stride=4)
    d.update(kw)
    return layers.LogitsDesc(**d)


def _call_logits(desc, **ptr):
    p = dict(logits=FAKE, history=FAKE, slot=FAKE, token=FAKE, mask=FAKE, count=None, rho=None, presence=None, frequency=None,
             bias_token=FAKE, bias=FAKE, allow=FAKE, out=0x2000)
    p.update(ptr)
    return bd.load_library().bdgdn_logits(desc, *p.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(num_req=-1), INV), (dict(nodes=0), INV), (dict(nodes=65), UNS), (dict(vocab=0), INV), (dict(n_bias=-1), INV),
    (dict(n_slots=-1), INV), (dict(dtype=2), UNS), (dict(dtype=bd.BDGDN_F32), UNS), (dict(num_req=70000), UNS),
    (dict(vocab=(1 << 30) + 1, row_stride=1 << 31), UNS), (dict(req_stride=-1), INV), (dict(row_stride=-1), INV),
    (dict(out_row_stride=99), INV), (dict(out_req_stride=399), INV), (dict(out_row_stride=0), INV), (dict(history_stride=99), INV),
    (dict(allow_req_stride=-1), INV), (dict(n_slots=0), INV),
])
def test_logits_reject_bad_descriptors(kw, status):
    assert _call_logits(_logits(**kw)) == status


def test_logits_reject_bad_pointers():
    for name in ("logits", "token", "bias_token", "bias", "out"):
        assert _call_logits(_logits(), **{name: None}) == INV, name
    for name, at in (("logits", 0x1001), ("history", 0x1002), ("mask", 0x1004), ("allow", 0x1001), ("out", 0x2001)):
        assert _call_logits(_logits(), **{name: at}) == INV, name
    assert _call_logits(_logits(n_bias=0)) == INV
    assert _call_logits(_logits(n_slots=1), slot=None) == INV
    assert _call_logits(_logits(out_dtype=bd.BDGDN_F32), out=FAKE) == INV
    assert _call_logits(_logits(out_row_stride=101, out_req_stride=404), out=FAKE) == INV
    assert _call_logits(_logits(num_req=0), logits=None) == OK


def test_history_add_rejects():
    f = bd.load_library().bdgdn_history_add
    ok = dict(R=2, N=3, V=10, slots=4, stride=10, history=FAKE, slot=FAKE, token=FAKE, path=None, count=None, prompt=0)

    def call(**kw):
        return f(*dict(ok, **kw).values(), None)

    for kw in (dict(R=-1), dict(N=-1), dict(V=0), dict(slots=0), dict(stride=-1), dict(stride=9), dict(prompt=2), dict(history=None),
               dict(token=None), dict(history=0x1002), dict(slot=None, R=5)):
        assert call(**kw) == INV, kw
    assert call(R=0, history=None) == OK and call(N=0, history=None) == OK


# ------------------------------------------------------------------ 8-bit products
def test_quant_rows_rejects():
    def call(x=FAKE, q=FAKE, scale=FAKE, **kw):
        d = dict(rows=3, cols=100, width=128, dtype=bd.BDGDN_F32, x_stride=100, q_stride=128)
        d.update(kw)
        return bd.load_library().bdgdn_quant_rows(layers.QuantDesc(**d), x, q, scale, None)

    for kw in (dict(rows=-1), dict(cols=0), dict(width=0), dict(width=100), dict(width=256), dict(x_stride=-1), dict(q_stride=112),
               dict(q_stride=136), dict(x=None), dict(q=None), dict(scale=None), dict(x=0x1002), dict(q=0x1008), dict(scale=0x1002)):
        assert call(**kw) == INV, kw
    assert call(dtype=2) == UNS and call(cols=(1 << 30) + 1) == UNS and call(rows=1 << 24) == UNS and call(rows=0, x=None) == OK


def test_quant_matmul_rejects():
    lib = bd.load_library()

    def call(a=FAKE, sa=FAKE, w=FAKE, sw=FAKE, bias=None, out=FAKE, ws=FAKE, size=1 << 40, **kw):
        d = dict(m=3, n=5, k=256, out_dtype=bd.BDGDN_BF16, a_stride=256, w_stride=256, out_stride=5)
        d.update(kw)
        return lib.bdgdn_quant_matmul(layers.QuantMatmulDesc(**d), a, sa, w, sw, bias, out, ws, size, None)

    for kw in (dict(m=-1), dict(n=0), dict(k=0), dict(k=192), dict(a_stride=-16), dict(a_stride=264), dict(w_stride=250),
               dict(out_stride=4), dict(a=None), dict(sa=None), dict(w=None), dict(sw=None), dict(out=None), dict(a=0x1008),
               dict(w=0x1008), dict(sa=0x1002), dict(bias=0x1001), dict(out=0x1001), dict(ws=0x1080)):
        assert call(**kw) == INV, kw
    for kw in (dict(out_dtype=2), dict(k=131072), dict(n=(1 << 26) + 1, out_stride=1 << 27), dict(m=(1 << 30) + 1),
               dict(m=1 << 24, n=1 << 20, out_stride=1 << 20)):
        assert call(**kw) == UNS, kw
    assert call(m=0, a=None) == OK
    for m in (1, 64, 65, 500):
        desc = layers.QuantMatmulDesc(m, 512, 2048, bd.BDGDN_F32, 2048, 2048, 512)
        need = bd.bdgdn_quant_matmul_workspace(desc)
        if need:
            assert call(m=m, n=512, k=2048, a_stride=2048, w_stride=2048, out_stride=512, size=need - 1) == WS


# ------------------------------------------------------------------ the binding
def test_the_binding_refuses_what_is_not_on_the_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x, w = torch.zeros(2, 8), torch.zeros(8, dtype=torch.int64)
    for call in (lambda: bd.bdgdn_rope(torch.zeros(1, 1, 1, 8), w), lambda: bd.bdgdn_norm_fwd(x), lambda: bd.bdgdn_norm_bwd(x, x),
                 lambda: bd.bdgdn_logits(torch.zeros(1, 1, 8)), lambda: bd.bdgdn_history_add(torch.zeros(1, 8, dtype=torch.int32), w),
                 lambda: bd.bdgdn_quant_rows(x), lambda: bd.bdgdn_quant_matmul(x.to(torch.int8), x, x.to(torch.int8), x)):
        with pytest.raises(ValueError, match="must be a device tensor"):
            call()


def test_the_binding_refuses_other_devices(monkeypatch):
    class Elsewhere(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 1

    class Stream:
        device_index, cuda_stream = 1, 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x = torch.zeros(2, 8).as_subclass(Elsewhere)
    with pytest.raises(ValueError, match="x is on device 1, the call runs on device 0"):
        bd.bdgdn_norm_fwd(x)
    with pytest.raises(ValueError, match="the stream is on device 1"):
        bd.bdgdn_norm_fwd(x, stream=Stream())


def test_kept_plans_follow_shapes_and_strides():
    def same(a, b):
        return bytes(a) == bytes(b)

    q = torch.empty(2, 3, 4, 8)
    plan = layers._rope_plan(q.shape, q.stride(), None, None, None, None, None, None, torch.float32, 8, 0, False, 1.0, 0)
    assert plan.q_out.req == 96 and plan.h_k == 0 and plan.dtype == bd.BDGDN_F32
    t = q.transpose(1, 2)
    other = layers._rope_plan(t.shape, t.stride(), None, None, None, None, None, None, torch.float32, 8, 0, False, 1.0, 0)
    assert not same(plan, other) and (other.q.row, other.q.head) == (8, 32)
    with pytest.raises(ValueError, match="contiguous"):
        u = torch.empty(2, 3, 8, 4).transpose(2, 3)
        layers._rope_plan(u.shape, u.stride(), None, None, None, None, None, None, torch.float32, 8, 0, False, 1.0, 0)
    with pytest.raises(ValueError, match="unknown layout"):
        layers._rope_plan(q.shape, q.stride(), None, None, None, None, None, None, torch.float32, 8, None, False, 1.0, 0)
    types, none = (torch.bfloat16, torch.float32, torch.bfloat16), (None,) * 9
    desc, need = layers._norm_plan((5, 64), ((70, 1),) + none, types, True, True, 1, 1.0, 1e-6)
    assert (desc.outer, desc.inner, desc.x.outer, desc.y.outer) == (5, 1, 70, 64) and need == bd.bdgdn_norm_bwd_workspace(desc)
    desc, _ = layers._norm_plan((5, 3, 64), ((400, 70, 1),) + none, types, True, False, 1, 1.0, 1e-6)
    assert (desc.inner, desc.x.inner, desc.y.outer, desc.y.inner) == (3, 70, 192, 64)
    for shape, strides, match in (((64,), (1,), "x must be"), ((5, 64), (1, 5), "contiguous")):
        with pytest.raises(ValueError, match=match):
            layers._norm_plan(shape, (strides,) + none, types, True, True, 1, 1.0, 1e-6)
    with pytest.raises(ValueError, match="unknown act"):
        layers._norm_plan((5, 64), none + (None,), types, True, True, None, 1.0, 1e-6)
