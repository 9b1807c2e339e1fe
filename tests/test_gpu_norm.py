"""bdgdn_norm_fwd and bdgdn_norm_bwd against the definition in 64 bits.

Tolerances.  fp32 sums of d squares are taken in chains of at most 16 elements, 6 steps across lanes and
16 across waves: 38 roundings of 2^-24, halved by the root, under 2^-19.7.  The gate's exponent -1.44 z is
rounded (2^-24 of up to 1.44 x 6 for the z here) and the exponential, sum and reciprocal a few more times:
under 2^-19.  Every factor adds a rounding, ten at most.  So a term of n factors is within 2^-18 of
itself, and each result within 2^-17 of the sum of its terms' magnitudes (``size``), which the
reference computes beside it, and half a step of its type.  The means in the backward are sums of d such
terms: their magnitudes enter ``size``.  Sums over the rows add rows / groups roundings, under 1000 here:
2^-14.
"""
import pytest
import torch

import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu

STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
NAMES = ("dx", "dz", "dr", "dw_post", "dw_pre", "dlayer_scale")
B, F = torch.bfloat16, torch.float32


def gate(z, act):
    if act == "none":
        return z, torch.ones_like(z)
    e = torch.sigmoid(z)
    return (e, e * (1 - e)) if act == "sigmoid" else (z * e, e * (1 + z * (1 - e)))


def parts(x, z, r, w, post, pre, act, scale, eps):
    one = torch.ones(x.shape[-1], dtype=torch.float64)
    wp, wq, ls = (one if t is None else t.double().cpu() for t in w)
    x = x.double().cpu()
    s1 = (x.square().mean(-1, keepdim=True) + eps).rsqrt() if post else torch.ones(x.shape[:-1] + (1,), dtype=torch.float64)
    xh = x * s1
    n = xh * wp if post else xh
    a, slope = (torch.ones_like(n), torch.zeros_like(n)) if z is None else gate(z.double().cpu(), act)
    return wp, wq, ls, s1, xh, n, a, slope


def forward(x, z, r, w, post, pre, act, scale, eps):
    """(y, r'), each with the magnitudes of its terms."""
    wp, wq, ls, s1, xh, n, a, _ = parts(x, z, r, w, post, pre, act, scale, eps)
    add = scale * ls * n * a
    rr = torch.zeros_like(add) if r is None else r.double().cpu()
    new, size = rr + add, rr.abs() + add.abs()
    if not pre:
        return (new, size), (new, size)
    s2 = (new.square().mean(-1, keepdim=True) + eps).rsqrt()
    # the row's statistic carries the errors of the sum's terms
    lost = (size * new.abs()).mean(-1, keepdim=True) * s2 * s2
    return (new * s2 * wq, (size + new.abs() * lost) * s2 * wq.abs()), (new, size)


def backward(x, z, r_new, dy, dr_new, w, post, pre, act, scale, eps):
    wp, wq, ls, s1, xh, n, a, slope = parts(x, z, None, w, post, pre, act, scale, eps)
    zero = torch.zeros_like(xh)
    dy = zero if dy is None else dy.double().cpu()
    dr_new = zero if dr_new is None else dr_new.double().cpu()
    new = scale * ls * n * a if r_new is None else r_new.double().cpu()
    out, size = {}, {}
    if pre:
        s2 = (new.square().mean(-1, keepdim=True) + eps).rsqrt()
        h, t = new * s2, dy * wq
        g = s2 * (t - h * (t * h).mean(-1, keepdim=True)) + dr_new
        gs = s2 * (t.abs() + 2 * h.abs() * (t * h).abs().mean(-1, keepdim=True)) + dr_new.abs()
        out["dw_pre"], size["dw_pre"] = (dy * h), (dy * h).abs()
    else:
        g, gs = dy + dr_new, dy.abs() + dr_new.abs()
    out["dr"], size["dr"] = g, gs
    out["dlayer_scale"], size["dlayer_scale"] = scale * g * n * a, (scale * gs * n * a).abs()
    du, dus = scale * ls * g, (scale * ls * gs).abs()
    out["dz"] = du * n * slope
    size["dz"] = dus * n.abs() * (slope.abs() + (0.3 if act != "none" else 0))   # (1 + z (1 - e) cancels)
    dn, dns = du * a, dus * a.abs()
    out["dw_post"], size["dw_post"] = dn * xh, dns * xh.abs()
    if post:
        t, ts = dn * wp, dns * wp.abs()
        out["dx"] = s1 * (t - xh * (t * xh).mean(-1, keepdim=True))
        size["dx"] = s1 * (ts + 2 * xh.abs() * (ts * xh.abs()).mean(-1, keepdim=True))
    else:
        out["dx"], size["dx"] = dn, dns
    rows = tuple(range(xh.dim() - 1))
    for k in ("dw_post", "dw_pre", "dlayer_scale"):
        if k in out:
            out[k], size[k] = out[k].sum(rows), size[k].sum(rows)
    return out, size


def near(got, want, size, name, extra=2.0 ** -17):
    err = (got.double().cpu() - want).abs()
    bound = extra * size + STEP[got.dtype] * want.abs() + 1e-37
    assert (err <= bound).all(), f"{name}: {float((err / bound).max()):.2f} of what is allowed"


def make(shape, types, seed, gated=True, weights=(True, True, True), residual=True):
    g = torch.Generator().manual_seed(seed)
    xt, rt, yt = types
    rand = lambda t, std: (torch.randn(*shape, generator=g) * std).to(t).cuda()  # noqa: E731
    x, z, r = rand(xt, 1.7), rand(yt, 1.5).clamp(-6, 6) if gated else None, rand(rt, 2.0) if residual else None
    w = [(1 + 0.3 * torch.randn(shape[-1], generator=g)).cuda() if there else None for there in weights]
    return x, z, r, w, rand(yt, 1.0), rand(rt, 1.0)


TYPES = [(B, F, B), (B, B, B), (F, F, F), (F, F, B), (F, B, B)]
SIZES = [(1, 1), (3, 2), (2, 8), (5, 100), (70, 128), (9, 129), (3, 512), (4, 776), (2, 2048), (5, 2051), (3, 4096), (2, 5000),
         (3, 8192), (1, 8200), (2, 16384), (1, 16383)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,d", SIZES)
def test_everything_at_once(rows, d, types):
    x, z, r, w, dy, dr = make((rows, d), types, rows + d)
    kw = dict(post=True, pre=True, act="silu", scale=0.8, eps=1e-5)
    ws = dict(w_post=w[0], w_pre=w[1], layer_scale=w[2])
    y, new = bd.bdgdn_norm_fwd(x, z=z, r=r, **ws, **kw)
    assert y.dtype is types[2] and new.dtype is types[1]
    for got, (want, size), name in zip((y, new), forward(x, z, r, w, True, True, "silu", 0.8, 1e-5), ("y", "r_out")):
        near(got, want, size, name)
    grads = bd.bdgdn_norm_bwd(x, dy, z=z, r_out=new, dr_out=dr, **ws, **kw)
    want, size = backward(x, z, new, dy, dr, w, True, True, "silu", 0.8, 1e-5)
    for name, got in zip(NAMES, grads):
        near(got, want[name], size[name], name, 2.0 ** -14 if got.dim() == 1 else 2.0 ** -16)


@pytest.mark.parametrize("types", [(B, F, B), (F, F, F)])
@pytest.mark.parametrize("d", [48, 1000, 1003])
@pytest.mark.parametrize("post,pre,act,gated,residual,weights", [
    (True, False, "none", False, False, (True, False, False)), (True, False, "none", False, False, (False, False, False)),
    (False, True, "none", False, True, (False, True, False)), (False, True, "none", False, True, (False, False, False)),
    (False, False, "sigmoid", True, True, (False, False, True)), (False, False, "none", True, False, (False, False, False)),
    (True, True, "sigmoid", True, False, (True, True, True)), (True, True, "none", False, False, (True, True, False)),
    (True, False, "silu", True, True, (True, False, False)), (False, True, "silu", True, False, (False, True, True)),
])
def test_parts(post, pre, act, gated, residual, weights, d, types):
    x, z, r, w, dy, dr = make((11, d), types, d + 5, gated, weights, residual)
    kw = dict(post=post, pre=pre, act=act, scale=-1.25, eps=1e-3)
    ws = dict(w_post=w[0], w_pre=w[1], layer_scale=w[2])
    y, new = bd.bdgdn_norm_fwd(x, z=z, r=r, out_dtype=types[2], **ws, **kw)
    (ref_y, size_y), (ref_r, size_r) = forward(x, z, r, w, post, pre, act, -1.25, 1e-3)
    near(y, ref_y, size_y, "y")
    assert (new is None) == (not residual)
    if residual:
        near(new, ref_r, size_r, "r_out")
    for up in ("both", "y", "r") if residual else ("y",):
        gy, gr = (None if up == "r" else dy), (None if up == "y" or not residual else dr)
        grads = bd.bdgdn_norm_bwd(x, gy, z=z, r_out=new, dr_out=gr, **ws, **kw) if gated or gy is not None or types[0] is types[2] \
            else bd.bdgdn_norm_bwd(x, torch.zeros_like(dy), z=z, r_out=new, dr_out=gr, **ws, **kw)
        want, size = backward(x, z, new, gy, gr, w, post, pre, act, -1.25, 1e-3)
        there = (True, gated, residual, weights[0] and post, weights[1] and pre, weights[2])
        for name, got, is_there in zip(NAMES, grads, there):
            assert (got is not None) == is_there, name
            if is_there:
                near(got, want[name], size[name], name, 2.0 ** -14 if got.dim() == 1 else 2.0 ** -16)


@pytest.mark.parametrize("d,heads", [(64, 3), (128, 16), (100, 2), (256, 5)])
def test_gated_norm_of_heads(d, heads):
    """The norm behind a Gated DeltaNet: fp32 outputs of the mixer, the gate a part of a projection's
    rows, many rows; and a call whose outputs are parts of longer rows, which stay as they were."""
    T = 700
    x, _, _, w, dy, _ = make((T, heads, d), (F, F, B), d, False, (True, False, False))
    proj = torch.randn(T, 3 * heads * d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    z = proj[:, heads * d:2 * heads * d].unflatten(1, (heads, d))
    kw = dict(w_post=w[0], post=True, act="silu")
    y, new = bd.bdgdn_norm_fwd(x, z=z, **kw)
    assert new is None
    (want, size), _ = forward(x, z, None, w, True, False, "silu", 1.0, 1e-6)
    near(y, want, size, "y")
    dx, dz, dr, dw, _, _ = bd.bdgdn_norm_bwd(x, dy, z=z, **kw)
    ref, mag = backward(x, z, None, dy, None, w, True, False, "silu", 1.0, 1e-6)
    for name, got in (("dx", dx), ("dz", dz), ("dw_post", dw)):
        near(got, ref[name], mag[name], name, 2.0 ** -14 if got.dim() == 1 else 2.0 ** -16)
    assert dr is None
    room = torch.full((T, 3 * heads * d), 9.0, dtype=B, device="cuda")
    into = room[:, heads * d:2 * heads * d].unflatten(1, (heads, d))
    dz2 = bd.bdgdn_norm_bwd(x, dy, z=z, dz=into, **kw)[1]
    assert dz2 is into and torch.equal(into, dz) and (room[:, :heads * d] == 9).all() and (room[:, 2 * heads * d:] == 9).all()
    bd.bdgdn_norm_fwd(x, z=z, y=into, **kw)
    assert torch.equal(into, y)


def test_gradients_against_differences():
    """Central differences of <y, dy> + <r', dr'> in fp32 at steps of 2^-6: the third derivative's part is
    2^-12 / 6 of numbers of some units, the loss's rounding 2^-24 x 100 / 2^-5; 2 % of the gradients' size."""
    rows, d = 3, 24
    x, z, r, w, dy, dr = make((rows, d), (F, F, F), 2)
    kw = dict(post=True, pre=True, act="silu", scale=0.9)

    def loss(x, z, r, w):
        y, new = bd.bdgdn_norm_fwd(x, z=z, r=r, w_post=w[0], w_pre=w[1], layer_scale=w[2], **kw)
        return float((y.double() * dy).sum() + (new.double() * dr).sum())

    new = bd.bdgdn_norm_fwd(x, z=z, r=r, w_post=w[0], w_pre=w[1], layer_scale=w[2], **kw)[1]
    grads = bd.bdgdn_norm_bwd(x, dy, z=z, r_out=new, dr_out=dr, w_post=w[0], w_pre=w[1], layer_scale=w[2], **kw)
    for i, grad in enumerate(grads):
        args = [x, z, r, *w]
        rms = float(grad.square().mean().sqrt())
        for at in (0, 5, grad.numel() - 1):
            step = torch.zeros_like(args[i]).flatten()
            step[at] = 2.0 ** -6
            lo, hi = ([a + s * step.view_as(a) if j == i else a for j, a in enumerate(args)] for s in (-1, 1))
            diff = (loss(hi[0], hi[1], hi[2], hi[3:]) - loss(lo[0], lo[1], lo[2], lo[3:])) / 2.0 ** -5
            assert abs(diff - float(grad.flatten()[at])) < 0.02 * (rms + abs(diff)), (NAMES[i], at)


def test_in_place_strides_and_rows_of_zeros():
    rows, d = 6, 96
    x, z, r, w, dy, dr = make((rows, d), (B, F, B), 3)
    x[2] = 0
    r[2] = 0
    kw = dict(z=z, w_post=w[0], w_pre=w[1], post=True, pre=True)
    y, new = bd.bdgdn_norm_fwd(x, r=r, **kw)
    assert (y[2] == 0).all() and (new[2] == 0).all()
    r2 = r.clone()
    y2, new2 = bd.bdgdn_norm_fwd(x, r=r2, r_out=r2, **kw)
    assert new2 is r2 and torch.equal(r2, new) and torch.equal(y2, y)
    up = dr.clone()
    grads = bd.bdgdn_norm_bwd(x, dy, r_out=new, dr_out=dr, **kw)
    inside = bd.bdgdn_norm_bwd(x, dy, r_out=new, dr_out=up, dr=up, **kw)
    for a, b in zip(grads, inside):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    # a row with a NaN or an infinity keeps it to itself
    for bad in (float("nan"), float("inf")):
        x3 = x.clone()
        x3[4, 7] = bad
        y3, new3 = bd.bdgdn_norm_fwd(x3, r=r, **kw)
        assert y3[4].isnan().any() and torch.equal(y3[:4], y[:4]) and torch.equal(new3[5], new[5])
    # addresses and strides that are no multiples of 16 bytes
    wide = torch.randn(rows, d + 3, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    y4, _ = bd.bdgdn_norm_fwd(wide[:, 1:d + 1], w_post=w[0], post=True)
    y5, _ = bd.bdgdn_norm_fwd(wide[:, 1:d + 1].contiguous(), w_post=w[0], post=True)
    (want, size), _ = forward(wide[:, 1:d + 1], None, None, (w[0], None, None), True, False, "none", 1.0, 1e-6)
    near(y4, want, size, "y")
    near(y5, want, size, "y")


@pytest.mark.parametrize("rows,d", [(20000, 16), (4097, 300), (3001, 1500), (2050, 4000)])
def test_sums_over_many_rows(rows, d):
    x, z, r, w, dy, dr = make((rows, d), (F, F, F), rows)
    kw = dict(z=z, r_out=r, dr_out=dr, w_post=w[0], w_pre=w[1], layer_scale=w[2], post=True, pre=True, act="sigmoid")
    first, again = (bd.bdgdn_norm_bwd(x, dy, **kw) for _ in range(2))
    want, size = backward(x, z, r, dy, dr, w, True, True, "sigmoid", 1.0, 1e-6)
    for name, a, b in zip(NAMES, first, again):
        assert torch.equal(a, b), name
        near(a, want[name], size[name], name, 2.0 ** -14 if a.dim() == 1 else 2.0 ** -16)


def test_no_rows():
    w = torch.ones(32, device="cuda")
    y, new = bd.bdgdn_norm_fwd(torch.zeros(0, 32, device="cuda"), r=torch.zeros(0, 32, device="cuda"), w_pre=w, pre=True)
    assert y.shape == new.shape == (0, 32)
    empty = torch.zeros(0, 3, 32, device="cuda")
    dx, _, _, dw, _, dls = bd.bdgdn_norm_bwd(empty, empty, w_post=w, layer_scale=w, post=True,
                                             dw_post=torch.full_like(w, 7.0))
    assert dx.shape == (0, 3, 32) and (dw == 0).all() and (dls == 0).all()
