"""Rows of more than 4096 elements, several to a workgroup (there are at most 256 in the backward, and in the
forward from 8192 on): sums over rows, alternating buffers, rows that are read again, every part.

Tolerances as for the other sizes: a lane's chain has up to 16 squares in the forward and 32 in the backward
(four chunks), then 6 steps across lanes and 8 or 16 across waves, under 54 roundings of 2^-24, halved by
the root: 2^-19.2, which the bounds of 2^-17 and 2^-16 of a result's terms hold as they hold 2^-19.7.
The weights' sums add 3 rows to a workgroup and 16 + 16 workgroups: 2^-14 holds them.
"""
import pytest
import torch

import paper_2606_01774_amd as bd
from test_gpu_norm import B, F, NAMES, backward, forward, make, near

pytestmark = pytest.mark.gpu

ROWS = 600


@pytest.mark.parametrize("types", [(B, F, B), (F, F, F)])
@pytest.mark.parametrize("d", [5000, 8192, 8200, 16383])
def test_several_long_rows_to_a_workgroup(d, types):
    x, z, r, w, dy, dr = make((ROWS, d), types, d)
    kw = dict(post=True, pre=True, act="silu", scale=0.8, eps=1e-5)
    ws = dict(w_post=w[0], w_pre=w[1], layer_scale=w[2])
    y, new = bd.bdgdn_norm_fwd(x, z=z, r=r, **ws, **kw)
    for got, (want, size), name in zip((y, new), forward(x, z, r, w, True, True, "silu", 0.8, 1e-5), ("y", "r_out")):
        near(got, want, size, name)
    first, again = (bd.bdgdn_norm_bwd(x, dy, z=z, r_out=new, dr_out=dr, **ws, **kw) for _ in range(2))
    want, size = backward(x, z, new, dy, dr, w, True, True, "silu", 0.8, 1e-5)
    for name, got, other in zip(NAMES, first, again):
        assert torch.equal(got, other), name
        near(got, want[name], size[name], name, 2.0 ** -14 if got.dim() == 1 else 2.0 ** -16)


@pytest.mark.parametrize("d,types", [(5000, (B, F, B)), (9001, (F, F, F))])
@pytest.mark.parametrize("post,pre,act,gated,residual,weights", [
    (True, False, "none", False, False, (True, False, False)), (False, True, "none", False, True, (False, True, False)),
    (False, True, "none", False, True, (False, False, False)), (False, False, "sigmoid", True, True, (False, False, True)),
    (False, False, "none", True, False, (False, False, False)), (True, True, "sigmoid", True, False, (True, True, True)),
    (True, True, "none", False, False, (True, True, False)), (True, False, "silu", True, True, (True, False, False)),
    (False, True, "silu", True, False, (False, True, True)),
])
def test_parts_of_long_rows(post, pre, act, gated, residual, weights, d, types):
    x, z, r, w, dy, dr = make((ROWS, d), types, d + 5, gated, weights, residual)
    kw = dict(post=post, pre=pre, act=act, scale=-1.25, eps=1e-3)
    ws = dict(w_post=w[0], w_pre=w[1], layer_scale=w[2])
    y, new = bd.bdgdn_norm_fwd(x, z=z, r=r, out_dtype=types[2], **ws, **kw)
    (ref_y, size_y), (ref_r, size_r) = forward(x, z, r, w, post, pre, act, -1.25, 1e-3)
    near(y, ref_y, size_y, "y")
    if residual:
        near(new, ref_r, size_r, "r_out")
    grads = bd.bdgdn_norm_bwd(x, dy, z=z, r_out=new, dr_out=dr if residual else None, **ws, **kw)
    want, size = backward(x, z, new, dy, dr if residual else None, w, post, pre, act, -1.25, 1e-3)
    there = (True, gated, residual, weights[0] and post, weights[1] and pre, weights[2])
    for name, got, is_there in zip(NAMES, grads, there):
        assert (got is not None) == is_there, name
        if is_there:
            near(got, want[name], size[name], name, 2.0 ** -14 if got.dim() == 1 else 2.0 ** -16)
