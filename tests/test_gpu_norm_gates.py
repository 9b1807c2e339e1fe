"""The gate's slope in bdgdn_norm_bwd where the gate is nearly open or nearly shut.

Tolerance.  The exponent -1.44 z is off by the constant's rounding and the product's, 2 x 2^-24 of itself, so
the exponential by 2 |z| 2^-24; the exponential, the sum with 1, the reciprocal, the slope's product and
the factors of dz add under 24 roundings of 2^-24: (2 |z| + 24) 2^-24 of the exact dz, and half a step of
its type.  Beyond |z| = 80 the slope leaves the range of fp32's normal numbers: under 2^-110 there.
"""
import pytest
import torch

import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu

STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.mark.parametrize("d", [64, 100, 5000, 9000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_slope_of_a_saturated_sigmoid(dtype, d):
    rows = 5
    g = torch.Generator().manual_seed(d)
    z = (torch.rand(rows, d, generator=g) * 160 - 80).to(dtype)
    z[:, :40] = torch.arange(-20, 20).to(dtype)
    z[0, 40:46] = torch.tensor([16.5, 17.0, 24.0, 80.0, -80.0, 0.0])
    x, dy = (torch.randn(rows, d, generator=g).to(dtype) for _ in range(2))
    dz = bd.bdgdn_norm_bwd(x.cuda(), dy.cuda(), z=z.cuda(), act="sigmoid")[1].cpu()
    zd = z.double()
    want = dy.double() * x.double() * torch.sigmoid(zd) * torch.sigmoid(-zd)
    err = (dz.double() - want).abs()
    bound = ((2 * zd.abs() + 24) * 2.0 ** -24 + STEP[dtype]) * want.abs() + 1e-37
    assert (err <= bound).all(), float((err / bound).max())


def test_slope_of_a_gate_without_bounds():
    z = torch.tensor([[100.0, -100.0, 3e38, -3e38, float("inf"), -float("inf"), 1e4, -1e4]], device="cuda")
    x = torch.ones_like(z)
    dx, dz = bd.bdgdn_norm_bwd(x, x, z=z, act="sigmoid")[:2]
    assert (dz.abs() <= 2.0 ** -110).all()
    assert ((dx - torch.tensor([[1.0, 0, 1, 0, 1, 0, 1, 0]], device="cuda")).abs() <= 2.0 ** -110).all()
