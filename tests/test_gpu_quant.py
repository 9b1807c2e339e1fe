"""bdgdn_quant_rows and bdgdn_quant_matmul.

quant_rows is held to its definition bit for bit: the product max |x| (1 / 127) and the quotients are single
correctly rounded fp32 operations, which numpy's are too.  The product's integer sums are exact; a_scale w_scale,
the sum as fp32, its product with the scales and the bias's sum are rounded once each (the last two
together): 3 x 2^-24 of |sum scales| + |bias|, and half a step of the result's type.
"""
import numpy as np
import pytest
import torch

import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu

STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
B, F = torch.bfloat16, torch.float32


def quantised(x):
    x = x.float().cpu().numpy()
    top = np.abs(x).max(-1, keepdims=True)
    scale = (top * (np.float32(1) / np.float32(127))).astype(np.float32)
    with np.errstate(all="ignore"):
        q = np.clip(np.rint(np.where(scale > 0, x / scale, 0)), -127, 127)
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(scale[:, 0])


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 128), (5, 129), (300, 1000), (4, 4096), (2, 20001)])
def test_rows(rows, cols, dtype):
    g = torch.Generator().manual_seed(rows + cols)
    x = (torch.randn(rows, cols, generator=g) * 10.0 ** torch.randint(-6, 6, (rows, 1), generator=g)).to(dtype)
    q, scale = bd.bdgdn_quant_rows(x.cuda())
    want, s = quantised(x)
    assert q.shape == (rows, -(-cols // 128) * 128) and torch.equal(scale.cpu(), s)
    assert torch.equal(q[:, :cols].cpu(), want) and not q[:, cols:].any()


def test_rows_at_the_ends():
    x = torch.zeros(8, 130)
    x[1, 129] = 1e-45              # its scale is zero in fp32
    x[2, 3], x[2, 4] = 3e38, -3.4e38
    x[3, 0] = float("nan")
    x[4, 7], x[4, 9] = float("inf"), 2.0
    x[5] = torch.arange(130) - 64.5
    x[5, 0], x[5, 129] = -127.0, 63.5     # scale 1: quotients half way between integers
    x[6, 5] = -1e-40
    x[7] = -7.25
    q, scale = bd.bdgdn_quant_rows(x.cuda())
    q, scale = q.cpu(), scale.cpu()
    assert not q[0].any() and scale[0] == 0 and not q[1].any() and scale[1] == 0
    assert not q[3].any() and scale[3].isnan() and not q[4].any() and scale[4].isnan()
    for r in (2, 5, 6, 7):
        want, s = quantised(x[r:r + 1])
        assert torch.equal(q[r:r + 1, :130], want) and scale[r] == s[0], r
    assert q[5, 2] == -62 and q[5, 3] == -62      # -62.5 and -61.5 go to the even one
    y = bd.bdgdn_quant_matmul(q.cuda(), scale.cuda(), q[5:6].cuda(), scale[5:6].cuda(), out_dtype=F)
    assert y[3].isnan() and y[4].isnan() and y[0] == 0 and y[5].isfinite()


def test_rows_of_longer_rows():
    room = torch.randn(6, 211, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    into = torch.full((6, 160), 77, dtype=torch.int8, device="cuda")
    q, scale = bd.bdgdn_quant_rows(room[:, 5:105], q=into[:, 16:144])
    want, s = quantised(room[:, 5:105])
    assert torch.equal(q[:, :100].cpu(), want) and torch.equal(scale.cpu(), s) and not q[:, 100:].any()
    assert (into[:, :16] == 77).all() and (into[:, 144:] == 77).all()


def product(a, sa, w, sw, bias):
    total = a.cpu().double() @ w.cpu().double().T
    terms = total * sa.cpu().double()[:, None] * sw.cpu().double()
    b = torch.zeros(w.shape[0], dtype=torch.float64) if bias is None else bias.cpu().double()
    return terms + b, terms.abs() + b.abs()


def near(y, want, size):
    err = (y.cpu().double() - want).abs()
    assert (err <= 3 * 2.0 ** -24 * size + STEP[y.dtype] * want.abs()).all(), float((err / (size + 1e-30)).max())


def make(m, n, k, seed, full=False):
    g = torch.Generator().manual_seed(seed)
    lo, hi = (-128, 128) if full else (-127, 128)
    a, w = (torch.randint(lo, hi, (r, k), generator=g).to(torch.int8).cuda() for r in (m, n))
    sa, sw = (torch.rand(r, generator=g).cuda() + 0.1 for r in (m, n))
    return a, sa, w, sw, torch.randn(n, generator=g).cuda() * 1000


@pytest.mark.parametrize("out", [B, F])
@pytest.mark.parametrize("n,k", [(1, 128), (17, 256), (64, 1024), (130, 2176), (333, 640)])
@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 33, 48, 64, 65, 100, 128, 129, 257, 300])
def test_product(m, n, k, out):
    a, sa, w, sw, bias = make(m, n, k, m + n + k)
    for b in (None, bias):
        near(bd.bdgdn_quant_matmul(a, sa, w, sw, bias=b, out_dtype=out), *product(a, sa, w, sw, b))


@pytest.mark.parametrize("m,n,k", [(3, 70, 130944), (70, 40, 130944), (200, 150, 16384), (1024, 2056, 384), (513, 3000, 2048),
                                   (40, 5000, 4096)])
def test_long_sums_and_many_tiles(m, n, k):
    a, sa, w, sw, bias = make(m, n, k, 5, full=True)
    if k == 130944:   # the largest sum there is
        a[-1], w[-1], w[0] = -128, -128, 127
    near(bd.bdgdn_quant_matmul(a, sa, w, sw, bias=bias, out_dtype=F), *product(a, sa, w, sw, bias))


@pytest.mark.parametrize("m", [5, 30, 64, 140])
def test_strides(m):
    """Operands and results that are parts of longer rows; what lies beside the result stays."""
    n, k = 75, 256
    a, sa, w, sw, bias = make(m, n, k + 128, 3)
    out = torch.full((m, n + 9), 3.0, device="cuda")
    y = bd.bdgdn_quant_matmul(a[:, 16:16 + k], sa, w[:, 32:32 + k], sw, out=out[:, 4:4 + n])
    near(y, *product(a[:, 16:16 + k], sa, w[:, 32:32 + k], sw, None))
    assert (out[:, :4] == 3).all() and (out[:, 4 + n:] == 3).all()
    one = a[:1, :k].expand(m, k)      # one row for all
    near(bd.bdgdn_quant_matmul(one, sa, w[:, :k], sw, out_dtype=F), *product(one, sa, w[:, :k], sw, None))


def test_a_projection_of_quantised_rows():
    """Quantised activations and weights: every entry off by half a step of its row at most, so a product
    of k is within sum |x| sw / 2 + |w| sx / 2 + k sx sw / 4 of the unquantised one."""
    m, n, k = 37, 90, 500
    g = torch.Generator().manual_seed(8)
    x, w = torch.randn(m, k, generator=g).cuda(), torch.randn(n, k, generator=g).cuda()
    qx, sx = bd.bdgdn_quant_rows(x)
    qw, sw = bd.bdgdn_quant_rows(w)
    y = bd.bdgdn_quant_matmul(qx, sx, qw, sw, out_dtype=F).double()
    x, w, sx, sw = x.double(), w.double(), sx.double(), sw.double()
    bound = x.abs().sum(1)[:, None] * sw / 2 + w.abs().sum(1) * sx[:, None] / 2 + k * sx[:, None] * sw / 4
    assert ((y - x @ w.T).abs() <= bound * (1 + 1e-5)).all()
    assert bd.bdgdn_quant_matmul(qx[:0], sx[:0].float(), qw, sw.float()).shape == (0, n)
    assert bd.bdgdn_quant_rows(x[:0].float())[0].shape == (0, 512)
