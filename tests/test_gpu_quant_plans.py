"""bdgdn_quant_matmul through each of its cuts: squares of 256 and 128 and 64 on a side with ragged
edges, and parts of a long k that are joined, in both types, with and without a bias, into rows of their
own and parts of longer rows, with a workspace of exactly the size that is asked for.  Tolerances:
test_gpu_quant."""
import ctypes

import pytest
import torch

import paper_2606_01774_amd as bd
from paper_2606_01774_amd import layers
from test_gpu_quant import B, F, make, near, product

pytestmark = pytest.mark.gpu


def into_a_part(m, n, dtype, left):
    """A result's place between guard columns, `left` of them in front."""
    room = torch.full((m, left + n + 7), 3.0, dtype=dtype, device="cuda")
    return room, room[:, left:left + n]


def untouched(room, n, left):
    return bool((room[:, :left] == 3).all() and (room[:, left + n:] == 3).all())


# steps of 128 x rounds of the chip at 0.47, 0.61 and 2.0 us: the least is that of squares of 256 for the first
# four, of 128 for the fifth, of 64 for the last two
SHAPES = [(4095, 4093, 384), (3585, 4350, 384), (4096, 4096, 128), (8191, 2047, 640), (1000, 2051, 512), (130, 1000, 384), (63, 4093, 256)]


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_squares_with_ragged_edges(m, n, k, dtype):
    a, sa, w, sw, bias = make(m, n, k, m + n, full=True)
    want, size = product(a, sa, w, sw, None)
    y = bd.bdgdn_quant_matmul(a, sa, w, sw, out_dtype=dtype)
    near(y, want, size)
    b = bias.cpu().double()
    for left in (0, 3):
        room, out = into_a_part(m, n, dtype, left)
        bd.bdgdn_quant_matmul(a, sa, w, sw, bias=bias, out=out)
        near(out, want + b, size + b.abs())
        assert untouched(room, n, left)


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("m,n,k", [(200, 150, 16384), (70, 75, 16384), (33, 40, 65536), (130, 129, 8192)])
def test_parts_of_a_long_sum(m, n, k, dtype):
    a, sa, w, sw, bias = make(m, n, k, m + n + k, full=True)
    want, size = product(a, sa, w, sw, bias)
    desc = layers.QuantMatmulDesc(m, n, k, bd.BDGDN_F32 if dtype is F else bd.BDGDN_BF16, k, k, n)
    need = bd.bdgdn_quant_matmul_workspace(desc)
    assert need > 0
    room = torch.full((need + 256,), 0x7f, dtype=torch.uint8, device="cuda")   # (what it holds before does not count)
    near(bd.bdgdn_quant_matmul(a, sa, w, sw, bias=bias, out_dtype=dtype, workspace=room[:need]), want, size)
    assert (room[need:] == 0x7f).all()
    for left in (0, 5):
        wide, out = into_a_part(m, n, dtype, left)
        bd.bdgdn_quant_matmul(a, sa, w, sw, bias=bias, out=out, workspace=room[:need])
        near(out, want, size)
        assert untouched(wide, n, left)
    short = bd.load_library().bdgdn_quant_matmul(ctypes.byref(desc), a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), None,
                                                 out.data_ptr(), room.data_ptr(), need - 1, None)
    assert short == bd.BDGDN_ERR_WORKSPACE
