"""C calls of the norms that leave results out: one does not depend on which others are wanted."""
import ctypes

import pytest
import torch

import paper_2606_01774_amd as bd
from paper_2606_01774_amd import layers

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


def normal(seed, *shape, dtype=F):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


SIZES = [(9, 64), (9, 100), (300, 520), (5, 4096), (300, 8192), (5, 9000)]   # one, two and four chunks to a lane


def desc(x, rt, rows, d):
    return layers._norm_plan((rows, d), (None,) * 10, (x.dtype, rt, B), True, True, 1, 0.75, 1e-6)[0]


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("rows,d", SIZES)
def test_forward_results_one_by_one(rows, d):
    x, z, r, w = normal(1, rows, d, dtype=B), normal(2, rows, d, dtype=B), normal(3, rows, d), normal(4, d)
    y, new = bd.bdgdn_norm_fwd(x, z=z, r=r, w_post=w, w_pre=w, layer_scale=w, post=True, pre=True, scale=0.75)
    lib, plan = bd.load_library(), desc(x, F, rows, d)
    for want_y, want_r in ((False, True), (True, False), (True, True)):
        yy, rr = torch.full_like(y, 5.0), torch.full_like(new, 5.0)
        st = lib.bdgdn_norm_fwd(plan, x.data_ptr(), z.data_ptr(), r.data_ptr(), w.data_ptr(), w.data_ptr(), w.data_ptr(),
                                rr.data_ptr() if want_r else None, yy.data_ptr() if want_y else None, stream())
        assert st == bd.BDGDN_OK
        assert torch.equal(yy, y) if want_y else (yy == 5).all()
        assert torch.equal(rr, new) if want_r else (rr == 5).all()


@pytest.mark.parametrize("rows,d", SIZES)
def test_gradients_one_by_one(rows, d):
    x, z, new, dr, w = (normal(1, rows, d, dtype=B), normal(2, rows, d, dtype=B), normal(3, rows, d), normal(5, rows, d), normal(4, d))
    dy = normal(6, rows, d, dtype=B)
    want = bd.bdgdn_norm_bwd(x, dy, z=z, r_out=new, dr_out=dr, w_post=w, w_pre=w, layer_scale=w, post=True, pre=True, scale=0.75)
    lib, plan = bd.load_library(), desc(x, F, rows, d)
    size = lib.bdgdn_norm_bwd_workspace(ctypes.byref(plan))
    for some in ((0,), (1,), (2,), (3,), (4,), (5,), (1, 2), (0, 4), (1, 3, 5), (0, 1, 2)):
        outs = [torch.full_like(t, 5.0) for t in want]
        room = torch.full((size + 256,), 7, dtype=torch.uint8, device="cuda")
        sums = any(i > 2 for i in some)
        st = lib.bdgdn_norm_bwd(plan, x.data_ptr(), z.data_ptr(), new.data_ptr(), w.data_ptr(), w.data_ptr(), w.data_ptr(),
                                dy.data_ptr(), dr.data_ptr(), *(t.data_ptr() if i in some else None for i, t in enumerate(outs)),
                                room.data_ptr() if sums else None, size if sums else 0, stream())
        assert st == bd.BDGDN_OK
        for i, (got, t) in enumerate(zip(outs, want)):
            assert torch.equal(got, t) if i in some else (got == 5).all(), (some, i)
        assert (room[size:] == 7).all()
