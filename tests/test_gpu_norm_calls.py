"""bdgdn_norm_bwd for an upstream gradient of the residual alone."""
import pytest
import torch

import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


def normal(seed, *shape, dtype=F):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("rt", [B, F])
@pytest.mark.parametrize("xt", [B, F])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False)])
def test_a_gradient_of_the_residual_alone(post, pre, xt, rt):
    """dy None is dy of zeros, whatever the types of x and the residual."""
    x, new, dr = normal(1, 7, 200, dtype=xt), normal(2, 7, 200, dtype=rt), normal(3, 7, 200, dtype=rt)
    w = normal(4, 200)
    kw = dict(r_out=new, dr_out=dr, w_post=w, w_pre=w, layer_scale=w, post=post, pre=pre, scale=0.5)
    got = bd.bdgdn_norm_bwd(x, None, **kw)
    want = bd.bdgdn_norm_bwd(x, torch.zeros(7, 200, dtype=B, device="cuda"), **kw)
    assert got[0].dtype is xt and got[2].dtype is rt
    for a, b in zip(got, want):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
