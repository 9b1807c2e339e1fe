"""Arguments that the entry points around a hybrid layer's mixers refuse before anything is launched (no GPU is
touched), beside those of test_layer_abi."""
import pytest
import torch

import paper_2606_01774_amd as bd
from paper_2606_01774_amd import layers
from test_layer_abi import FAKE, INV, WS, _call_logits, _call_rope, _logits, _rope


@pytest.mark.parametrize("name", ["pos", "len", "slot", "count"])
def test_rope_rejects_arrays_off_their_words(name):
    for off in (1, 2, 3):
        assert _call_rope(_rope(), **{name: FAKE + off}) == INV, off


@pytest.mark.parametrize("name", ["slot", "token", "count", "rho", "presence", "frequency", "bias_token", "bias"])
def test_logits_reject_arrays_off_their_words(name):
    for off in (1, 2, 3):
        assert _call_logits(_logits(), **{name: FAKE + off}) == INV, off


@pytest.mark.parametrize("name", ["history", "slot", "token", "path", "count"])
def test_history_add_rejects_arrays_off_their_words(name):
    ok = dict(R=2, N=3, V=10, slots=4, stride=10, history=FAKE, slot=FAKE, token=FAKE, path=FAKE, count=FAKE, prompt=0)
    for off in (1, 2, 3):
        assert bd.load_library().bdgdn_history_add(*dict(ok, **{name: FAKE + off}).values(), None) == INV, off


@pytest.mark.parametrize("m,n,k", [(70, 40, 130944), (200, 150, 16384), (70, 75, 16384), (130, 129, 8192)])
def test_quant_matmul_asks_for_the_workspace_of_its_parts(m, n, k):
    desc = layers.QuantMatmulDesc(m, n, k, bd.BDGDN_F32, k, k, n)
    need = bd.bdgdn_quant_matmul_workspace(desc)
    assert need > 0 and need % (m * n * 4) == 0      # whole sums, at least two of them
    assert need >= 2 * m * n * 4

    def call(ws, size):
        return bd.load_library().bdgdn_quant_matmul(desc, FAKE, FAKE, FAKE, FAKE, None, FAKE, ws, size, None)

    assert call(FAKE, need - 1) == WS and call(FAKE, 0) == WS and call(None, need) == WS and call(None, 1 << 40) == WS
    assert call(FAKE + 128, need) == INV


@pytest.mark.parametrize("m,n,k", [(1, 512, 2048), (16, 40, 130944), (64, 512, 2048), (500, 512, 2048), (4096, 4096, 1024), (0, 40, 130944)])
def test_quant_matmul_needs_no_workspace_for_one_part(m, n, k):
    assert bd.bdgdn_quant_matmul_workspace(layers.QuantMatmulDesc(m, n, k, bd.BDGDN_F32, k, k, n)) == 0


# ------------------------------------------------------------------ the binding
class Here(torch.Tensor):
    """Passes for a tensor on the device that the call runs on."""
    is_cuda = True

    def get_device(self):
        return 0


def here(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Here)


def test_the_binding_refuses_what_is_missing(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(layers, "_raw_stream", lambda at: 0)
    q, x, ints = here(1, 2, 3, 8), here(2, 128), here(2, 128, dtype=torch.int32)
    a, s = here(2, 128, dtype=torch.int8), here(2)
    for call, name in (
            (lambda: bd.bdgdn_rope(None, here(4, dtype=torch.int64)), "q"), (lambda: bd.bdgdn_rope(q, None), "turns"),
            (lambda: bd.bdgdn_norm_fwd(None), "x"), (lambda: bd.bdgdn_norm_bwd(None, x), "x"),
            (lambda: bd.bdgdn_logits(None), "logits"), (lambda: bd.bdgdn_history_add(None, ints), "history"),
            (lambda: bd.bdgdn_history_add(ints, None), "token"), (lambda: bd.bdgdn_quant_rows(None), "x"),
            (lambda: bd.bdgdn_quant_matmul(None, s, a, s), "a"), (lambda: bd.bdgdn_quant_matmul(a, None, a, s), "a_scale"),
            (lambda: bd.bdgdn_quant_matmul(a, s, None, s), "w"), (lambda: bd.bdgdn_quant_matmul(a, s, a, None), "w_scale")):
        with pytest.raises(ValueError, match=f"^{name} must be a device tensor"):
            call()
