"""Arguments that the entry points around a hybrid layer's mixers refuse before anything is launched (no GPU is
touched), beside those of test_layer_abi."""

import pytest

import paper_2606_01774_amd as bd
from test_layer_abi import FAKE, INV, _call_logits, _call_rope, _logits, _rope


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
