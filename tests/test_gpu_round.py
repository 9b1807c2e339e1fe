"""Whole serving rounds of a small hybrid model (examples/speculative_decode.py), whose tokens,
caches and states are compared with the same model run over the emitted sequences in fp64.

Tolerances.  A layer's inputs, projections, weights and outputs are rounded to bf16 (a relative
2^-8 at most, 2^-8 / sqrt 3 in the mean square) some ten times, and a softmax passes on the
errors of its scores (a few per cent of a score of size 3): about 1.5 % a layer, 6 % after
four.  A cache row or a state that belongs to another token differs by 100 %.  Caches and states: 8 % of the
Frobenius norm.  A greedy token's logit lies within the error of two logits of the largest one:
0.08 x sqrt 2 x 4 standard deviations.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle
import paper_2606_01774_amd as bd
from paper_2606_01774_amd import rounds

pytestmark = pytest.mark.gpu

REL = 0.08
_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "speculative_decode.py")
_spec = importlib.util.spec_from_file_location("speculative_decode", _path)
sd = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(sd)


def _norm(x):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)


def _np(t):
    return t.double().cpu().numpy()


def reference(model, tokens):
    """Logits [T, V], and for each layer the final state or the cached (k, v), in fp64."""
    x = _np(model.embed)[tokens]
    T, kept = len(tokens), []
    for kind, w_in, w_out in zip(model.layers, model.w_in, model.w_out):
        y = _norm(x) @ _np(w_in)
        if kind == "g":
            H, d = sd.GDN_HEADS, sd.GDN_DIM
            q, k, v = (y[:, i * H * d:(i + 1) * H * d].reshape(1, T, H, d) for i in range(3))
            q, k = (t / np.linalg.norm(t, axis=-1, keepdims=True) for t in (q, k))
            g, beta = y[None, :, 3 * H * d:3 * H * d + H], y[None, :, 3 * H * d + H:]
            pool, o = oracle.commit(np.zeros((1, H, d, d)), q, k, v, -np.logaddexp(0, g), 1 / (1 + np.exp(-beta)),
                                    scale=d ** -0.5)
            kept.append(pool[0])
        else:
            y = y.reshape(T, -1, sd.DIM)
            q, k, v = y[:, :sd.HEADS], y[:, sd.HEADS:sd.HEADS + sd.KV_HEADS], y[:, sd.HEADS + sd.KV_HEADS:]
            G = sd.HEADS // sd.KV_HEADS
            s = np.einsum("thd,shd->hts", q, k.repeat(G, 1)) * sd.DIM ** -0.5
            s = np.where(np.tril(np.ones((T, T), bool)), s, -np.inf)
            p = np.exp(s - s.max(-1, keepdims=True))
            o = np.einsum("hts,shd->thd", p / p.sum(-1, keepdims=True), v.repeat(G, 1))
            kept.append((k, v))
        x = x + o.reshape(T, -1) @ _np(w_out)
    return _norm(x) @ _np(model.out), kept


def cached(model, pool, slot):
    n = int(model.tables.seq_len[slot])
    pages = model.tables.page_table[slot, :-(-n // model.page)].long()
    return model.pools[pool][pages].reshape(-1, sd.KV_HEADS, sd.DIM)[:n]


def _near(got, want, what):
    err = np.linalg.norm(_np(got) - want) / np.linalg.norm(want)
    assert err < REL, f"{what}: {err:.3f}"


def check(model, sequences, new_from, greedy):
    """Sequences: lists of tokens by slot, of which all but the last have gone through the model."""
    for slot, seq in enumerate(sequences):
        assert int(model.tables.seq_len[slot]) == len(seq) - 1
        logits, kept = reference(model, np.array(seq[:-1]))
        a = 0
        for i, kind in enumerate(model.layers):
            if kind == "g":
                _near(model.states[i][slot], kept[i], f"state of layer {i}, sequence {slot}")
            else:
                for j in range(2):
                    _near(cached(model, a + j, slot), kept[i][j], f"cache of layer {i}, sequence {slot}")
                a += 2
        if greedy:
            at = np.arange(new_from - 1, len(seq) - 1)
            gap = logits[at].max(-1) - logits[at, np.array(seq)[new_from:]]
            assert gap.max() < REL * 2 ** 0.5 * 4 * logits.std(), gap.max()


def _prompts(R, T, vocab):
    return torch.randint(vocab, (R, T), dtype=torch.int32, generator=torch.Generator().manual_seed(3)).cuda()


@pytest.mark.parametrize("temperature", [0.0, 1.0])
@pytest.mark.parametrize("drafts", [1, 6])
def test_chains_through_a_hybrid_model(temperature, drafts):
    torch.manual_seed(11)
    R, ways, T, rounds = 3, 2, 45, 12
    model = sd.Decoder("gaga", slots=R * ways, max_len=T + rounds * (drafts + 1), pages=96)
    slot = torch.arange(R * ways, dtype=torch.int32, device="cuda")
    prompt = _prompts(R, T, model.vocab)
    anchor, status = model.prefill(prompt, slot[:R])
    assert not status.any() and not model.fork(slot[:R].clone(), slot[R:].clone()).any()
    anchor = anchor.repeat(ways)
    sequences = [prompt[i % R].tolist() for i in range(R * ways)]
    accepted = 0
    for _ in range(rounds):
        token, n_accept, anchor, status = model.round(anchor, slot, drafts, temperature)
        assert not status.any()
        for s, (t, n, nxt) in enumerate(zip(token.tolist(), n_accept.tolist(), anchor.tolist())):
            sequences[s] += t[1:1 + n] + [nxt]
            accepted += n
    assert 0 < accepted < R * ways * rounds * drafts   # both outcomes occur
    check(model, sequences, T, temperature == 0)
    model.finish(slot)
    assert not model.tables.refcount.any() and not model.tables.seq_len.any()


def test_trees_through_an_attention_model():
    torch.manual_seed(12)
    R, T, rounds = 4, 19, 10
    model = sd.Decoder("aa", slots=R, max_len=T + rounds * 4)
    slot = torch.arange(R, dtype=torch.int32, device="cuda")
    prompt = _prompts(R, T, model.vocab)
    anchor, _ = model.prefill(prompt, slot)
    sequences, accepted = prompt.tolist(), 0
    for _ in range(rounds):
        token, n_accept, anchor, status = model.tree_round(anchor, slot, [3, 2, 1], 0.0)
        assert not status.any()
        for s, (t, n, nxt) in enumerate(zip(token.tolist(), n_accept.tolist(), anchor.tolist())):
            sequences[s] += t[1:1 + n] + [nxt]
            accepted += n
    assert 0 < accepted <= R * rounds * 3
    check(model, sequences, T, True)


def test_a_window_keeps_the_rows_it_keeps():
    torch.manual_seed(13)
    R, T = 3, 70
    model = sd.Decoder("ga", slots=R, max_len=96, pages=40)
    slot = torch.arange(R, dtype=torch.int32, device="cuda")
    anchor, _ = model.prefill(_prompts(R, T, model.vocab), slot)
    before = [[cached(model, p, s) for p in range(2)] for s in range(R)]
    assert not model.shorten(slot, 4, 30).any()
    for s in range(R):
        for p in range(2):
            assert torch.equal(cached(model, p, s), torch.cat([before[s][p][:4], before[s][p][-30:]]))
    *_, status = model.round(anchor, slot)
    assert not status.any() and not model.shorten(slot, 4, 40).any()   # (nothing to drop)
    assert (model.tables.seq_len >= 35).all()


@pytest.mark.parametrize("argv", [["--prompts", "2", "--ways", "2", "--rounds", "12", "--window", "48"],
                                  ["--layers", "aa", "--tree", "2,2", "--rounds", "6", "--temperature", "0"]])
def test_the_command(argv, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["speculative_decode.py", *argv])
    sd.main()
    assert "tokens a sequence and round" in capsys.readouterr().out


def test_trees_need_attention_layers():
    model = sd.Decoder("ga", slots=1, max_len=16)
    with pytest.raises(ValueError, match="chain"):
        model.tree_round(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"),
                         [2])


def _calls():
    """Calls with temporaries of their own, on tensors made beforehand: (name, call(stream) ->
    results, its workspace's bytes)."""
    gen = torch.Generator(device="cuda").manual_seed(5)

    def rand(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    R, N, V = 4, 8, 4096
    model = sd.Decoder("a", slots=R, max_len=4096)
    slot = torch.arange(R, dtype=torch.int32, device="cuda")
    prompt = _prompts(R, 1500, model.vocab)
    model.prefill(prompt, slot)
    q, k = rand(R, N, sd.HEADS, sd.DIM), rand(R, N, sd.KV_HEADS, sd.DIM)
    t = model.tables
    cache = rounds.CacheDesc(t.refcount.numel(), model.page, R, t.page_table.shape[1], sd.KV_HEADS, sd.DIM,
                             bd.BDGDN_BF16, *model.pools[0].stride()[:3])
    attn = rounds.AttnDesc(R, N, sd.HEADS, sd.KV_HEADS, sd.DIM, 0.125, bd.BDGDN_BF16, bd.BDGDN_BF16,
                           bd.BDGDN_MASK_CAUSAL)
    target, token = rand(R, N, V, dtype=torch.float32), torch.zeros(R, N, dtype=torch.int32, device="cuda")
    u, noise = torch.full((R, N), 0.5, device="cuda"), torch.empty(R, V, device="cuda").exponential_(generator=gen)
    none = torch.zeros(R, dtype=torch.int32, device="cuda")
    return [
        ("tree_attn", lambda s: bd.bdgdn_tree_attn(q, k, k, *model.pools, t.page_table, t.seq_len, mask="causal", stream=s,
                                                   scale=0.125)[:1], bd.bdgdn_tree_attn_workspace(attn, cache)),
        ("verify", lambda s: bd.bdgdn_verify(target, token, u, noise, stream=s),
         bd.bdgdn_verify_workspace(rounds.VerifyDesc(R, N, V, bd.BDGDN_F32, N * V, V, 0, 0, V))),
        ("append", lambda s: (bd.bdgdn_cache_append(t, model.pools, [k, k], slot, none, stream=s),),
         bd.bdgdn_cache_workspace(cache, R, N)),
    ]


@pytest.mark.parametrize("which", range(3))
def test_temporaries_belong_to_the_stream_of_the_call(which):
    """A call on a stream that is busy for a while must not leave its memory to the stream that
    the caller goes on with."""
    name, call, need = _calls()[which]
    want = [x.clone() for x in call(None)]
    side, big = torch.cuda.Stream(), torch.zeros(1 << 28, device="cuda")
    call(side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(60):
            big.add_(1)
    got = call(side)
    taken = [torch.full((need,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool((x == 7).all()) for x in taken), name
    assert all(torch.equal(g, w) for g, w in zip(got, want)), name


@pytest.mark.parametrize("argv", [["--prompts", "2", "--ways", "2", "--rounds", "1"],
                                  ["--layers", "aa", "--tree", "2,2", "--rounds", "1", "--prompts", "1", "--ways", "1"]])
def test_the_command_for_one_round(argv, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["speculative_decode.py", *argv])
    sd.main()
    assert "tokens a sequence and round" in capsys.readouterr().out
