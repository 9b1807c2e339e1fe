"""The calls around the mixers as they are used: on other streams, captured into graphs and replayed, and
together in serving rounds of a small hybrid model (examples/speculative_decode.py).

Rounds.  As in the rounds' own tests, a layer's roundings to bf16 come to about 1.5 % a layer, 6 % after
four.  Quantised activations add half a step of max / 127 at most, 0.3 steps in the mean square: with a
largest of 256 normal entries near 3 their standard deviations, 0.7 % to each of eight projections (2 %
together); quantised weights are the reference's own.  8 % of the Frobenius norm in all; a greedy token's
processed logit lies within the error of two logits, which the repetition's factor stretches, of the
largest.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle
import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu

REL = 0.08
_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "speculative_decode.py")
_spec = importlib.util.spec_from_file_location("speculative_decode_layer", _path)
sd = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(sd)


# ------------------------------------------------------------------ streams and graphs
def inputs(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)

    R, N, V, D = 3, 4, 1501, 520
    return dict(q=normal(R, N, 6, 64), k=normal(R, N, 2, 64), seq_len=torch.randint(0, 9999, (R,), generator=g, device="cuda").to(torch.int32),
                x=normal(40, D), z=normal(40, D), r=normal(40, D, dtype=torch.float32), dy=normal(40, D),
                w=normal(D, dtype=torch.float32), logits=normal(R, N, V),
                token=torch.randint(0, V, (R, N), generator=g, device="cuda").to(torch.int32),
                history=torch.randint(0, 3, (R, V), generator=g, device="cuda").to(torch.int32),
                rho=torch.full((R,), 1.3, device="cuda"), weights=normal(600, D))


def calls(s, turns, stream=None):
    """One of each, fed into each other where they are in a program."""
    q, k = bd.bdgdn_rope(s["q"], turns, s["k"], seq_len=s["seq_len"], stream=stream)
    kw = dict(z=s["z"], w_post=s["w"], w_pre=s["w"], layer_scale=s["w"], post=True, pre=True, stream=stream)
    y, new = bd.bdgdn_norm_fwd(s["x"], r=s["r"], **kw)
    grads = bd.bdgdn_norm_bwd(s["x"], s["dy"], r_out=new, dr_out=new, **kw)
    qx, sx = bd.bdgdn_quant_rows(y, stream=stream)
    qw, sw = bd.bdgdn_quant_rows(s["weights"], stream=stream)
    few = bd.bdgdn_quant_matmul(qx[:5], sx[:5], qw, sw, stream=stream)
    many = bd.bdgdn_quant_matmul(qx, sx, qw, sw, stream=stream)
    bd.bdgdn_history_add(s["history"], s["token"], stream=stream)
    out = bd.bdgdn_logits(s["logits"], token=s["token"], history=s["history"], repetition=s["rho"], stream=stream)
    return [q, k, y, new, *grads, qx, sx, few, many, out, s["history"]]


def copy(s):
    return {k: v.clone() for k, v in s.items()}


def same(a, b):
    return all((x is None) == (y is None) and (x is None or torch.equal(x, y)) for x, y in zip(a, b))


def test_on_another_stream():
    turns, _ = bd.make_rope_turns(64)
    s = inputs(1)
    want = calls(copy(s), turns)
    given, own = copy(s), copy(s)
    torch.cuda.synchronize()
    stream, busy = torch.cuda.Stream(), torch.empty(1 << 28, device="cuda")
    for _ in range(8):
        busy.fill_(1.0)        # the current stream has work before it
    got = calls(given, turns, stream)
    with torch.cuda.stream(stream):
        again = calls(own, turns)
    stream.synchronize()
    assert same(got, want) and same(again, want)
    torch.cuda.synchronize()


def test_two_streams_at_once():
    turns, _ = bd.make_rope_turns(64)
    sets = [inputs(k) for k in range(2)]
    want = [calls(copy(s), turns) for s in sets]
    for _ in range(5):
        now = [copy(s) for s in sets]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in sets]
        got = [calls(s, turns, st) for s, st in zip(now, streams)]
        torch.cuda.synchronize()
        assert all(same(g, w) for g, w in zip(got, want))


def test_captured_and_replayed():
    turns, _ = bd.make_rope_turns(64)
    held = [copy(inputs(k)) for k in (10, 11)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for s in held:
            calls(copy(s), turns)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in held:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(calls(s, turns))
        graphs.append(graph)
    for turn in range(4):   # two graphs in turn, other inputs each time, eager work in between
        for s, graph, out in zip(held, graphs, outs):
            fresh = inputs(20 + turn)
            for k in s:
                s[k].copy_(fresh[k])
            graph.replay()
            want = calls(fresh, turns)
            torch.cuda.synchronize()
            assert same(out, want), turn


def test_tensors_the_calls_refuse():
    turns, _ = bd.make_rope_turns(64)
    q = torch.zeros(2, 3, 4, 64, device="cuda")
    x = torch.zeros(4, 32, device="cuda")
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for call, match in (
            (lambda: bd.bdgdn_rope(q[0], turns), "q must be"), (lambda: bd.bdgdn_rope(q, turns, q.half()), "q's type"),
            (lambda: bd.bdgdn_rope(q, turns, pos=ints(1, 2)), "pos must have 6"), (lambda: bd.bdgdn_rope(q, turns.float()), "turns must be"),
            (lambda: bd.bdgdn_rope(q, turns, layout="other"), "unknown layout"), (lambda: bd.bdgdn_rope(q, turns, k_out=q), "without k"),
            (lambda: bd.bdgdn_rope(q, turns, q_out=q.bfloat16()), "q_out must be"), (lambda: bd.bdgdn_rope(q.transpose(2, 3), turns), "contiguous"),
            (lambda: bd.bdgdn_rope(q.cpu(), turns), "device tensor"),
            (lambda: bd.bdgdn_norm_fwd(x, z=x[:2]), "z must be"), (lambda: bd.bdgdn_norm_fwd(x, w_pre=x[0, :8], pre=True), "w_pre must have"),
            (lambda: bd.bdgdn_norm_fwd(x[0]), "x must be"), (lambda: bd.bdgdn_norm_fwd(x, act="gelu"), "unknown act"),
            (lambda: bd.bdgdn_norm_fwd(x.t()), "contiguous"), (lambda: bd.bdgdn_norm_fwd(x, z=x, out_dtype=torch.bfloat16), "type of z"),
            (lambda: bd.bdgdn_norm_bwd(x, x, dw_post=x[0], post=True), "without w_post"), (lambda: bd.bdgdn_norm_bwd(x, x[:1]), "dy must be"),
            (lambda: bd.bdgdn_logits(x), "must be \\[R, N, V\\]"), (lambda: bd.bdgdn_logits(x[None], history=x.int()[:, :8]), "history must be"),
            (lambda: bd.bdgdn_logits(x[None], history=x), "history must be torch.int32"), (lambda: bd.bdgdn_logits(x[None], bias=x), "bias_token and bias"),
            (lambda: bd.bdgdn_logits(x[None], allow=ints(1)[None, None][:, :, :0]), "allow must be"), (lambda: bd.bdgdn_logits(x[None], out=x[None], out_dtype=torch.bfloat16), "out is of"),
            (lambda: bd.bdgdn_history_add(x, ints(1)[None]), "history must be"), (lambda: bd.bdgdn_history_add(x.int(), ints(1)), "token must be"),
            (lambda: bd.bdgdn_quant_rows(x[0]), "x must be"), (lambda: bd.bdgdn_quant_rows(x.t()), "contiguous"),
            (lambda: bd.bdgdn_quant_matmul(x, x[0], x, x[0]), "must be torch.int8"),
            (lambda: bd.bdgdn_quant_matmul(x.to(torch.int8), x[:, 0], x[:, :16].to(torch.int8), x[:, 0]), "a and w must be")):
        with pytest.raises(ValueError, match=match):
            call()
    for call in (lambda: bd.bdgdn_rope(q, turns, q_out=torch.zeros(1, 3, 4, 64, device="cuda").expand(2, 3, 4, 64)),
                 lambda: bd.bdgdn_rope(q.half(), turns), lambda: bd.bdgdn_rope(q[..., :32], turns),
                 lambda: bd.bdgdn_norm_fwd(x, r_out=torch.zeros(1, 32, device="cuda").expand(4, 32)),
                 lambda: bd.bdgdn_norm_fwd(x.bfloat16(), out_dtype=torch.float32), lambda: bd.bdgdn_norm_bwd(x, None),
                 lambda: bd.bdgdn_logits(x[None].half()), lambda: bd.bdgdn_logits(x[None], mask=torch.zeros(1, 4, dtype=torch.int64, device="cuda")),
                 lambda: bd.bdgdn_logits(torch.zeros(1, 65, 8, device="cuda")),
                 lambda: bd.bdgdn_quant_matmul(x.to(torch.int8), x[:, 0].contiguous(), x.to(torch.int8), x[:, 0].contiguous())):
        with pytest.raises(bd.BdgdnError):
            call()


def test_offsets_beyond_32_bits():
    """The last rows of tensors of more than 2^32 bytes, as calls of their own give them."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)

    turns, _ = bd.make_rope_turns(64)
    q = normal(1, 9000, 2000, 128)
    out = bd.bdgdn_rope(q, turns)
    pos = torch.tensor([[8998, 8999]], dtype=torch.int32, device="cuda")
    assert q.numel() > 2 ** 31 and torch.equal(bd.bdgdn_rope(q[:, -2:], turns, pos=pos), out[:, -2:])
    del q, out
    x, w = normal(300000, 8000), torch.ones(8000, device="cuda")
    kw = dict(w_post=w, post=True)
    y, _ = bd.bdgdn_norm_fwd(x, **kw)
    assert x.numel() > 2 ** 31 and torch.equal(bd.bdgdn_norm_fwd(x[-3:], **kw)[0], y[-3:])
    dx = bd.bdgdn_norm_bwd(x, y, **kw)[0]
    assert torch.equal(bd.bdgdn_norm_bwd(x[-3:], y[-3:], **kw)[0], dx[-3:])
    del y, dx
    a, sa = bd.bdgdn_quant_rows(x)
    few, few_s = bd.bdgdn_quant_rows(x[-300:])
    assert a.numel() > 2 ** 31 and torch.equal(a[-300:], few) and torch.equal(sa[-300:], few_s)
    wide = bd.bdgdn_quant_matmul(few, few_s, a, sa)            # [300, 300000]
    tall = bd.bdgdn_quant_matmul(a, sa, a[:8000], sa[:8000])   # [300000, 8000]
    assert tall.numel() > 2 ** 31
    assert torch.equal(wide[:, -300:], bd.bdgdn_quant_matmul(few, few_s, few, few_s))
    assert torch.equal(tall[-300:], bd.bdgdn_quant_matmul(few, few_s, a[:8000], sa[:8000]))
    del a, x, wide, tall
    R, N, V = 40, 60, 1000003
    logits, history = normal(R, N, V), torch.zeros(2200, V, dtype=torch.int32, device="cuda")
    assert logits.numel() > 2 ** 31 and history.numel() > 2 ** 31
    token = torch.full((R, N), V - 1, dtype=torch.int32, device="cuda")
    slot = torch.arange(2160, 2200, dtype=torch.int32, device="cuda")
    bd.bdgdn_history_add(history, token, slot=slot)
    assert (history[2160:, -1] == N).all() and not history[:2160].any() and not history[:, :-1].any()
    kw = dict(frequency=torch.full((R,), 0.01, device="cuda"))
    out = bd.bdgdn_logits(logits, token=token, history=history, slot=slot, **kw)
    last = bd.bdgdn_logits(logits[-1:], token=token[-1:], history=history[-1:], frequency=kw["frequency"][:1])
    assert torch.equal(out[-1], last[0]) and torch.equal(out[-1, -1, :-1], logits[-1, -1, :-1])
    assert float(out[-1, -1, -1]) != float(logits[-1, -1, -1])


# ------------------------------------------------------------------ rounds of a model
def _np(t):
    return t.double().cpu().numpy()


def _norm(x):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)


def turned(x, positions, base):
    """Rotary positions of [T, heads, d], halves, as complex numbers."""
    d = x.shape[-1]
    w = base ** (-2 * np.arange(d // 2) / d)
    c = (x[..., :d // 2] + 1j * x[..., d // 2:]) * np.exp(1j * positions[:, None, None] * w)
    return np.concatenate([c.real, c.imag], -1)


def reference(model, tokens, base):
    """Logits [T, V], and for each layer the final state or the cached (k, v), in 64 bits."""
    x = _np(model.embed)[tokens]
    T, kept = len(tokens), []
    weights = [[_np(w) for w in ws] for ws in (model.w_in, model.w_out)]
    if model.eight_bit:
        weights = [[(_np(q) * _np(s)[:, None])[:, :w.shape[0]].T for (q, s), w in zip(qs, ws)]
                   for qs, ws in zip(model.eight_bit, weights)]
    for kind, w_in, w_out in zip(model.layers, *weights):
        y = _norm(x) @ w_in
        if kind == "g":
            H, d = sd.GDN_HEADS, sd.GDN_DIM
            q, k, v = (y[:, i * H * d:(i + 1) * H * d].reshape(1, T, H, d) for i in range(3))
            q, k = (t / np.linalg.norm(t, axis=-1, keepdims=True) for t in (q, k))
            g, beta = y[None, :, 3 * H * d:3 * H * d + H], y[None, :, 3 * H * d + H:]
            pool, o = oracle.commit(np.zeros((1, H, d, d)), q, k, v, -np.logaddexp(0, g), 1 / (1 + np.exp(-beta)), scale=d ** -0.5)
            kept.append(pool[0])
        else:
            y = y.reshape(T, -1, sd.DIM)
            q, k, v = y[:, :sd.HEADS], y[:, sd.HEADS:sd.HEADS + sd.KV_HEADS], y[:, sd.HEADS + sd.KV_HEADS:]
            q, k = turned(q, np.arange(T), base), turned(k, np.arange(T), base)
            s = np.einsum("thd,shd->hts", q, k.repeat(sd.HEADS // sd.KV_HEADS, 1)) * sd.DIM ** -0.5
            s = np.where(np.tril(np.ones((T, T), bool)), s, -np.inf)
            p = np.exp(s - s.max(-1, keepdims=True))
            o = np.einsum("hts,shd->thd", p / p.sum(-1, keepdims=True), v.repeat(sd.HEADS // sd.KV_HEADS, 1))
            kept.append((k, v))
        x = x + o.reshape(T, -1) @ w_out
    return _norm(x) @ _np(model.out), kept


def near(got, want, what):
    err = np.linalg.norm(_np(got) - want) / np.linalg.norm(want)
    assert err < REL, f"{what}: {err:.3f}"


def check(model, sequences, T, base, penalties):
    rho, presence, frequency = penalties
    for slot, seq in enumerate(sequences):
        assert int(model.tables.seq_len[slot]) == int(model.taken[slot]) == len(seq) - 1
        logits, kept = reference(model, np.array(seq[:-1]), base)
        a = 0
        for i, kind in enumerate(model.layers):
            if kind == "g":
                near(model.states[i][slot], kept[i], f"state of layer {i}, sequence {slot}")
                continue
            n, pages = len(seq) - 1, model.tables.page_table[slot, :-(-(len(seq) - 1) // model.page)].long()
            for j in range(2):
                near(model.pools[a + j][pages].reshape(-1, sd.KV_HEADS, sd.DIM)[:n], kept[i][j], f"cache of layer {i}, sequence {slot}")
            a += 2
        # every token behind the prompt is the best of the logits as they stood, with what came before it
        history = np.zeros(model.vocab, int)
        prompt = np.zeros(model.vocab, bool)
        prompt[seq[:T - 1]] = True
        for t in range(T - 1, len(seq) - 1):
            history[seq[t]] += 1
            seen = prompt | (history > 0)
            row = np.where(seen, np.where(logits[t] > 0, logits[t] / rho, logits[t] * rho), logits[t])
            row = row - presence * (history > 0) - frequency * history
            assert row.max() - row[seq[t + 1]] < REL * 2 ** 0.5 * 4 * rho * logits.std(), (slot, t)
        got = model.history[slot].cpu().numpy()
        assert (got % (1 << 30) == history).all() and ((got >> 30) == prompt).all()


@pytest.mark.parametrize("eight_bit", [False, True])
def test_chains_with_positions_penalties_and_integers(eight_bit):
    torch.manual_seed(21)
    R, ways, T, rounds, drafts, penalties, base = 3, 2, 45, 10, 5, (1.2, 0.3, 0.1), 500.0
    model = sd.Decoder("gaga", slots=R * ways, max_len=T + rounds * (drafts + 1), pages=96, rotary=base, eight_bit=eight_bit,
                       penalties=penalties)
    slot = torch.arange(R * ways, dtype=torch.int32, device="cuda")
    prompt = torch.randint(model.vocab, (R, T), dtype=torch.int32, generator=torch.Generator().manual_seed(3)).cuda()
    anchor, status = model.prefill(prompt, slot[:R])
    assert not status.any() and not model.fork(slot[:R].clone(), slot[R:].clone()).any()
    anchor = anchor.repeat(ways)
    sequences = [prompt[i % R].tolist() for i in range(R * ways)]
    for _ in range(rounds):
        token, n_accept, anchor, status = model.round(anchor, slot, drafts, 0.0)
        assert not status.any()
        for s, (t, n, nxt) in enumerate(zip(token.tolist(), n_accept.tolist(), anchor.tolist())):
            sequences[s] += t[1:1 + n] + [nxt]
    check(model, sequences, T, base, penalties)
    model.finish(slot)
    assert not model.history.any() and not model.taken.any()


def test_trees_with_positions_and_penalties():
    torch.manual_seed(22)
    R, T, rounds, penalties, base = 4, 19, 8, (1.1, 0.2, 0.3), 10000.0
    model = sd.Decoder("aa", slots=R, max_len=T + rounds * 4, rotary=base, penalties=penalties)
    slot = torch.arange(R, dtype=torch.int32, device="cuda")
    prompt = torch.randint(model.vocab, (R, T), dtype=torch.int32, generator=torch.Generator().manual_seed(4)).cuda()
    anchor, _ = model.prefill(prompt, slot)
    sequences = prompt.tolist()
    for _ in range(rounds):
        token, n_accept, anchor, status = model.tree_round(anchor, slot, [3, 2, 1], 0.0)
        assert not status.any()
        for s, (t, n, nxt) in enumerate(zip(token.tolist(), n_accept.tolist(), anchor.tolist())):
            sequences[s] += t[1:1 + n] + [nxt]
    check(model, sequences, T, base, penalties)


def test_a_window_keeps_positions():
    """After a window has shortened the caches, new tokens go on from the positions they have."""
    torch.manual_seed(23)
    R, T = 2, 40
    model = sd.Decoder("a", slots=R, max_len=96, pages=40, rotary=10000.0)
    slot = torch.arange(R, dtype=torch.int32, device="cuda")
    prompt = torch.randint(model.vocab, (R, T), dtype=torch.int32, generator=torch.Generator().manual_seed(5)).cuda()
    anchor, _ = model.prefill(prompt, slot)
    assert not model.shorten(slot, 4, 20).any() and (model.taken == T - 1).all() and (model.tables.seq_len == 24).all()
    _, rows, _ = model.forward(anchor[:, None], slot)
    for r in range(R):
        x = _norm(_np(model.embed)[int(anchor[r])][None]) @ _np(model.w_in[0])
        k = turned(x.reshape(1, -1, sd.DIM)[:, sd.HEADS:sd.HEADS + sd.KV_HEADS], np.array([T - 1]), 10000.0)
        near(rows[0][r], k, f"key of sequence {r}")


def test_the_command_runs(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["speculative_decode.py", "--prompts", "2", "--ways", "2", "--rounds", "3", "--length", "20", "--rotary",
                                     "10000", "--eight-bit", "--repetition", "1.2", "--frequency", "0.1"])
    sd.main()
    assert "tokens a sequence and round" in capsys.readouterr().out
