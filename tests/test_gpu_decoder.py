"""What examples/speculative_decode.py keeps of a sequence beside its cache.  The reference model and its
tolerances: test_gpu_layer."""
import numpy as np
import pytest
import torch

import paper_2606_01774_amd as bd
from test_gpu_layer import REL, check, reference, sd

pytestmark = pytest.mark.gpu


def prompts(model, R, T, seed=3):
    return torch.randint(model.vocab, (R, T), dtype=torch.int32, generator=torch.Generator().manual_seed(seed)).cuda()


def go_on(sequences, step):
    token, n_accept, anchor, _ = step
    for seq, t, n, nxt in zip(sequences, token.tolist(), n_accept.tolist(), anchor.tolist()):
        seq += t[1:1 + n] + [nxt]
    return anchor


def check_penalties(model, sequences, T, base, penalties):
    """The prompt is the first T tokens, all of them; what comes behind them was generated."""
    rho, presence, frequency = penalties
    for slot, seq in enumerate(sequences):
        logits, _ = reference(model, np.array(seq[:-1]), base)
        history, prompt = np.zeros(model.vocab, int), np.zeros(model.vocab, bool)
        prompt[seq[:T]] = True
        for t in range(T - 1, len(seq) - 1):
            if t >= T:
                history[seq[t]] += 1
            seen = prompt | (history > 0)
            row = np.where(seen, np.where(logits[t] > 0, logits[t] / rho, logits[t] * rho), logits[t])
            row = row - presence * (history > 0) - frequency * history
            assert row.max() - row[seq[t + 1]] < REL * 2 ** 0.5 * 4 * rho * logits.std(), (slot, t)
        got = model.history[slot].cpu().numpy()
        assert (got % (1 << 30) == history).all() and ((got >> 30) == prompt).all()


@pytest.mark.parametrize("argv", [["--layers", "gaga"], ["--layers", "aa", "--tree", "2,2"]])
def test_the_command_penalises_generated_tokens_alone(argv, monkeypatch, capsys):
    """The last token of a prompt, the first anchor, is the prompt's like the others."""
    seen, prefill, finish = {}, sd.Decoder.prefill, sd.Decoder.finish

    def keep_prompt(self, prompt, *args, **kw):
        seen["prompt"] = prompt.cpu()
        return prefill(self, prompt, *args, **kw)

    def keep_history(self, slot):
        seen["history"], seen["taken"] = self.history.cpu(), self.taken.cpu()
        return finish(self, slot)

    monkeypatch.setattr(sd.Decoder, "prefill", keep_prompt)
    monkeypatch.setattr(sd.Decoder, "finish", keep_history)
    monkeypatch.setattr("sys.argv", ["speculative_decode.py", "--prompts", "3", "--ways", "2", "--rounds", "4", "--length", "20",
                                     "--presence", "0.5", *argv])
    sd.main()
    assert "tokens a sequence and round" in capsys.readouterr().out
    prompt, history = seen["prompt"], seen["history"]
    for s in range(6):
        marks = torch.zeros(history.shape[1], dtype=torch.bool)
        marks[prompt[s % 3].long()] = True
        assert torch.equal(history[s] >= bd.BDGDN_HISTORY_PROMPT, marks)
        # every token behind the prompt that the sequence has taken in, once
        assert int((history[s] % bd.BDGDN_HISTORY_PROMPT).sum()) == int(seen["taken"][s]) - prompt.shape[1]


def test_generated_tokens_alone_are_penalised():
    R, ways, T, drafts, penalties, base = 2, 2, 30, 4, (1.2, 1.5, 0.4), 500.0
    model = sd.Decoder("ga", slots=R * ways, max_len=128, rotary=base, penalties=penalties)
    slot = torch.arange(R * ways, dtype=torch.int32, device="cuda")
    prompt = prompts(model, R, T)
    anchor, status = model.prefill(prompt, slot[:R], whole=True)
    assert not status.any() and not model.fork(slot[:R].clone(), slot[R:].clone()).any()
    anchor, sequences = anchor.repeat(ways), [prompt[i % R].tolist() for i in range(R * ways)]
    for _ in range(6):
        anchor = go_on(sequences, model.round(anchor, slot, drafts, 0.0))
    check_penalties(model, sequences, T, base, penalties)


def test_an_anchor_that_was_generated_counts():
    """Without `whole` the first anchor is a token that another program has generated."""
    R, T, penalties, base = 2, 30, (1.2, 1.5, 0.4), 500.0
    model = sd.Decoder("ga", slots=R, max_len=128, rotary=base, penalties=penalties)
    slot = torch.arange(R, dtype=torch.int32, device="cuda")
    prompt = prompts(model, R, T)
    anchor, _ = model.prefill(prompt, slot)
    sequences = prompt.tolist()
    for _ in range(3):
        anchor = go_on(sequences, model.round(anchor, slot, 4, 0.0))
    check(model, sequences, T, base, penalties)


def test_trees_penalise_generated_tokens_alone():
    R, T, penalties, base = 3, 12, (1.1, 1.0, 0.3), 10000.0
    model = sd.Decoder("aa", slots=R, max_len=64, rotary=base, penalties=penalties)
    slot = torch.arange(R, dtype=torch.int32, device="cuda")
    prompt = prompts(model, R, T)
    anchor, _ = model.prefill(prompt, slot, whole=True)
    sequences = prompt.tolist()
    for _ in range(5):
        token, n_accept, nxt, _ = model.tree_round(anchor, slot, [3, 2], 0.0)
        anchor = go_on(sequences, (token, n_accept, nxt, None))
    check_penalties(model, sequences, T, base, penalties)


def held(model, s):
    return [t[s].clone() for t in (model.taken, model.history, model.tables.seq_len, *(x for x in model.states if x is not None))]


def test_a_refused_append_leaves_the_sequence_as_it_was():
    """Five pages of 16: slot 0 fills two, slot 1 a part of its second, slot 2 one.  A round finds no page for
    slot 0; when slot 2 has ended, the same round goes through."""
    T, penalties, base = 33, (1.2, 0.3, 0.1), 500.0
    model = sd.Decoder("gaga", slots=3, max_len=64, pages=5, rotary=base, penalties=penalties)
    slot = torch.arange(3, dtype=torch.int32, device="cuda")
    prompt = prompts(model, 3, T)
    anchors = []
    for s, n in enumerate((T, 21, 11)):
        anchor, status = model.prefill(prompt[s:s + 1, :n], slot[s:s + 1])
        assert not status.any()
        anchors.append(anchor)
    before, other = held(model, 0), held(model, 1)
    *_, status = model.round(torch.cat(anchors[:2]), slot[:2], 5, 0.0)
    assert status.tolist() == [bd.BDGDN_CACHE_NO_PAGES, bd.BDGDN_CACHE_DONE]
    for name, a, b in zip(("taken", "history", "seq_len", "state", "state"), before, held(model, 0)):
        assert torch.equal(a, b), name
    assert int(model.taken[1]) == int(model.tables.seq_len[1]) > int(other[0])
    model.finish(slot[2:])
    sequences, anchor = [prompt[0].tolist()], anchors[0]
    for _ in range(2):
        step = model.round(anchor, slot[:1], 5, 0.0)
        assert not step[3].any()
        anchor = go_on(sequences, step)
    check(model, sequences, T, base, penalties)


def test_a_refused_fork_leaves_the_sequence_as_it_was():
    model = sd.Decoder("ga", slots=3, max_len=64, rotary=500.0, penalties=(1.2, 0.3, 0.1))
    slot = torch.arange(3, dtype=torch.int32, device="cuda")
    prompt = prompts(model, 2, 20)
    for s in range(2):
        model.prefill(prompt[s:s + 1, :20 - 5 * s], slot[s:s + 1])
    source, taken = held(model, 0), held(model, 1)
    status = model.fork(slot[:1].repeat(2), slot[1:])   # slot 1 is in use
    assert status.tolist() == [bd.BDGDN_CACHE_BAD_SLOT, bd.BDGDN_CACHE_DONE]
    assert all(torch.equal(a, b) for a, b in zip(taken, held(model, 1)))
    assert all(torch.equal(a, b) for a, b in zip(source, held(model, 2)))


def test_a_slot_that_is_used_again():
    model = sd.Decoder("ga", slots=2, max_len=64, rotary=500.0, penalties=(1.2, 0.3, 0.1))
    slot = torch.arange(2, dtype=torch.int32, device="cuda")
    prompt = prompts(model, 2, 20)
    model.prefill(prompt[:1], slot[:1])
    model.finish(slot[:1])
    for s in range(2):   # the same prompt where a sequence has been, and where none has
        model.prefill(prompt[1:], slot[s:s + 1])
    assert all(torch.equal(a, b) for a, b in zip(held(model, 0), held(model, 1)))
