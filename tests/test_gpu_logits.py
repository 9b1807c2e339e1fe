"""bdgdn_logits and bdgdn_history_add against the definition, token by token, in 64 bits.

Tolerance.  fp32 steps, in order: the reciprocal of repetition and the product with it (2 roundings of
2^-24 of the logit), presence + frequency c (one), the difference and the sum with the bias (one each,
of terms that are at most the sum of the magnitudes).  So 5 x 2^-24 of |x| max(rho, 1 / rho) + presence +
|frequency| c + |bias|, and half a step of the result's type.
"""
import pytest
import torch

import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu

STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
B, F = torch.bfloat16, torch.float32
PROMPT = bd.BDGDN_HISTORY_PROMPT


def ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def parents_words(parent):
    words = []
    for row in parent:
        w = []
        for n, p in enumerate(row):
            w.append((w[p] if 0 <= p < n else 0) | 1 << n)
        words.append(w)
    return words


def signed(words):
    return torch.tensor([[w - (1 << 64) if w >> 63 else w for w in row] for row in words], dtype=torch.int64).cuda()


def reference(x, token, words, count, history, slot, rho, presence, frequency, bias_token, bias, allow):
    """The processed rows (rows behind a request's nodes: NaN) and the magnitudes of their terms."""
    R, N, V = x.shape
    out, size = torch.full((R, N, V), float("nan"), dtype=torch.float64), torch.zeros(R, N, V, dtype=torch.float64)
    for r in range(R):
        nodes = N if count is None else min(count[r], N)
        s = r if slot is None else slot[r]
        word = history[s].long() if history is not None and 0 <= s < len(history) else torch.zeros(V, dtype=torch.int64)
        f = rho[r] if rho is not None and rho[r] > 0 else 1.0
        f = float(torch.tensor(f, dtype=torch.float32))
        pr, fr = (0.0 if t is None else float(torch.tensor(t[r], dtype=torch.float32)) for t in (presence, frequency))
        for n in range(nodes):
            c = word & (PROMPT - 1)
            if token is not None:
                for j in range(nodes):
                    sees = words[r][n] >> j & 1 if words is not None else j <= n
                    if sees and 0 <= token[r][j] < V:
                        c[token[r][j]] += 1
            seen = (c > 0) | ((word & PROMPT) > 0)
            v = x[r, n].double()
            v = torch.where(seen, torch.where(v > 0, v / f, v * f), v)
            size[r, n] = v.abs() + (c > 0) * abs(pr) + c * abs(fr)
            v = v - (c > 0) * pr - c * fr
            if bias is not None:
                last = {t: b for t, b in zip(bias_token[r], bias[r].tolist())}
                for t, b in last.items():
                    if 0 <= t < V:
                        v[t] += b
                        size[r, n, t] += abs(b)
            if allow is not None:
                bits = allow[r if len(allow) > 1 else 0][n if len(allow[0]) > 1 else 0]
                for t in range(V):
                    if not bits[t // 32] >> t % 32 & 1:
                        v[t] = -float("inf")
            out[r, n] = v
    return out, size


def check(got, want, size, before=None):
    got = got.cpu()
    there = ~want.isnan()
    g, w, s = got.double()[there], want[there], size[there]
    gone = w == -float("inf")
    assert (g[gone] == -float("inf")).all()
    err = (g - w)[~gone].abs()
    assert (err <= 5 * 2.0 ** -24 * s[~gone] + STEP[got.dtype] * w[~gone].abs()).all(), float(err.max())
    if before is not None:
        assert torch.equal(got[~there], before.cpu().to(got.dtype)[~there])


def make(R, N, V, seed, slots=None):
    g = torch.Generator().manual_seed(seed)
    slots = R + 2 if slots is None else slots
    history = torch.where(torch.rand(slots, V, generator=g) < 0.3, torch.randint(0, 5, (slots, V), generator=g), 0)
    history = (history + PROMPT * (torch.rand(slots, V, generator=g) < 0.2)).to(torch.int32)
    token = torch.randint(-2, V + 2, (R, N), generator=g).tolist()
    for row in token:   # tokens that come twice, at the row's ends
        row[-1] = row[0]
        if N > 3:
            row[1], row[2] = 0, V - 1
    parent = [[-1] + [int(torch.randint(max(0, n - 4), n, (1,), generator=g)) for n in range(1, N)] for _ in range(R)]
    allow = torch.randint(0, 2 ** 32, (R, N, (V + 31) // 32), generator=g)
    allow[0, 0] = 0   # a grammar that allows nothing
    return g, history, token, parents_words(parent), allow


@pytest.mark.parametrize("types", [(B, B), (B, F), (F, F)])
@pytest.mark.parametrize("R,N,V", [(1, 1, 1), (1, 8, 33), (3, 5, 100), (2, 64, 2047), (2, 3, 2049), (5, 2, 4100), (1, 24, 5000)])
def test_everything_at_once(R, N, V, types):
    g, history, token, words, allow = make(R, N, V, V + N)
    x = (torch.randn(R, N, V, generator=g) * 3).to(types[0])
    slot = torch.randperm(R + 2, generator=g)[:R].tolist()
    K = min(9, 2 * V)
    bias_token = torch.randint(-1, V + 1, (R, K), generator=g).tolist()
    for row in bias_token:
        row[-1] = row[0]   # the last of equal tokens counts
    bias = torch.randn(R, K, generator=g)
    count = [max(0, N - i) for i in range(R)]
    rho, presence, frequency = ([1.3, 0.7, 1.0, -1.0, 2.0][:R], [0.5, 0.0, -0.25, 0.1, 0.0][:R], [0.125, 0.3, 0.0, -0.2, 0.0][:R])
    want, size = reference(x, token, words, count, history, slot, rho, presence, frequency, bias_token, bias, allow.tolist())
    low = torch.where(allow >= 2 ** 31, allow - 2 ** 32, allow).to(torch.int32).cuda()
    kw = dict(token=ints(token), mask=signed(words), count=ints(count), history=history.cuda(), slot=ints(slot),
              repetition=torch.tensor(rho).cuda(), presence=torch.tensor(presence).cuda(),
              frequency=torch.tensor(frequency).cuda(), bias_token=ints(bias_token), bias=bias.cuda(), allow=low)
    out = torch.full((R, N, V), 3.0, dtype=types[1], device="cuda")
    got = bd.bdgdn_logits(x.cuda(), out=out, **kw)
    assert got is out
    check(got, want, size, torch.full((R, N, V), 3.0))
    if types[0] is types[1]:
        inside = x.cuda()
        bd.bdgdn_logits(inside, out=inside, **kw)
        check(inside, want, size, x)
        there = ~want.isnan()
        assert torch.equal(inside.cpu()[there], got.cpu()[there])


@pytest.mark.parametrize("V", [2048, 3001])
@pytest.mark.parametrize("what", ["nothing", "history", "chain", "presence", "bias", "request", "shared", "all_gone"])
def test_parts(what, V):
    R, N = 3, 4
    g, history, token, words, allow = make(R, N, V, 3, slots=R)
    x = torch.randn(R, N, V, generator=g)
    a = dict(token=None, words=None, count=None, history=None, slot=None, rho=None, presence=None, frequency=None,
             bias_token=None, bias=None, allow=None)
    kw = {}
    if what in ("history", "chain"):
        a.update(history=history, rho=[1.2, 3.0, 0.5])
        kw.update(history=history.cuda(), repetition=torch.tensor([1.2, 3.0, 0.5]).cuda())
    if what == "chain":
        a.update(token=token, slot=[2, 7, 0])
        kw.update(token=ints(token), slot=ints([2, 7, 0]))
    if what == "presence":   # without a history the block's tokens count
        a.update(token=token, words=words, presence=[0.5, -1.0, 2.0])
        kw.update(token=ints(token), mask=signed(words), presence=torch.tensor([0.5, -1.0, 2.0]).cuda())
    if what == "bias":
        bt, b = [[5, V - 1, 5], [0, 1, 2], [V, -1, 7]], torch.tensor([[1.0, -float("inf"), 2.0], [0.5, 0.25, 0.125], [9.0, 9.0, -3.0]])
        a.update(bias_token=bt, bias=b)
        kw.update(bias_token=ints(bt), bias=b.cuda())
    if what in ("request", "shared", "all_gone"):
        part = allow[:, :1] if what == "request" else allow[1:2, 1:2]
        part = part * 0 if what == "all_gone" else part
        a.update(allow=part.tolist())
        kw.update(allow=torch.where(part >= 2 ** 31, part - 2 ** 32, part).to(torch.int32).cuda())
    want, size = reference(x, **a)
    check(bd.bdgdn_logits(x.cuda(), **kw), want, size)
    if what == "nothing":
        assert torch.equal(bd.bdgdn_logits(x.cuda()).cpu(), x)


def test_values_that_are_not_finite():
    V = 70
    x = torch.randn(1, 2, V)
    x[0, 0, 3], x[0, 0, 4], x[0, 0, 5], x[0, 1, 3] = float("nan"), float("inf"), -float("inf"), float("nan")
    allow = torch.full((1, 1, 3), -1, dtype=torch.int32)
    allow[0, 0, 0] &= ~(1 << 3)
    history = torch.zeros(1, V, dtype=torch.int32)
    history[0, 4], history[0, 5] = 2, PROMPT
    got = bd.bdgdn_logits(x.cuda(), allow=allow.cuda(), history=history.cuda(), repetition=torch.tensor([1.5]).cuda(),
                          frequency=torch.tensor([0.5]).cuda()).cpu()
    assert got[0, 0, 3] == got[0, 1, 3] == -float("inf")   # a masked NaN is masked
    assert got[0, 0, 4] == float("inf") and got[0, 0, 5] == -float("inf")
    got = bd.bdgdn_logits(x.cuda()).cpu()
    assert got[0, 0, 3].isnan() and int(got.isnan().sum()) == 2


@pytest.mark.parametrize("dtype", [B, F])
def test_strides(dtype):
    """Rows that are parts of longer ones, at addresses of an element; one row shared by all nodes."""
    R, N, V = 2, 3, 2500
    g, history, token, words, allow = make(R, N, V, 9)
    room = torch.randn(R, N + 1, V + 5, generator=g).to(dtype).cuda()
    x = room[:, 1:, 3:3 + V]
    out = torch.full((R, N, V + 3), 4.0, dtype=dtype, device="cuda")
    wide = torch.zeros(R + 2, V + 9, dtype=torch.int32, device="cuda")
    wide[:, 2:V + 2] = history.cuda()
    kw = dict(rho=[1.5, 0.5], frequency=[0.1, 0.2])
    got = bd.bdgdn_logits(x, token=ints(token), mask=signed(words), history=wide[:, 2:V + 2], slot=ints([3, 0]),
                          repetition=torch.tensor(kw["rho"]).cuda(), frequency=torch.tensor(kw["frequency"]).cuda(),
                          out=out[:, :, 1:V + 1])
    want, size = reference(x.cpu(), token, words, None, history, [3, 0], kw["rho"], None, kw["frequency"], None, None, None)
    check(got, want, size)
    assert (out[:, :, 0] == 4).all() and (out[:, :, V + 1:] == 4).all()
    one = x[:, :1].expand(R, N, V)
    got = bd.bdgdn_logits(one, token=ints(token), mask=signed(words), presence=torch.tensor([1.0, 0.5]).cuda())
    want, size = reference(one.cpu(), token, words, None, None, None, None, [1.0, 0.5], None, None, None, None)
    check(got, want, size)


def test_nodes_shared_out_among_workgroups_give_the_same():
    R, N, V = 40, 16, 40000   # all nodes to a workgroup; alone, one to each
    x = torch.randn(R, N, V, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    token = torch.randint(0, V, (R, N), generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()
    history = torch.randint(0, 2, (R, V), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    rho = torch.full((R,), 1.25, device="cuda")
    whole = bd.bdgdn_logits(x, token=token, history=history, repetition=rho)
    for r in (0, 17, 39):
        one = bd.bdgdn_logits(x[r:r + 1], token=token[r:r + 1], history=history[r:r + 1], repetition=rho[:1])
        assert torch.equal(one[0], whole[r])


def test_history_add():
    slots, V, R, N = 4, 50, 5, 6
    g = torch.Generator().manual_seed(6)
    token = torch.randint(-3, V + 3, (R, N), generator=g)
    token[0, 3:] = 7      # one token several times
    token[4] = 7
    slot, count = [2, 0, 2, 9, 2], [6, 3, -1, 4, 20]   # a slot twice, slots that are not there
    path = [[5, 4, 3, 2, 1, 0], [0, 2, -1, 9, 0, 0], [0] * 6, [0] * 6, [1, 1, 1, 7, 2, 3]]
    want, marks = torch.zeros(slots, V, dtype=torch.int64), torch.zeros(slots, V, dtype=torch.int64)
    for r in range(R):
        for j in range(min(max(count[r], 0), N)):
            n, s = path[r][j], slot[r]
            if 0 <= n < N and 0 <= s < slots and 0 <= token[r, n] < V:
                want[s, token[r, n]] += 1
                marks[s, token[r, n]] = PROMPT
    history = torch.zeros(slots, V, dtype=torch.int32, device="cuda")
    args = (token.to(torch.int32).cuda(),)
    kw = dict(slot=ints(slot), path=ints(path), count=ints(count))
    bd.bdgdn_history_add(history, *args, **kw)
    assert torch.equal(history.cpu().long(), want)
    bd.bdgdn_history_add(history, *args, prompt=True, **kw)
    assert torch.equal(history.cpu().long(), want + marks)
    part = torch.zeros(3, V + 6, dtype=torch.int32, device="cuda")
    long = torch.randint(0, V, (2, 3000), generator=g)
    bd.bdgdn_history_add(part[:, 2:V + 2], long.to(torch.int32).cuda())
    assert torch.equal(part[:2, 2:V + 2].cpu().long(), torch.stack([torch.bincount(row, minlength=V) for row in long]))
    assert not part[2].any() and not part[:, :2].any() and not part[:, V + 2:].any()
    bd.bdgdn_history_add(history, torch.zeros(0, 4, dtype=torch.int32, device="cuda"))
    bd.bdgdn_history_add(history, torch.zeros(2, 0, dtype=torch.int32, device="cuda"))
    assert torch.equal(history.cpu().long(), want + marks)
