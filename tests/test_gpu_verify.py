"""bdgdn_verify against the rule in 64 bits, at the places where it can go wrong, and against
the law that it is meant to give: the first token that comes out is distributed as the target's.
Integers have to be equal: the inputs are drawn so that no decision is nearer than 1e-5 to its
border (checked by the reference)."""
import math

import numpy as np
import pytest
import torch

import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu


def _law(x, T):
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or not np.isfinite(x.max()):
        return None
    if not T > 0:
        p = np.zeros_like(x)
        p[int(np.argmax(x))] = 1
        return p
    e = np.exp((x - x.max()) / T)
    return e / e.sum()


def _reference(target, draft, token, parent, count, T, u, noise):
    """One request; (n_accept, path, next, margin of the closest decision)."""
    path, cur, margin = [0], 0, math.inf
    while True:
        p = _law(target[cur], T)
        if p is None:
            return len(path) - 1, path, -1, margin
        left, q = p, None
        if draft is not None and T > 0 and cur < len(draft):
            q = _law(draft[cur], T)
            lawless = q is None
            q = np.zeros_like(p) if lawless else q
        else:
            lawless = False
        taken = False
        for n in range(cur + 1, count):
            if parent[n] != cur or not 0 <= token[n] < len(p) or lawless:
                continue
            odds = 1.0 if draft is None or not T > 0 else q[token[n]]
            a, b = u[n] * odds, left[token[n]]
            if a != b:
                margin = min(margin, abs(a - b) / max(a, b))
            if a < b:
                cur, taken = n, True
                path.append(n)
                break
            if draft is None or not T > 0:
                left = left.copy()
                left[token[n]] = 0
            else:
                left = np.maximum(left - q, 0)
            if left.sum() > 0:
                left = left / left.sum()
        if not taken:
            break
    score = (left if left.max() > 0 else p) / noise
    best = np.sort(score)[::-1]
    if best[0] <= 0:
        return len(path) - 1, path, -1, margin
    if len(best) > 1 and best[1] != best[0]:
        margin = min(margin, (best[0] - best[1]) / best[0])
    return len(path) - 1, path, int(np.argmax(score)), margin


def _random(R, N, V, dtype, draft, tree, seed, T):
    g = torch.Generator(device="cuda").manual_seed(seed)
    target = torch.empty(R, N, V, device="cuda").normal_(0, 2, generator=g).to(dtype)
    near = (target.float() + torch.empty(R, N, V, device="cuda").normal_(0, 0.8, generator=g)).to(dtype)
    rng = np.random.default_rng(seed)
    parent = np.stack([[-1] + [int(rng.integers(max(0, n - 4), n)) if tree else n - 1 for n in range(1, N)]
                       for _ in range(R)]).astype(np.int32)
    token = np.zeros((R, N), dtype=np.int32)
    for r in range(R):
        for n in range(1, N):
            row = near[r, parent[r, n]].double().cpu().numpy()
            if draft == "sampled":
                token[r, n] = int(np.argmax(_law(row, T[r] if T[r] > 0 else 1.0) / rng.exponential(size=V)))
            else:
                rank = int((parent[r, :n] == parent[r, n]).sum())
                token[r, n] = int(np.argsort(-row, kind="stable")[min(rank, V - 1)])
    u = torch.rand(R, N, device="cuda", generator=g)
    noise = torch.empty(R, V, device="cuda").exponential_(generator=g)
    return dict(target=target, draft=near if draft == "sampled" else None, token=torch.from_numpy(token).cuda(),
                parent=torch.from_numpy(parent).cuda(), u=u, noise=noise,
                temperature=torch.tensor(T, dtype=torch.float32, device="cuda"))


def _check(c, count=None, **given):
    R, N, V = c["target"].shape
    got = bd.bdgdn_verify(c["target"], c["token"], c["u"], c["noise"], draft=c["draft"], parent=c["parent"],
                          temperature=c["temperature"], count=count, want_n_path=True, **given)
    acc, path, nxt, n_path = (t.cpu().numpy() for t in got)
    host = {k: None if v is None else v.double().cpu().numpy() for k, v in c.items()}
    T = host["temperature"] if host["temperature"] is not None else np.ones(R)
    skipped = 0
    for r in range(R):
        live = N if count is None else int(count[r])
        parent = [-1] + list(range(N - 1)) if host["parent"] is None else host["parent"][r].astype(int)
        a, p, t, margin = _reference(host["target"][r], None if host["draft"] is None else host["draft"][r],
                                     host["token"][r].astype(int), parent, live, T[r], host["u"][r], host["noise"][r])
        if margin < 1e-5:
            skipped += 1
            continue
        assert (acc[r], n_path[r], nxt[r]) == (a, a + 1, t), (r, a, p, t)
        assert path[r].tolist() == p + [-1] * (N - len(p))
    assert skipped <= max(1, R // 20)
    return acc, path, nxt


@pytest.mark.parametrize("R,N,V,dtype,draft,tree", [
    (1, 1, 7, torch.float32, "sampled", False),
    (3, 2, 1, torch.float32, "point", False),
    (9, 8, 1000, torch.bfloat16, "sampled", False),
    (7, 8, 4099, torch.float32, "sampled", False),
    (5, 13, 777, torch.bfloat16, "sampled", True),
    (6, 24, 2500, torch.float32, "sampled", True),
    (6, 16, 5001, torch.bfloat16, "point", True),
    (4, 64, 300, torch.float32, "point", True),
    (2, 6, 70001, torch.bfloat16, "sampled", True),
    (70, 4, 33, torch.float32, "sampled", True),
])
def test_against_the_rule(R, N, V, dtype, draft, tree):
    T = [(1.0, 0.6, 0.0, 1.4)[r % 4] for r in range(R)]
    _check(_random(R, N, V, dtype, draft, tree, seed=R * N + V, T=T))


@pytest.mark.parametrize("draft", ["sampled", "point"])
def test_temperatures_at_the_ends_of_fp32(draft):
    """The law tends to one token, and to all of them alike."""
    T = [1e-45, 1e-39, 1e-30, 1e30, 3e38, math.inf]
    _check(_random(6, 5, 501, torch.float32, draft, False, seed=8, T=T))


def test_chains_need_no_parents_and_no_last_draft_row():
    c = _random(6, 5, 501, torch.bfloat16, "sampled", False, seed=3, T=[1.0] * 6)
    want = [t.clone() for t in bd.bdgdn_verify(c["target"], c["token"], c["u"], c["noise"], draft=c["draft"],
                                               parent=c["parent"])]
    for draft in (c["draft"][:, :4], c["draft"][:, :4].contiguous()):
        got = bd.bdgdn_verify(c["target"], c["token"], c["u"], c["noise"], draft=draft)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    c["parent"], c["temperature"] = None, None
    c["draft"] = c["draft"][:, :4]
    _check(c)


def test_rows_inside_longer_ones():
    """Logits and noise that are columns of wider arrays, at odd places."""
    c = _random(4, 6, 2003, torch.bfloat16, "sampled", True, seed=8, T=[1.0, 0.8, 0.0, 1.0])
    for k, lead in (("target", 3), ("draft", 5)):
        wide = torch.full((4, 6, 2019), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, :, lead:lead + 2003] = c[k]
        c[k] = wide[:, :, lead:lead + 2003]
    wide = torch.full((4, 2010), float("nan"), device="cuda")
    wide[:, 1:2004] = c["noise"]
    c["noise"] = wide[:, 1:2004]
    _check(c)


def test_counts_tokens_and_parents_that_are_none():
    c = _random(6, 8, 300, torch.float32, "sampled", True, seed=5, T=[1.0] * 6)
    c["token"][0, 1:4] = torch.tensor([-1, 300, 2 ** 31 - 1], dtype=torch.int32)
    c["parent"][1, 2:5] = torch.tensor([7, -5, 100], dtype=torch.int32)
    count = torch.tensor([8, 8, 1, 5, 8, 99], dtype=torch.int32).cuda()
    ws = torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    host = count.clamp(max=8)
    got = bd.bdgdn_verify(c["target"], c["token"], c["u"], c["noise"], draft=c["draft"], parent=c["parent"], count=count,
                          workspace=ws)
    want = _check(c, count=host)
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want))
    zero = torch.tensor([0, -3, 1, 1, 1, 1], dtype=torch.int32).cuda()
    acc, path, nxt, n_path = bd.bdgdn_verify(c["target"], c["token"], c["u"], c["noise"], draft=c["draft"],
                                             parent=c["parent"], count=zero, want_n_path=True)
    assert nxt[:2].tolist() == [-1, -1] and n_path.tolist() == [0, 0, 1, 1, 1, 1] and not acc.any()
    assert (path[:2] == -1).all() and (nxt[2:] >= 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_without_a_law_and_tokens_of_probability_zero(dtype):
    c = _random(8, 3, 400, dtype, "sampled", False, seed=4, T=[1.0, 1.0, 1.0, 0.0, 0.0, 1.0, 1.0, 0.5])
    inf = float("inf")
    c["target"][0, 0] = -inf
    c["target"][1, 0, 7] = float("nan")
    c["target"][2, 0, 9] = inf
    c["target"][3, 0] = -inf
    c["target"][4, 0, 399] = float("nan")
    c["target"][5, :, 1:] = -inf            # all on token 0
    c["draft"][6, 0, 3] = float("nan")      # a draft without a law: its children are refused
    c["target"][7, :, ::2] = -inf
    c["u"][:, 1] = 0.5
    c["u"][5, 1] = 0.999
    acc, path, nxt = _check(c)
    assert nxt[:5].tolist() == [-1] * 5 and not acc[:5].any() and nxt[5] == 0 and acc[6] == 0 and nxt[7] % 2 == 1


def test_ties_go_to_the_lowest_index():
    V = 5000
    target = torch.zeros(3, 2, V, device="cuda", dtype=torch.bfloat16)
    target[:, :, 1234] = target[:, :, 77] = target[:, :, 4321] = 3.0
    noise = torch.ones(3, V, device="cuda")
    token = torch.tensor([[0, 77], [0, 1234], [0, 4000]], dtype=torch.int32).cuda()
    u = torch.full((3, 2), 0.99999, device="cuda")
    greedy = torch.tensor([0.0, 0.0, -1.0], device="cuda")
    acc, path, nxt = bd.bdgdn_verify(target, token, u, noise, temperature=greedy)
    assert acc.tolist() == [1, 0, 0] and nxt.tolist() == [77, 77, 77]
    acc, path, nxt = bd.bdgdn_verify(target, token, u, noise)   # certain drafts: the refused token is out
    assert acc.tolist() == [0, 0, 0] and nxt.tolist() == [1234, 77, 77]


@pytest.mark.parametrize("V", [32760, 32768, 32769, 40003])
@pytest.mark.parametrize("dtype,draft,tree", [(torch.float32, "point", True), (torch.bfloat16, "sampled", False)])
def test_vocabularies_about_the_length_that_one_workgroup_races_over(V, dtype, draft, tree):
    T = [(1.0, 0.6, 0.0, 1.4)[r % 4] for r in range(6)]
    _check(_random(6, 6, V, dtype, draft, tree, seed=V, T=T))


@pytest.mark.parametrize("V", [300, 40003])
def test_long_and_short_rows_without_a_law_and_ties(V):
    c = _random(6, 3, V, torch.float32, "sampled", False, seed=5, T=[1.0] * 6)
    c["target"][0, 0] = float("-inf")
    c["target"][1, 0, V - 1] = float("nan")
    c["target"][2, :, 1:] = float("-inf")       # all on token 0
    c["target"][3] = c["draft"][3]              # a refusal leaves nothing: the target's own law
    c["u"][3, 1] = 1.0
    c["target"][4, :, :] = 0                    # ties: the lowest of equal scores
    c["noise"][4] = 1
    c["u"][4, 1] = 0.9999
    c["draft"][4, 0] = 0
    c["draft"][4, 0, int(c["token"][4, 1])] = 3
    count = torch.tensor([3, 3, 3, 2, 2, 0], dtype=torch.int32).cuda()
    acc, path, nxt, n_path = (x.tolist() for x in bd.bdgdn_verify(
        c["target"], c["token"], c["u"], c["noise"], draft=c["draft"], count=count, want_n_path=True))
    assert nxt[0] == nxt[1] == nxt[5] == -1 and nxt[2] == 0
    assert acc[:2] == [0, 0] and acc[3:] == [0, 0, 0] and n_path[5] == 0 and path[5] == [-1] * 3
    score = torch.softmax(c["target"][3, 0].double(), 0) / c["noise"][3].double()
    assert nxt[3] == int(score.argmax())
    refused = int(c["token"][4, 1])
    assert nxt[4] == (1 if refused == 0 else 0)


@pytest.mark.parametrize("draft", ["sampled", "point"])
def test_what_comes_out_is_distributed_as_the_target(draft):
    """The first token after the anchor, accepted or drawn, over 40000 requests with three drafts
    side by side: chi-squared against p with 9 degrees of freedom stays under its 1 - 1e-6 point."""
    R, V = 40000, 10
    g = torch.Generator(device="cuda").manual_seed(1)
    row = torch.tensor([1.0, 0.2, -0.5, 2.0, 0.0, -1.0, 0.7, 1.4, -2.0, 0.3], device="cuda")
    other = torch.tensor([0.1, 1.2, 0.5, 1.0, -1.0, 0.0, 1.7, -0.4, 0.0, 0.3], device="cuda")
    target = row.expand(R, 4, V).contiguous()
    near = other.expand(R, 4, V).contiguous()
    q = torch.softmax(other, 0).expand(R, V)
    if draft == "sampled":
        token = torch.stack([torch.zeros(R, device="cuda")] + [
            (q / torch.empty(R, V, device="cuda").exponential_(generator=g)).argmax(-1) for _ in range(3)], 1)
    else:
        token = torch.tensor([0, 6, 1, 3], device="cuda").expand(R, 4)
    token = token.to(torch.int32).contiguous()
    parent = torch.tensor([-1, 0, 0, 0], dtype=torch.int32).expand(R, 4).contiguous().cuda()
    u = torch.rand(R, 4, device="cuda", generator=g)
    noise = torch.empty(R, V, device="cuda").exponential_(generator=g)
    acc, path, nxt = bd.bdgdn_verify(target, token, u, noise, draft=near if draft == "sampled" else None, parent=parent)
    first = torch.where(acc > 0, token.gather(1, path[:, 1:2].clamp(min=0).long())[:, 0], nxt)
    seen = torch.bincount(first.long(), minlength=V).double()
    want = torch.softmax(row.double(), 0) * R
    assert float(((seen - want) ** 2 / want).sum()) < 44.9   # the 1 - 1e-6 point is 44.81
    assert 0.2 < float((acc > 0).double().mean()) < 0.999


def test_another_stream_and_a_replayed_graph():
    c = _random(5, 6, 3001, torch.bfloat16, "sampled", True, seed=21, T=[1.0] * 5)
    args = (c["target"], c["token"], c["u"], c["noise"])
    kw = dict(draft=c["draft"], parent=c["parent"])
    out = [torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(5, 6, dtype=torch.int32, device="cuda"),
           torch.zeros(5, dtype=torch.int32, device="cuda")]
    keep = dict(n_accept=out[0], path=out[1], next_token=out[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bd.bdgdn_verify(*args, **kw, **keep)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, bd.bdgdn_verify(*args, **kw)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bd.bdgdn_verify(*args, **kw, **keep)
    for _ in range(4):
        c["u"].copy_(torch.rand_like(c["u"]))
        c["noise"].exponential_()
        for t in out:
            t.fill_(-7)
        want = [t.clone() for t in bd.bdgdn_verify(*args, **kw)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
