"""bdgdn_tree_attn and bdgdn_tree_mask against the definition in 64 bits.

Tolerances: with w the softmax weights and A = sum w |v|, a bf16 output is off by its own
rounding (2^-8 |o|: bf16 keeps 8 significant bits) and that of the weights (2^-8 A).  Scores are sums of d products in fp32,
off by at most (d + 8) 2^-24 S with S the largest scale * sum |q_i k_i|, which enters a weight
as a factor; n weights are summed in fp32.  So fp32 outputs are off by at most
(4 (d + 8) S + n + 64) 2^-24 A, plus 2^-16 A where the weights are in two bf16 parts.
"""
import math

import pytest
import torch

import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(R, N, h_q, h_kv, d, page, lens, dtype, *, htd=False, seed=0, slots=None, spare=2, std=2.0, max_pages=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[dtype]
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    max_pages = max(1, max(need)) + 1 if max_pages is None else max_pages
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    slots = list(range(R)) if slots is None else slots
    table = torch.full((max(slots) + 1, max_pages), -1, dtype=torch.int32)
    seq = torch.zeros(max(slots) + 1, dtype=torch.int32)
    at = 0
    for s, n, k in zip(slots, lens, need):
        table[s, :k] = order[at:at + k]
        seq[s] = n
        at += k

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(0, std, generator=g)

    def pool():
        return normal(n_pages, h_kv, page, d).transpose(1, 2) if htd else normal(n_pages, page, h_kv, d)

    return dict(q=normal(R, N, h_q, d, std=std), k=normal(R, N, h_kv, d), v=normal(R, N, h_kv, d), kp=pool(), vp=pool(),
                table=table.cuda(), seq=seq.cuda(), slots=slots, lens=list(lens), page=page,
                slot=torch.tensor(slots, dtype=torch.int32).cuda())


def _sees(mask, R, N):
    if isinstance(mask, torch.Tensor):
        m = mask.cpu()
        return torch.stack([(m >> j) & 1 for j in range(N)], -1).bool()
    full = torch.ones(N, N, dtype=torch.bool)
    return (full.tril() if mask == "causal" else full).expand(R, N, N)


def _reference(c, mask, scale, count=None):
    """(o, lse, A, S, keys) in float64."""
    R, N, h_q, d = c["q"].shape
    h_kv, page = c["k"].shape[2], c["page"]
    G = h_q // h_kv
    sees = _sees(mask, R, N).cuda()
    o = torch.zeros(R, N, h_q, d, dtype=torch.float64, device="cuda")
    lse = torch.full((R, N, h_q), -math.inf, dtype=torch.float64, device="cuda")
    A, S = torch.zeros_like(o), torch.zeros_like(lse)
    table = c["table"].cpu()
    for r in range(R):
        t = [x for x in range(c["lens"][r]) if 0 <= int(table[c["slots"][r], x // page]) < c["kp"].shape[0]]
        pg = torch.tensor([int(table[c["slots"][r], x // page]) for x in t], dtype=torch.long, device="cuda")
        pl = torch.tensor([x % page for x in t], dtype=torch.long, device="cuda")
        live = N if count is None else int(count[r])
        for n in range(live):
            own = [j for j in range(live) if bool(sees[r, n, j])]
            if not t and not own:
                continue
            k = torch.cat([c["kp"][pg, pl], c["k"][r, own]]).double()
            v = torch.cat([c["vp"][pg, pl], c["v"][r, own]]).double()
            for h in range(h_q):
                x = c["q"][r, n, h].double()
                s = (k[:, h // G] * x).sum(-1) * scale
                z = torch.logsumexp(s, 0)
                w = torch.exp(s - z)
                o[r, n, h] = (w[:, None] * v[:, h // G]).sum(0)
                A[r, n, h] = (w[:, None] * v[:, h // G].abs()).sum(0)
                S[r, n, h] = ((k[:, h // G] * x).abs().sum(-1) * abs(scale)).max()
                lse[r, n, h] = z
    return o, lse, A, S


def _compare(c, out, mask, scale, dtype, out_dtype, count=None):
    o, lse = out
    ro, rl, A, S = _reference(c, mask, scale, count)
    d, n = o.shape[-1], max(c["lens"]) + o.shape[1]
    assert torch.isfinite(o).all()
    unit = (4 * (d + 8) * S + n + 64) * 2.0 ** -24
    tol = unit[..., None] * A
    if dtype == "bf16":
        tol += 2.0 ** -16 * A
        if out_dtype == "bf16":
            tol += 2.0 ** -8 * 1.01 * (A + ro.abs())
    err = (o.double() - ro).abs()
    assert (err <= tol + 1e-30).all(), float((err / (tol + 1e-30)).max())
    none = torch.isinf(rl)
    assert torch.equal(torch.isinf(lse), none) and (lse[none] < 0).all() and not o[none].any()
    lerr = (lse.double() - rl)[~none].abs()
    assert (lerr <= unit[~none] + 2.0 ** -22 * (1 + rl[~none].abs())).all()


@pytest.mark.parametrize("R,N,h_q,h_kv,d,page,lens,dtype,out,mask,htd", [
    (1, 1, 4, 1, 128, 64, [1], "bf16", "bf16", "full", False),
    (1, 1, 8, 8, 64, 16, [0], "bf16", "f32", "causal", False),
    (3, 5, 6, 2, 128, 64, [70, 0, 333], "bf16", "bf16", "causal", False),
    (2, 8, 8, 2, 128, 16, [129, 1000], "bf16", "f32", "tree", True),
    (2, 33, 4, 1, 128, 32, [31, 257], "bf16", "bf16", "full", False),
    (1, 64, 3, 3, 64, 24, [100], "bf16", "bf16", "tree", False),
    (2, 64, 8, 1, 64, 128, [40, 700], "bf16", "f32", "causal", True),
    (2, 7, 10, 2, 256, 16, [37, 515], "bf16", "bf16", "tree", False),
    (1, 20, 4, 2, 256, 100, [300], "bf16", "f32", "full", True),
    (3, 3, 5, 1, 128, 1, [9, 64, 33], "bf16", "bf16", "causal", False),
    (2, 6, 4, 4, 128, 7, [50, 96], "bf16", "bf16", "full", False),
    (2, 4, 4, 2, 64, 24, [0, 77], "f32", "f32", "tree", False),
    (1, 17, 6, 2, 128, 32, [150], "f32", "f32", "causal", True),
    (2, 9, 4, 1, 256, 64, [65, 130], "f32", "f32", "full", False),
    (1, 40, 2, 2, 64, 5, [44], "f32", "f32", "full", False),
    (5, 2, 32, 8, 128, 64, [64, 63, 65, 2000, 1], "bf16", "bf16", "causal", False),
    (70, 1, 2, 1, 64, 16, [(37 * i) % 90 for i in range(70)], "bf16", "bf16", "full", False),
    # many rows to a key head: each number of row waves and head size, one tile to many stages
    (2, 12, 8, 2, 64, 16, [5, 300], "bf16", "bf16", "tree", False),
    (2, 25, 8, 2, 64, 48, [1100, 16], "bf16", "f32", "causal", True),
    (1, 50, 4, 1, 64, 64, [777], "bf16", "bf16", "full", False),
    (3, 10, 6, 1, 128, 32, [0, 31, 1500], "bf16", "f32", "tree", True),
    (2, 32, 8, 2, 128, 64, [2049, 95], "bf16", "bf16", "full", False),
    (1, 64, 16, 2, 128, 16, [1000], "bf16", "bf16", "causal", False),
    (2, 9, 4, 1, 256, 32, [40, 650], "bf16", "f32", "full", False),
    (2, 30, 8, 2, 256, 64, [129, 512], "bf16", "bf16", "causal", True),
    (1, 64, 6, 1, 256, 16, [333], "bf16", "bf16", "tree", False),
    (1, 37, 3, 1, 128, 128, [4000], "bf16", "f32", "full", False),
])
def test_against_the_definition(R, N, h_q, h_kv, d, page, lens, dtype, out, mask, htd):
    c = _case(R, N, h_q, h_kv, d, page, lens, dtype, htd=htd, seed=R + N + d, slots=list(range(R, 0, -1)))
    if mask == "tree":
        parent = torch.tensor([[-1] + [(7 * n + r) % n for n in range(1, N)] for r in range(R)], dtype=torch.int32)
        mask = bd.bdgdn_tree_mask(parent.cuda())
    scale = 1 / math.sqrt(d)
    got = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"], mask=mask, slot=c["slot"],
                             out_dtype=DT[out], want_lse=True)
    _compare(c, got, mask, scale, dtype, out)


@pytest.mark.parametrize("dtype,scale", [("bf16", -0.11), ("f32", -0.2), ("bf16", 0.0), ("f32", 0.0), ("bf16", 1.0)])
def test_scales_of_any_sign(dtype, scale):
    c = _case(2, 6, 4, 2, 64, 16, [75, 20], dtype, seed=3)
    got = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"], mask="causal", scale=scale,
                             out_dtype=torch.float32, want_lse=True)
    _compare(c, got, "causal", scale, dtype, "f32")


def test_scores_that_grow_and_scores_far_apart():
    """Keys that grow along the sequence move the running maximum in every step."""
    c = _case(1, 4, 4, 2, 128, 16, [600], "bf16", seed=5)
    grow = torch.linspace(0.01, 6, 600, device="cuda")
    t = torch.arange(600, device="cuda")
    at = c["table"][0].long()[t // 16]
    c["kp"][at, t % 16] = (c["q"][0, 0, :1].float() * grow[:, None, None] / 8).expand(600, 2, 128).to(torch.bfloat16)
    got = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"], out_dtype=torch.float32,
                             want_lse=True)
    _compare(c, got, "full", 1 / math.sqrt(128), "bf16", "f32")


@pytest.mark.parametrize("dtype,h_q", [("bf16", 4), ("f32", 4), ("bf16", 16)])
@pytest.mark.parametrize("page", [16, 32, 20])
def test_nothing_unseen_enters(dtype, h_q, page):
    """Stale places, pages that are not there, refused nodes: NaN and infinities in all of them."""
    c = _case(3, 6, h_q, 2, 64, page, [5 * page + 3, 0, 2 * page], dtype, seed=9, max_pages=7)
    t = c["table"]
    for pool in (c["kp"], c["vp"]):
        used = torch.zeros(pool.shape[:2], dtype=torch.bool, device="cuda")
        for r, n in enumerate(c["lens"]):
            x = torch.arange(n, device="cuda")
            used[t[r].long()[x // page], x % page] = True
        gone = int(t[0, 2])
        used[gone] = False
        pool[~used] = float("nan")
    t[0, 2] = -1
    t[0, 3:5] = torch.tensor([c["kp"].shape[0], 2 ** 31 - 1])   # pages beyond the pool
    count = torch.tensor([4, 6, 0], dtype=torch.int32).cuda()
    c["k"][0, 4:], c["v"][0, 4:] = float("nan"), float("inf")
    words = torch.tensor([[1, 3, 1, 9, 63, 63], [0, 2, 6, 8, 1 << 40, 16], [1] * 6], dtype=torch.int64).cuda()
    c["v"][1, 5], c["k"][1, 5] = float("-inf"), float("nan")     # seen by nobody
    c["v"][1, 0, 0, 7], c["k"][1, 0] = float("nan"), 1e30         # seen by nobody either
    ws = torch.full((1 << 26,), 0x7f, dtype=torch.uint8, device="cuda").fill_(255)
    got = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], t, c["seq"], mask=words, count=count,
                             out_dtype=torch.float32, want_lse=True, workspace=ws)
    _compare(c, got, words, 1 / 8, dtype, "f32", count.tolist())
    assert torch.isinf(got[1][1, 0]).all() and torch.isinf(got[1][1, 4]).all()   # rows that see nothing


@pytest.mark.parametrize("dtype,page", [("bf16", 32), ("f32", 32), ("bf16", 20)])
def test_what_is_seen_is_not_hidden(dtype, page):
    """A node's NaN reaches the rows that see it, in its element alone, and no other row."""
    c = _case(1, 40, 2, 1, 128, page, [45], dtype, seed=2)
    c["v"][0, 3, 0, 17] = float("nan")
    c["v"][0, 35, 0, 99] = float("inf")
    o, lse = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"], mask="causal",
                                want_lse=True)
    bad = ~torch.isfinite(o[0]).all(1)   # [N, d]
    want = torch.zeros_like(bad)
    want[3:, 17] = True
    want[35:, 99] = True
    assert torch.equal(bad, want) and torch.isinf(o[0, 35:, :, 99]).all() and torch.isfinite(lse).all()


def test_parts_of_a_projection_and_lengths_past_the_table():
    """q, k, v as parts of one projection's rows; a length past the table counts as its end."""
    c = _case(3, 5, 4, 2, 128, 16, [48, 20, 31], "bf16", seed=4)
    whole = _case(3, 5, 8, 1, 128, 16, [1, 1, 1], "bf16", seed=6)["q"]
    c["q"], c["k"], c["v"] = whole[:, :, :4], whole[:, :, 4:6], whole[:, :, 6:]
    table = c["table"][:, :3].contiguous()
    seq = c["seq"].clone()
    seq[0] = 100000
    seq[1] = 20
    got = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], table, seq, mask="causal", want_lse=True)
    _compare(c, got, "causal", 1 / math.sqrt(128), "bf16", "bf16")


def test_offsets_past_32_bits():
    """Pages that lie more than 2^32 elements into a pool."""
    d, h, page, n_pages = 128, 8, 64, 70000   # 4.6e9 elements a pool
    pools = [torch.empty(n_pages, page, h, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    c = _case(1, 3, 8, 8, d, page, [130], "bf16", seed=8)
    high = torch.tensor([n_pages - 1, 66000, n_pages - 9], device="cuda")
    for pool, small in zip(pools, (c["kp"], c["vp"])):
        pool[high] = small[c["table"][0, :3].long()]
    want = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"])[0]
    table = high.to(torch.int32)[None].contiguous()
    got = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], *pools, table, c["seq"])[0]
    assert torch.equal(got, want)


def test_another_stream_and_a_replayed_graph():
    c = _case(4, 8, 8, 2, 128, 64, [100, 0, 900, 64], "bf16", seed=12)
    args = (c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"])
    want = bd.bdgdn_tree_attn(*args, mask="causal")[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o = torch.zeros_like(want)
    with torch.cuda.stream(side):
        bd.bdgdn_tree_attn(*args, mask="causal", o=o)
    side.synchronize()
    assert torch.equal(o, want)
    o.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bd.bdgdn_tree_attn(*args, mask="causal", o=o)
    for step in range(3):
        c["q"].mul_(0.9)
        want = bd.bdgdn_tree_attn(*args, mask="causal")[0].clone()
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want), step


@pytest.mark.parametrize("N", [1, 2, 13, 64])
def test_masks_of_trees(N):
    rng = torch.Generator().manual_seed(N)
    parent = torch.stack([torch.tensor([int(torch.randint(-1, max(n, 1), (1,), generator=rng)) for n in range(N)])
                          for _ in range(5)]).to(torch.int32)
    parent[1] = torch.arange(N) - 1           # a chain
    parent[2, N // 2] = N + 7                  # no such node: a root
    mask, depth = bd.bdgdn_tree_mask(parent.cuda(), want_depth=True)
    for r in range(5):
        for n in range(N):
            word, a, up = 0, n, 0
            while True:
                word |= 1 << a
                a2 = int(parent[r, a])
                if not 0 <= a2 < a:
                    break
                a, up = a2, up + 1
            assert int(mask[r, n]) & (2 ** 64 - 1) == word and int(depth[r, n]) == up


@pytest.fixture
def wide_tables(monkeypatch):
    """Cases whose tables have room for long requests, which are cut into pieces however short they are."""
    narrow = _case
    monkeypatch.setitem(globals(), "_case", lambda *args, **kw: narrow(*args, **{**kw, "max_pages": 700}))


@pytest.mark.parametrize("dtype,h_q", [("bf16", 4), ("f32", 4), ("bf16", 16)])
@pytest.mark.parametrize("page", [16, 32, 20])
def test_nothing_unseen_enters_from_wide_tables(wide_tables, dtype, h_q, page):
    test_nothing_unseen_enters(dtype, h_q, page)


@pytest.mark.parametrize("dtype,page", [("bf16", 32), ("f32", 32), ("bf16", 20)])
def test_what_is_seen_is_not_hidden_by_wide_tables(wide_tables, dtype, page):
    test_what_is_seen_is_not_hidden(dtype, page)


_SHORT = [
    (1, 1, 4, 1, 128, 16, [128], "bf16", "bf16", "full", False),
    (3, 8, 8, 2, 128, 16, [0, 127, 1], "bf16", "f32", "causal", True),
    (2, 16, 8, 2, 128, 32, [256, 200], "bf16", "bf16", "tree", False),
    (2, 17, 8, 2, 128, 32, [256, 33], "bf16", "bf16", "full", False),
    (2, 64, 16, 2, 64, 16, [111, 96], "bf16", "bf16", "causal", False),
    (2, 64, 8, 1, 256, 64, [64, 30], "bf16", "f32", "full", False),
    (2, 5, 6, 3, 256, 64, [128, 90], "bf16", "bf16", "causal", False),
    (2, 6, 4, 2, 128, 12, [120, 5], "bf16", "bf16", "tree", False),
    (2, 50, 8, 2, 64, 20, [100, 61], "bf16", "bf16", "full", False),
    (3, 7, 4, 2, 128, 24, [240, 0, 17], "f32", "f32", "tree", True),
    (1, 40, 8, 2, 256, 16, [128], "f32", "f32", "causal", False),
    (600, 2, 4, 2, 64, 16, [(53 * i) % 113 for i in range(600)], "bf16", "bf16", "causal", False),
]


@pytest.mark.parametrize("case", range(len(_SHORT)))
def test_short_requests(case):
    test_against_the_definition(*_SHORT[case])


@pytest.mark.parametrize("case", range(len(_SHORT)))
def test_short_requests_in_wide_tables(wide_tables, case):
    test_against_the_definition(*_SHORT[case])


def test_narrow_tables_with_lengths_past_their_end_and_odd_slots():
    """Lengths beyond the columns, negative ones, slots that are none."""
    c = _case(4, 5, 4, 2, 128, 16, [64, 20, 31, 64], "bf16", seed=4)
    table = c["table"][:, :4].contiguous()
    seq = torch.tensor([100000, 20, 31, 64], dtype=torch.int32).cuda()
    got = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], table, seq, mask="causal", want_lse=True)
    _compare(c, got, "causal", 1 / math.sqrt(128), "bf16", "bf16")
    seq[1] = -5
    slot = torch.tensor([0, 1, -1, 4], dtype=torch.int32).cuda()
    got = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], table, seq, mask="causal", want_lse=True, slot=slot)
    c["lens"] = [64, 0, 0, 0]
    _compare(c, got, "causal", 1 / math.sqrt(128), "bf16", "bf16")


@pytest.mark.parametrize("R,N,h_q,h_kv,d,page,lens,dtype,out,mask,htd", [
    # many rows to a key head over pages that are not whole runs of 16 tokens
    (2, 40, 8, 2, 128, 24, [700, 77], "bf16", "bf16", "causal", False),
    (1, 64, 8, 1, 128, 1, [450], "bf16", "f32", "tree", True),
    (2, 30, 8, 2, 256, 20, [129, 912], "bf16", "bf16", "full", False),
    (2, 11, 4, 1, 256, 100, [1300, 0], "bf16", "f32", "causal", True),
    (3, 12, 8, 2, 64, 36, [5, 700, 36], "bf16", "bf16", "tree", False),
    (1, 50, 8, 2, 64, 7, [333], "bf16", "f32", "causal", False),
    (2, 10, 4, 1, 128, 100, [1500, 99], "bf16", "bf16", "full", True),
    (90, 9, 4, 1, 128, 40, [(91 * i) % 390 for i in range(90)], "bf16", "bf16", "causal", False),
])
def test_many_rows_over_odd_pages(R, N, h_q, h_kv, d, page, lens, dtype, out, mask, htd):
    test_against_the_definition(R, N, h_q, h_kv, d, page, lens, dtype, out, mask, htd)


def test_expanded_inputs_are_refused():
    """One row for all requests, as a fork's first token has it: refused, and taken as a copy."""
    c = _case(4, 1, 8, 2, 128, 16, [40, 0, 7, 16], "bf16", seed=15)
    args = (c["kp"], c["vp"], c["table"], c["seq"])
    for name in ("q", "k", "v"):
        x = {n: c[n] for n in ("q", "k", "v")}
        x[name] = x[name][:1].expand(4, -1, -1, -1)
        with pytest.raises(ValueError, match=f"{name} must have"):
            bd.bdgdn_tree_attn(x["q"], x["k"], x["v"], *args)
        kept, c[name] = c[name], x[name].contiguous()
        _compare(c, bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], *args, want_lse=True), "full", 1 / math.sqrt(128), "bf16", "bf16")
        c[name] = kept


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("N,page", [(3, 32), (40, 32), (3, 20), (40, 20)])
def test_infinite_cached_values(dtype, out, N, page):
    """A weight above zero takes an infinity over as it is; infinities of both signs, and a NaN, give NaN.  The
    first key has the largest score of all rows, so that weights of exactly one are among them."""
    c = _case(1, N, 2, 1, 128, page, [75], dtype, seed=2, std=0.3)
    c["q"][...] = c["q"].abs() + 0.5
    at = [(int(c["table"][0, t // page]), t % page) for t in range(75)]
    c["kp"][at[0]] = 1.0
    for t, x, value in ((0, 5, "inf"), (31, 6, "-inf"), (70, 7, "inf"), (3, 8, "inf"), (9, 8, "-inf"), (44, 9, "nan")):
        c["vp"][at[t]][0, x] = float(value)
    o, lse = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"], out_dtype=DT[out],
                                want_lse=True)
    inf = float("inf")
    assert (o[..., 5] == inf).all() and (o[..., 6] == -inf).all() and (o[..., 7] == inf).all()
    assert torch.isnan(o[..., 8:10]).all() and torch.isfinite(lse).all()
    assert torch.isfinite(o[..., :5]).all() and torch.isfinite(o[..., 10:]).all()


@pytest.mark.parametrize("R,N,h_q,h_kv,d,page,lens,mask", [
    (1, 1, 4, 1, 128, 64, [300], "full"),
    (2, 8, 8, 2, 128, 16, [129, 1000], "causal"),
    (2, 32, 8, 2, 128, 64, [2049, 95], "full"),
    (2, 30, 8, 2, 64, 16, [700, 0], "causal"),
    (1, 9, 4, 1, 256, 32, [650], "full"),
    (2, 30, 8, 2, 256, 64, [129, 512], "causal"),
    (2, 3, 4, 2, 128, 24, [500, 33], "full"),
    (2, 40, 8, 2, 128, 24, [700, 77], "causal"),
])
def test_bf16_results_are_off_by_their_own_rounding(R, N, h_q, h_kv, d, page, lens, mask):
    """A bf16 output is an fp32 one rounded: 2^-8 |o| on top of the fp32 output's tolerance (above), which the
    rounding of the weights, in two parts, enters with 2^-16 A alone."""
    c = _case(R, N, h_q, h_kv, d, page, lens, "bf16", seed=R + N + d)
    o, _ = bd.bdgdn_tree_attn(c["q"], c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"], mask=mask)
    ro, _, A, S = _reference(c, mask, 1 / math.sqrt(d))
    tol = ((4 * (d + 8) * S + max(lens) + N + 64) * 2.0 ** -24 + 2.0 ** -16)[..., None] * A
    err = (o.double() - ro).abs()
    assert (err <= 2.0 ** -8 * (ro.abs() + tol) + tol).all(), float((err / (2.0 ** -8 * ro.abs() + tol)).max())
