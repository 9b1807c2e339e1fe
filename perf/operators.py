"""The operators that serve the softmax half of a hybrid backbone, as timed cases.

Beside the Gated DeltaNet layers, a serving round of the hybrid model attends with a block of new
nodes over a paged cache (``attn``), verifies drafted tokens against the target's logits from
given random numbers (``verify``), and keeps the cache's pages: rows of the accepted path go in
(``append``), sequences are forked (``fork``) and thinned out (``compact``).

A case is a dict of plain values.  ``prepare`` makes what the server holds before the call from the
seed alone; ``run`` is one pass, in plain torch or, with ``own`` set, through the framework's
entry points; ``exact`` is the definition in 64 bits.
"""
import math
import random

import torch

own = False


def listed():
    return [
        # One chat at a time: the next token of a single request, where the call's latency counts.
        dict(name="attn_one_token", op="attn", req=1, nodes=1, mask="full", h_q=32, h_kv=8, d=128, page=64,
             len_lo=1500, len_hi=1500, dtype="bf16", layout="thd"),
        # A loaded server's AR-Trust verify pass: the anchor and 7 drafts per request.
        dict(name="attn_verify_64", op="attn", req=64, nodes=8, mask="causal", h_q=32, h_kv=8, d=128, page=64,
             len_lo=101, len_hi=4096, dtype="bf16", layout="thd"),
        # The same server's Diffusion-Trust denoise pass: blocks of 32 that see themselves whole.
        dict(name="attn_denoise_64", op="attn", req=64, nodes=32, mask="full", h_q=32, h_kv=8, d=128, page=64,
             len_lo=101, len_hi=4096, dtype="bf16", layout="thd"),
        # Few requests with long documents: a tree of drafts over 128k tokens.
        dict(name="attn_tree_128k", op="attn", req=2, nodes=24, mask="tree", h_q=32, h_kv=8, d=128, page=64,
             len_lo=98765, len_hi=131072, dtype="bf16", layout="htd"),
        # Heads of 256 with few key heads, small pages.
        dict(name="attn_d256", op="attn", req=16, nodes=6, mask="tree", h_q=16, h_kv=2, d=256, page=16,
             len_lo=900, len_hi=8000, dtype="bf16", layout="thd"),
        # A developer's check in fp32 with odd sizes.
        dict(name="attn_f32_odd", op="attn", req=3, nodes=5, mask="tree", h_q=6, h_kv=2, d=64, page=24,
             len_lo=0, len_hi=1003, dtype="f32", layout="thd"),
        # One chat: a chain of 7 drafts sampled from the draft's distribution, an odd vocabulary.
        dict(name="verify_one", op="verify", req=1, nodes=8, shape="chain", vocab=32001, dtype="bf16",
             draft="sampled", temperature="one"),
        # A loaded server, a large vocabulary, some requests greedy.
        dict(name="verify_64", op="verify", req=64, nodes=8, shape="chain", vocab=131072, dtype="bf16",
             draft="sampled", temperature="mixed"),
        # Trees of the draft's most likely tokens, fp32 logits, an odd vocabulary.
        dict(name="verify_tree_point", op="verify", req=12, nodes=24, shape="tree", vocab=100003, dtype="f32",
             draft="point", temperature="mixed"),
        # The accepted paths' rows of 64 requests into the pages of 4 layers.
        dict(name="append_64", op="append", req=64, nodes=8, h_kv=8, d=128, page=64, pools=8, len_lo=33, len_hi=640,
             dtype="bf16"),
        # Best of several: prompts forked eight ways, the first token of each (pages copied on write).
        dict(name="fork_8x8", op="fork", req=8, ways=8, h_kv=8, d=128, page=64, pools=8, len_lo=500, len_hi=2000,
             dtype="bf16"),
        # Long sequences thinned out to the positions worth keeping.
        dict(name="compact_8", op="compact", req=8, h_kv=8, d=128, page=64, pools=4, len_lo=2500, len_hi=4096,
             keep=0.5, dtype="bf16"),
    ]


# What the largest listed cases move and compute: no drawn case costs more.
_MOST = {"attn": (1.0e9, 1.0e11), "verify": (3.0e8, 1e12), "pages": (2.0e8, 1e12)}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "verify", "verify", "append", "fork", "compact"])
    if op == "attn":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        d = rng.choice([64, 128, 128, 256])
        h_kv = rng.choice([1, 2, 3, 4, 8])
        hi = _log(rng, 20, 131072)
        case = dict(op=op, req=_log(rng, 1, 64), nodes=_log(rng, 1, 64), mask=rng.choice(["full", "causal", "tree"]),
                    h_q=h_kv * rng.choice([1, 2, 3, 4, 8]), h_kv=h_kv, d=d, page=rng.choice([16, 24, 32, 64, 100]),
                    len_lo=int(hi * rng.choice([0, 0.1, 0.5, 1])), len_hi=hi, dtype=dtype,
                    layout=rng.choice(["thd", "htd"]))
        most = _MOST["attn"]
        if dtype == "f32":   # fp32 stands for checks on small shapes
            most = (most[0] / 16, most[1] / 64)
    elif op == "verify":
        case = dict(op=op, req=_log(rng, 1, 64), nodes=rng.randint(2, 24), shape=rng.choice(["chain", "tree"]),
                    vocab=_log(rng, 1000, 131072), dtype=rng.choice(["bf16", "f32"]),
                    draft=rng.choice(["sampled", "point"]), temperature=rng.choice(["one", "mixed"]))
        most = _MOST["verify"]
    else:
        case = dict(op=op, req=_log(rng, 1, 64), h_kv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128, 256]),
                    page=rng.choice([16, 24, 32, 64, 100]), pools=2 * rng.randint(1, 4), len_lo=0,
                    len_hi=_log(rng, 30, 4096), dtype=rng.choice(["bf16", "bf16", "f32"]))
        if op == "append":
            case["nodes"] = _log(rng, 1, 64)
        elif op == "fork":
            case["ways"] = rng.randint(1, 8)
        else:
            case["keep"] = rng.choice([0.1, 0.5, 0.9])
        most = _MOST["pages"]
    for _ in range(40):
        w = work(case)
        if w["bytes"] <= most[0] and w["flops"] <= most[1] and _pool_bytes(case) <= 1.2e9:
            break
        if case["req"] > 1:
            case["req"] = case["req"] // 2
        elif op == "verify":
            case["nodes"] = max(2, case["nodes"] // 2)
        else:
            case["len_hi"] //= 2
            case["len_lo"] //= 2
    return case


_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}


def _lens(case):
    """The requests' cached lengths, spread evenly from len_lo to len_hi in a mixed order."""
    n, lo, hi = case["req"], case["len_lo"], case["len_hi"]
    if n == 1:
        return [hi]
    step = 7 if n % 7 else 1
    return [lo + (hi - lo) * ((step * i + 5) % n) // (n - 1) for i in range(n)]


def _pages_of(tokens, page):
    return (tokens + page - 1) // page


def _pool_bytes(case):
    if case["op"] == "verify":
        return 0
    tokens = sum(_lens(case)) + case["req"] * 2 * case["page"]
    copies = {"attn": 2, "append": case.get("pools", 0), "fork": case.get("pools", 0),
              "compact": 2 * case.get("pools", 0)}[case["op"]]
    tokens += case["req"] * case.get("ways", 0) * case["page"]
    return copies * tokens * case["h_kv"] * case["d"] * _SIZE[case["dtype"]]


def _parents(case, seed):
    """Parent of every node: a chain, or random trees with the root 0."""
    R, N = case["req"], case["nodes"]
    rng = random.Random(seed * 7919 + 17)
    if case.get("shape") == "chain" or case.get("mask") == "causal":
        rows = [[max(n - 1, 0) for n in range(N)] for _ in range(R)]
    else:
        rows = [[0] + [rng.randint(max(0, n - 5), n - 1) for n in range(1, N)] for _ in range(R)]
    for row in rows:
        row[0] = -1
    return rows


def work(case):
    op, size = case["op"], _SIZE[case["dtype"]]
    if op == "attn":
        R, N, lens = case["req"], case["nodes"], _lens(case)
        row = case["d"] * size
        seen = {"full": N * N, "causal": N * (N + 1) // 2, "tree": 4 * N}[case["mask"]]
        return {"bytes": row * (2 * R * N * case["h_q"] + 2 * case["h_kv"] * (sum(lens) + R * N))
                + 4 * R * N * case["h_q"],
                "flops": 4 * case["d"] * case["h_q"] * (N * sum(lens) + R * seen)}
    if op == "verify":
        R, N, V = case["req"], case["nodes"], case["vocab"]
        inner = (N - 1 if case["shape"] == "chain" else max(1, N // 2)) if case["draft"] == "sampled" else 0
        return {"bytes": R * V * (size * (N + inner) + 4), "flops": 4 * R * V * (N + inner)}
    row = case["pools"] * case["h_kv"] * case["d"] * size
    if op == "append":
        return {"bytes": 2 * row * sum(_append_counts(case)), "flops": 0}
    if op == "fork":   # one row of each way, and the shared page's rows before it
        lens = _lens(case)
        return {"bytes": 2 * row * case["ways"] * sum(1 + n % case["page"] for n in lens), "flops": 0}
    return {"bytes": 2 * row * sum(_kept(case)), "flops": 0}


def _append_counts(case):
    return [1 + (5 * i + 2) % case["nodes"] for i in range(case["req"])]


def _kept(case):
    return [int(case["keep"] * n) for n in _lens(case)]


# ------------------------------------------------------------------ what the server holds
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tables(slots, lens, page, max_pages, n_pages, order):
    """page_table, seq_len, refcount and free bits of sequences laid on the pages of ``order``."""
    table = torch.full((slots, max_pages), -1, dtype=torch.int32)
    refcount = torch.zeros(n_pages, dtype=torch.int32)
    at = 0
    for r, n in enumerate(lens):
        k = _pages_of(n, page)
        table[r, :k] = order[at:at + k]
        at += k
    refcount[order[:at].long()] = 1
    seq_len = torch.zeros(slots, dtype=torch.int32)
    seq_len[:len(lens)] = torch.tensor(lens, dtype=torch.int32)
    return [t.cuda() for t in (table, seq_len, refcount)]


def _pack_bits(refcount):
    """Bit p % 32 of word p // 32 is set where page p is free."""
    free = torch.zeros((refcount.numel() + 31) // 32 * 32, dtype=torch.int64, device=refcount.device)
    free[:refcount.numel()] = refcount == 0
    words = (free.view(-1, 32) << torch.arange(32, device=free.device)).sum(1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def _prepare_attn(case, seed):
    g, dt = _gen(seed), _DT[case["dtype"]]
    R, N, h_q, h_kv, d, page = (case[k] for k in ("req", "nodes", "h_q", "h_kv", "d", "page"))
    lens = _lens(case)
    max_pages = max(1, _pages_of(max(lens), page))
    n_pages = sum(_pages_of(n, page) for n in lens) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table, seq_len, _ = _tables(R, lens, page, max_pages, n_pages, order)
    s = dict(case=case, lens=lens, table=table, seq_len=seq_len, scale=1 / math.sqrt(d))

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(0, std, generator=g)

    # Scores of standard deviation 2: some keys stand out, as trained heads have them.
    s["q"], s["k"], s["v"] = normal(R, N, h_q, d, std=2.0), normal(R, N, h_kv, d), normal(R, N, h_kv, d)
    if case["layout"] == "thd":
        s["kp"], s["vp"] = normal(n_pages, page, h_kv, d), normal(n_pages, page, h_kv, d)
    else:
        s["kp"], s["vp"] = (normal(n_pages, h_kv, page, d).transpose(1, 2) for _ in range(2))
    if case["mask"] == "tree":
        s["parent_host"] = _parents(case, seed)
        s["parent"] = torch.tensor(s["parent_host"], dtype=torch.int32).cuda()
    return s


def _prepare_verify(case, seed):
    g, dt = _gen(seed), _DT[case["dtype"]]
    R, N, V = case["req"], case["nodes"], case["vocab"]
    parents = _parents(case, seed)
    # A target of a few hundred likely tokens, and a draft that is near it.
    target = torch.empty(R, N, V, dtype=dt, device="cuda").normal_(0, 2.5, generator=g)
    temperature = torch.tensor([1.0 if case["temperature"] == "one" else (1.0, 0.7, 0.0, 0.9)[r % 4]
                                for r in range(R)], device="cuda")
    parent = torch.tensor(parents, dtype=torch.int32).cuda()
    draft = torch.empty_like(target)
    token = torch.zeros(R, N, dtype=torch.int32, device="cuda")
    for n in range(N):
        draft[:, n] = (target[:, n].float()
                       + torch.empty(R, V, device="cuda").normal_(0, 0.7, generator=g)).to(dt)
    temp = torch.where(temperature > 0, temperature, torch.ones_like(temperature))[:, None]
    which = [[row[:n].count(row[n]) for n in range(N)] for row in parents]
    for n in range(1, N):
        rows = draft[torch.arange(R, device="cuda"), parent[:, n].long()].float()
        if case["draft"] == "sampled":
            race = torch.softmax(rows / temp, -1) / torch.empty(R, V, device="cuda").exponential_(generator=g)
            token[:, n] = race.argmax(-1).to(torch.int32)
        else:   # the child's rank among its parent's most likely tokens
            top = torch.topk(rows, min(N, V), dim=-1).indices
            rank = torch.tensor([w[n] for w in which], device="cuda")
            token[:, n] = top.gather(1, rank[:, None])[:, 0].to(torch.int32)
    u = torch.rand(R, N, device="cuda", generator=g)
    noise = torch.empty(R, V, device="cuda").exponential_(generator=g)
    return dict(case=case, target=target, draft=draft if case["draft"] == "sampled" else None, token=token,
                parent=None if case["shape"] == "chain" else parent, parent_host=parents, temperature=temperature,
                u=u, noise=noise)


def _prepare_pages(case, seed):
    g, dt, op = _gen(seed), _DT[case["dtype"]], case["op"]
    R, h_kv, d, page, pools = (case[k] for k in ("req", "h_kv", "d", "page", "pools"))
    lens = _lens(case)
    W = case.get("ways", 1)
    spare = {"append": R * (_pages_of(case.get("nodes", 0), page) + 1), "fork": R * W * 2,
             "compact": sum(_pages_of(n, page) for n in lens) + R}[op]
    n_pages = sum(_pages_of(n, page) for n in lens) + spare + 5
    max_pages = _pages_of(max(lens) + case.get("nodes", 1) + 1, page)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    slots = R if op == "append" else R * (1 + W)
    table, seq_len, refcount = _tables(slots, lens, page, max_pages, n_pages, order)
    # One page more than the cache has: where the plain form's masked writes go.
    pool = torch.empty(pools, n_pages + 1, page, h_kv, d, dtype=dt, device="cuda").normal_(generator=g)
    s = dict(case=case, lens=lens, table=table, seq_len=seq_len, refcount=refcount, bits=_pack_bits(refcount),
             pool=pool, views=[pool[i, :n_pages] for i in range(pools)])

    def ints(values):
        return torch.tensor(values, dtype=torch.int32).cuda()

    if op == "append":
        N, rng = case["nodes"], random.Random(seed)
        counts = _append_counts(case)
        s["slot"], s["before"], s["count"] = ints(list(range(R))[::-1]), ints(lens[::-1]), ints(counts)
        s["path"] = ints([sorted(rng.sample(range(N), c)) + [-1] * (N - c) for c in counts])
        s["rows"] = torch.empty(pools, R, N, h_kv, d, dtype=dt, device="cuda").normal_(generator=g)
    else:
        s["src"] = ints([i // W for i in range(R * W)])
        s["dst"] = s["slot"] = ints([R + i for i in range(R * W)])
        s["zero"] = torch.zeros_like(s["dst"])
    if op == "fork":
        s["count"] = torch.ones_like(s["dst"])
        s["rows"] = torch.empty(pools, R * W, 1, h_kv, d, dtype=dt, device="cuda").normal_(generator=g)
    if op == "compact":
        rng, kept = random.Random(seed), _kept(case)
        most = max(max(kept), 1)
        s["keep"] = ints([sorted(rng.sample(range(n), k)) + [-1] * (most - k) for n, k in zip(lens, kept)])
        s["count"] = ints(kept)
    s["row_views"] = [s["rows"][i] for i in range(pools)] if "rows" in s else None
    return s


def prepare(case, seed):
    if case["op"] == "attn":
        return _prepare_attn(case, seed)
    return _prepare_verify(case, seed) if case["op"] == "verify" else _prepare_pages(case, seed)


# ------------------------------------------------------------------ one pass, plain
def _plain_mask(parent):
    """Which node sees which: itself and its ancestors, bit j of word n."""
    R, N = parent.shape
    sees = torch.zeros(R, N, N, dtype=torch.bool, device=parent.device)
    rows = torch.arange(R, device=parent.device)
    for n in range(N):
        p = parent[:, n].long()
        ok = (p >= 0) & (p < n)
        sees[:, n] = sees[rows, p.clamp(0, N - 1)] & ok[:, None]
        sees[:, n, n] = True
    return sees, (sees.long() << torch.arange(N, device=parent.device)).sum(-1)


def _plain_attn(s):
    case = s["case"]
    R, N, h_q, h_kv, d, page = (case[k] for k in ("req", "nodes", "h_q", "h_kv", "d", "page"))
    q, G = s["q"], h_q // h_kv
    o = torch.empty(R, N, h_q, d, device=q.device)
    lse = torch.empty(R, N, h_q, device=q.device)
    bits = None
    if case["mask"] == "tree":
        sees, bits = _plain_mask(s["parent"])
    else:
        sees = torch.ones(N, N, dtype=torch.bool, device=q.device)
        sees = (sees.tril() if case["mask"] == "causal" else sees).expand(R, N, N)
    for r in range(R):
        n = s["lens"][r]
        idx = s["table"][r, :_pages_of(n, page)].long()
        kc = s["kp"][idx].reshape(-1, h_kv, d)[:n]
        vc = s["vp"][idx].reshape(-1, h_kv, d)[:n]
        keys = torch.cat([kc, s["k"][r]]).float().permute(1, 2, 0).contiguous()      # [h_kv, d, n + N]
        vals = torch.cat([vc, s["v"][r]]).float().permute(1, 0, 2).contiguous()      # [h_kv, n + N, d]
        rows = q[r].float().view(N, h_kv, G, d).permute(1, 0, 2, 3).reshape(h_kv, N * G, d)
        score = torch.matmul(rows, keys) * s["scale"]
        hide = ~sees[r].repeat_interleave(G, 0)
        score[:, :, n:] = score[:, :, n:].masked_fill(hide, -math.inf)
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - top)
        total = e.sum(-1, keepdim=True)
        out = torch.matmul(e, vals) / total
        o[r] = out.view(h_kv, N, G, d).permute(1, 0, 2, 3).reshape(N, h_q, d)
        lse[r] = (top + torch.log(total)).view(h_kv, N, G).permute(1, 0, 2).reshape(N, h_q)
    out = (o.to(q.dtype), lse)
    return out if bits is None else (*out, bits)


def _softmax_rows(x, temperature):
    """softmax(x / T) of every row in fp32; T <= 0 is all on the largest entry (the first of equals)."""
    V = x.shape[-1]
    x = x.float()
    T = temperature.view(-1, *[1] * (x.dim() - 1))
    z = x / torch.where(T > 0, T, torch.ones_like(T))
    e = torch.exp(z - z.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    index = torch.arange(V, device=x.device)
    first = torch.where(x == x.amax(-1, keepdim=True), index, V).amin(-1, keepdim=True)
    return torch.where(T > 0, p, (index == first).float())


def _plain_verify(s):
    case = s["case"]
    R, N, V = case["req"], case["nodes"], case["vocab"]
    dev, token = s["target"].device, s["token"].long()
    sampled = s["draft"] is not None
    p = _softmax_rows(s["target"], s["temperature"])
    # (a greedy request takes the target's first choice alone, whatever the draft thought of it)
    q = _softmax_rows(s["draft"], s["temperature"]) * (s["temperature"] > 0).view(-1, 1, 1) if sampled else None
    parent = s["parent"].long() if s["parent"] is not None else torch.arange(-1, N - 1, device=dev).expand(R, N)
    rows, zero = torch.arange(R, device=dev), torch.zeros(R, device=dev)
    cur = torch.zeros(R, dtype=torch.long, device=dev)
    c, mass = zero.clone(), zero + 1
    res = p[:, 0].clone()
    count = torch.zeros(R, dtype=torch.long, device=dev)
    path = torch.full((R, N), -1, dtype=torch.long, device=dev)
    path[:, 0] = 0
    for n in range(1, N):
        here = parent[:, n] == cur
        tok = token[:, n]
        left = res.gather(1, tok[:, None])[:, 0]
        odds = q[rows, cur].gather(1, tok[:, None])[:, 0] if sampled else torch.ones_like(left)
        taken = here & (s["u"][:, n] * mass * odds < left)
        refused = here & ~taken
        count += taken
        path.scatter_(1, torch.where(taken, count, 0)[:, None],
                      torch.where(taken, n, path.gather(1, torch.where(taken, count, 0)[:, None])[:, 0])[:, None])
        cur = torch.where(taken, n, cur)
        if sampled:
            c = torch.where(taken, zero, torch.where(refused, c + mass, c))
            res = torch.clamp(p[rows, cur] - c[:, None] * q[rows, cur], min=0)
        else:
            gone = torch.arange(V, device=dev) == tok[:, None]
            res = torch.where(taken[:, None], p[rows, cur], torch.where(refused[:, None] & gone, 0.0, res))
        mass = torch.where(taken, zero + 1, torch.where(refused, res.sum(-1), mass))
    last = p[rows, cur]
    res = torch.where(res.amax(-1, keepdim=True) > 0, res, last)
    score = res / s["noise"]
    best = score.amax(-1, keepdim=True)
    index = torch.arange(V, device=dev)
    nxt = torch.where((score == best) & (best > 0), index, V).amin(-1)
    nxt = torch.where(nxt == V, -1, nxt)
    return count.to(torch.int32), path.to(torch.int32), nxt.to(torch.int32)


def _plain_free(s):
    """The free pages, lowest first."""
    n = s["refcount"].numel()
    free = s["refcount"] == 0
    rank = torch.where(free, torch.cumsum(free, 0) - 1, n)
    index = torch.arange(n, device=free.device)
    return torch.zeros(n + 1, dtype=torch.long, device=free.device).scatter_(0, rank, index)


def _plain_truncate(s, slot, length):
    page, slot = s["case"]["page"], slot.long()
    now = s["seq_len"][slot]
    new = torch.minimum(now, length)
    col = torch.arange(s["table"].shape[1], device=slot.device)
    gone = (col < _pages_of(now, page)[:, None]) & (col >= _pages_of(new, page)[:, None])
    rows = s["table"][slot]
    s["refcount"].index_add_(0, rows.clamp(min=0).flatten().long(), -gone.to(torch.int32).flatten())
    s["table"][slot] = torch.where(gone, -1, rows)
    s["seq_len"][slot] = new


def _plain_fork(s, src, dst):
    page = s["case"]["page"]
    rows, n = s["table"][src.long()], s["seq_len"][src.long()]
    held = torch.arange(rows.shape[1], device=src.device) < _pages_of(n, page)[:, None]
    s["refcount"].index_add_(0, rows.clamp(min=0).flatten().long(), held.to(torch.int32).flatten())
    s["table"][dst.long()] = torch.where(held, rows, -1)
    s["seq_len"][dst.long()] = n


def _plain_append(s, slot, rows, count, path=None):
    page, pool, slot = s["case"]["page"], s["pool"], slot.long()
    R, N = rows.shape[1:3]
    dev, dummy = slot.device, pool.shape[1] - 1
    old, table = s["seq_len"][slot], s["table"][slot]
    first = _pages_of(old, page)
    last = table.gather(1, (first - 1).clamp(min=0)[:, None].long())[:, 0]
    shared = (old % page > 0) & (count > 0) & (s["refcount"][last.clamp(min=0).long()] > 1)
    start = first - shared.int()
    need = _pages_of(old + count, page) - start
    offset = torch.cumsum(need, 0) - need
    col = torch.arange(table.shape[1], device=dev)
    fresh = (col >= start[:, None]) & (col < (start + need)[:, None])
    take = torch.where(fresh, offset[:, None] + col - start[:, None], 0)
    table = torch.where(fresh, _plain_free(s)[take].to(torch.int32), table)
    # the rows of a shared last page, then the new ones
    tok = torch.arange(page, device=dev)
    copied = shared[:, None] & (tok < (old % page)[:, None])
    at = table.gather(1, start[:, None].clamp(max=table.shape[1] - 1).long())
    pool[:, torch.where(copied, at, dummy).long(), tok] = pool[:, torch.where(copied, last[:, None], dummy).long(), tok]
    j = torch.arange(N, device=dev)
    new = j < count[:, None]
    pos = torch.where(new, old[:, None] + j, 0)
    node = j.expand(R, N) if path is None else torch.where(new, path, 0).long()
    at = torch.where(new, table.gather(1, (pos // page).long()), dummy)
    pool[:, at.long(), (pos % page).long()] = rows[:, torch.arange(R, device=dev)[:, None], node]
    s["refcount"].index_add_(0, last.clamp(min=0).long(), -shared.int())
    s["refcount"].index_add_(0, torch.where(fresh, table, 0).flatten().long(), fresh.to(torch.int32).flatten())
    s["table"][slot] = table
    s["seq_len"][slot] = old + count
    return torch.zeros_like(count)


def _plain_compact(s, slot, keep, count):
    page, pool, slot = s["case"]["page"], s["pool"], slot.long()
    dev, dummy = slot.device, pool.shape[1] - 1
    old, table = s["seq_len"][slot], s["table"][slot]
    j = torch.arange(keep.shape[1], device=dev)
    kept = j < count[:, None]
    stay = ((keep == j) & kept).sum(1).int()                # positions that do not move
    start = torch.where(stay == count, _pages_of(stay, page), stay // page)
    need = _pages_of(count, page) - start
    offset = torch.cumsum(need, 0) - need
    col = torch.arange(table.shape[1], device=dev)
    fresh = (col >= start[:, None]) & (col < (start + need)[:, None])
    take = torch.where(fresh, offset[:, None] + col - start[:, None], 0)
    new = torch.where(fresh, _plain_free(s)[take].to(torch.int32), torch.where(col < start[:, None], table, -1))
    moved = kept & (j >= (start * page)[:, None])
    src = torch.where(moved, keep, 0)
    frm = torch.where(moved, table.gather(1, (src // page).long()), dummy)
    to = torch.where(moved, new.gather(1, (j // page).expand_as(keep).clamp(max=new.shape[1] - 1)), dummy)
    pool[:, to.long(), (j % page).expand_as(keep)] = pool[:, frm.long(), (src % page).long()]
    gone = (col >= start[:, None]) & (col < _pages_of(old, page)[:, None])
    s["refcount"].index_add_(0, table.clamp(min=0).flatten().long(), -gone.to(torch.int32).flatten())
    s["refcount"].index_add_(0, torch.where(fresh, new, 0).flatten().long(), fresh.to(torch.int32).flatten())
    s["table"][slot] = new
    s["seq_len"][slot] = count
    return torch.zeros_like(count)


def _plain_pages(s):
    op = s["case"]["op"]
    if op == "append":   # the round before is taken back, then this one's rows go in
        _plain_truncate(s, s["slot"], s["before"])
        status = _plain_append(s, s["slot"], s["rows"], s["count"], s["path"])
    else:
        _plain_truncate(s, s["dst"], s["zero"])
        _plain_fork(s, s["src"], s["dst"])
        status = (_plain_append(s, s["dst"], s["rows"], s["count"]) if op == "fork" else
                  _plain_compact(s, s["dst"], s["keep"], s["count"]))
    s["bits"].copy_(_pack_bits(s["refcount"]))
    return s["pool"][:, :-1], s["table"], s["seq_len"], s["refcount"], s["bits"], status


# ------------------------------------------------------------------ one pass, the framework's
def _own(s):
    import paper_2606_01774_amd as bd

    op = s["case"]["op"]
    if op == "attn":
        kind = s["case"]["mask"]
        bits = bd.bdgdn_tree_mask(s["parent"]) if kind == "tree" else None
        out = bd.bdgdn_tree_attn(s["q"], s["k"], s["v"], s["kp"], s["vp"], s["table"], s["seq_len"],
                                 mask=bits if kind == "tree" else kind, scale=s["scale"], out_dtype=s["q"].dtype,
                                 want_lse=True)
        return out if bits is None else (*out, bits)
    if op == "verify":
        return bd.bdgdn_verify(s["target"], s["token"], s["u"], s["noise"], draft=s["draft"], parent=s["parent"],
                               temperature=s["temperature"])
    tables = bd.CacheTables(s["table"], s["seq_len"], s["refcount"], s["bits"])
    if op == "append":
        bd.bdgdn_cache_truncate(tables, s["slot"], s["before"], page=s["case"]["page"])
        status = bd.bdgdn_cache_append(tables, s["views"], s["row_views"], s["slot"], s["count"], path=s["path"])
    else:
        bd.bdgdn_cache_truncate(tables, s["dst"], s["zero"], page=s["case"]["page"])
        bd.bdgdn_cache_fork(tables, s["src"], s["dst"], page=s["case"]["page"])
        status = (bd.bdgdn_cache_append(tables, s["views"], s["row_views"], s["dst"], s["count"]) if op == "fork" else
                  bd.bdgdn_cache_compact(tables, s["views"], s["dst"], s["keep"], s["count"]))
    return s["pool"][:, :-1], s["table"], s["seq_len"], s["refcount"], s["bits"], status


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_attn(state) if op == "attn" else _plain_verify(state) if op == "verify" else _plain_pages(state)


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_attn(case, seed):
    s = _prepare_attn(case, seed)
    R, N, h_q, h_kv, d, page = (case[k] for k in ("req", "nodes", "h_q", "h_kv", "d", "page"))
    G = h_q // h_kv
    o = torch.zeros(R, N, h_q, d, dtype=torch.float64, device="cuda")
    lse = torch.full((R, N, h_q), -math.inf, dtype=torch.float64, device="cuda")
    tree = case["mask"] == "tree"
    words = torch.zeros(R, N, dtype=torch.int64)
    for r in range(R):
        sees = torch.zeros(N, N, dtype=torch.bool)
        for n in range(N):
            if tree:   # climb to the root
                a = n
                while a >= 0:
                    sees[n, a] = True
                    words[r, n] |= 1 << a
                    a = s["parent_host"][r][a]
            else:
                sees[n, :(n + 1 if case["mask"] == "causal" else N)] = True
        sees = sees.cuda()
        t = torch.arange(s["lens"][r], device="cuda")
        at = s["table"][r].long()[t // page]
        for h in range(h_kv):
            keys = torch.cat([s["kp"][at, t % page, h], s["k"][r, :, h]]).double()
            vals = torch.cat([s["vp"][at, t % page, h], s["v"][r, :, h]]).double()
            rows = s["q"][r, :, h * G:(h + 1) * G].double().reshape(N * G, d)
            score = (rows @ keys.T.contiguous()) * s["scale"]
            score[:, len(t):][~sees.repeat_interleave(G, 0)] = -math.inf
            z = torch.logsumexp(score, -1)
            o[r, :, h * G:(h + 1) * G] = (torch.exp(score - z[:, None]) @ vals).view(N, G, d)
            lse[r, :, h * G:(h + 1) * G] = z.view(N, G)
    return (o, lse, words.cuda()) if tree else (o, lse)


def _exact_verify(case, seed):
    s = _prepare_verify(case, seed)
    R, N = case["req"], case["nodes"]
    count, path, nxt = torch.zeros(R, dtype=torch.int32), torch.full((R, N), -1, dtype=torch.int32), []

    def law(x, T):
        x = x.double()
        if T > 0:
            return torch.softmax(x / T, -1)
        return torch.zeros_like(x).index_fill_(0, (x == x.max()).nonzero()[0], 1.0)

    for r in range(R):
        T = float(s["temperature"][r])
        tok, u = s["token"][r].tolist(), s["u"][r].double().tolist()
        cur, steps = 0, 0
        path[r, 0] = 0
        while True:
            left = law(s["target"][r, cur], T)
            whole = left
            prop = None if s["draft"] is None else law(s["draft"][r, cur], T) * (T > 0)
            for n in [n for n in range(cur + 1, N) if s["parent_host"][r][n] == cur]:
                odds = 1.0 if prop is None else float(prop[tok[n]])
                if u[n] * odds < float(left[tok[n]]):
                    cur, steps = n, steps + 1
                    path[r, steps] = n
                    break
                if prop is None:
                    left = left.clone()
                    left[tok[n]] = 0
                else:
                    left = (left - prop).clamp(min=0)
                if float(left.sum()) > 0:
                    left = left / left.sum()
            else:
                break
        count[r] = steps
        score = (left if float(left.max()) > 0 else whole) / s["noise"][r].double()
        nxt.append(int((score == score.max()).nonzero()[0, 0]) if float(score.max()) > 0 else -1)
    return count.cuda(), path.cuda(), torch.tensor(nxt, dtype=torch.int32).cuda()


def _exact_pages(case, seed):
    """The round on lists: sequences as lists of (page, place), one after the other."""
    s = _prepare_pages(case, seed)
    page, op, pool = case["page"], case["op"], s["pool"][:, :-1].double()
    table, lens = s["table"].tolist(), s["seq_len"].tolist()
    refs = s["refcount"].tolist()
    before = list(refs)
    free = [p for p, n in enumerate(refs) if n == 0]
    source = pool.clone()
    count = s["count"].tolist()

    def put(cols, rows, at):   # rows [pools, n, h_kv, d] to the positions from ``at`` on
        for j in range(rows.shape[1]):
            pool[:, cols[(at + j) // page], (at + j) % page] = rows[:, j]

    if op != "append":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            table[b], lens[b] = list(table[a]), lens[a]
            for p in table[b][:_pages_of(lens[b], page)]:
                refs[p] += 1
        before = list(refs)
    for i, b in enumerate(s["slot"].tolist()):
        n, k = lens[b], count[i]
        cols = table[b][:_pages_of(n, page)]
        if op == "compact":
            keep = s["keep"][i, :k].tolist()
            still = next((j for j, t in enumerate(keep) if t != j), k)
            whole = _pages_of(k, page) if still == k else still // page
            for p in cols[whole:]:
                refs[p] -= 1
            where = [(cols[t // page], t % page) for t in keep[whole * page:]]
            cols, n = cols[:whole], min(whole * page, k)
            rows = source[:, [w[0] for w in where], [w[1] for w in where]]
        else:
            path = s["path"][i, :k].tolist() if op == "append" else [0] * k
            rows = s["rows"][:, i, path].double()
            if n % page and k and before[cols[-1]] > 1:   # a page that others read too
                old = cols.pop()
                refs[old] -= 1
                rows = torch.cat([source[:, old, :n % page], rows], 1)
                n -= n % page
        end = n + rows.shape[1]
        while len(cols) < _pages_of(end, page):
            cols.append(free.pop(0))
            refs[cols[-1]] = 1
        put(cols, rows, n)
        table[b], lens[b] = cols + [-1] * (len(table[b]) - len(cols)), end
    refcount = torch.tensor(refs, dtype=torch.int32).cuda()
    return (pool, torch.tensor(table, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
            refcount, _pack_bits(refcount), torch.zeros(len(count), dtype=torch.int32).cuda())


def exact(case, seed):
    if case["op"] == "attn":
        return _exact_attn(case, seed)
    return _exact_verify(case, seed) if case["op"] == "verify" else _exact_pages(case, seed)
