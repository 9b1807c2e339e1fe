"""The operators around the mixers of a hybrid layer and in front of verification, as timed cases.

``rope`` turns queries and keys by their positions, ``norm`` and ``norm_bwd`` are the norms after
and before a mixer with its gate, scale and residual, ``project`` is a product of 8-bit integers
whose activations are quantised on the way, ``logits`` applies penalties for repeated tokens,
biases and the grammar's mask to the rows that the verification reads.

A case is a dict of plain values.  ``prepare`` makes what the program holds before the call from the
seed alone; ``run`` is one pass, in plain torch or, with ``own`` set, through the framework's entry
points; ``exact`` is the definition in 64 bits.
"""
import math
import random

import torch

own = False


def listed():
    return [
        # One chat at a time: q and k of the next token, behind 1500 cached ones; latency counts.
        dict(name="rope_one_token", op="rope", req=1, nodes=1, h_q=32, h_k=8, d=128, rot=128, layout="half",
             scaling="none", where="cache", far=1500, inverse=False, dtype="bf16"),
        # A training step's attention layer, q and k of 4 x 4096 tokens, positions stretched eight times.
        dict(name="rope_train", op="rope", req=4, nodes=4096, h_q=32, h_k=8, d=128, rot=128, layout="half",
             scaling="parts", where="row", far=0, inverse=False, dtype="bf16"),
        # The gradient of packed documents' rotation, a quarter of each head, neighbours as pairs, fp32.
        dict(name="rope_packed_grad", op="rope", req=1, nodes=32749, h_q=6, h_k=2, d=64, rot=16, layout="pairs",
             scaling="none", where="packed", far=1000000, inverse=True, dtype="f32"),
        # One chat: the norms between two blocks of a layer for one token.
        dict(name="norm_one_token", op="norm", outer=1, inner=1, d=4096, post=True, pre=True, gate="none",
             layer_scale=False, residual=True, x="f32", r="f32", y="bf16"),
        # A training step: 4 x 4096 tokens, the mixer's output normed, gated, scaled, added, normed again.
        dict(name="norm_block", op="norm", outer=16384, inner=1, d=4096, post=True, pre=True, gate="silu",
             layer_scale=True, residual=True, x="bf16", r="f32", y="bf16"),
        # The same block's backward pass.
        dict(name="norm_block_bwd", op="norm_bwd", outer=16384, inner=1, d=4096, post=True, pre=True, gate="silu",
             layer_scale=True, residual=True, x="bf16", r="f32", y="bf16"),
        # The gated norm behind the Gated DeltaNet: 4 x 4096 tokens, 16 heads of 128, fp32 outputs of the mixer.
        dict(name="norm_heads_bwd", op="norm_bwd", outer=16384, inner=16, d=128, post=True, pre=False, gate="silu",
             layer_scale=False, residual=False, x="f32", r="f32", y="bf16"),
        # One chat's round: the anchor and 7 drafts, an odd vocabulary, a grammar.
        dict(name="logits_one", op="logits", req=1, nodes=8, vocab=32001, shape="chain", penalties=True, biases=20,
             allow="node", x="bf16", y="bf16"),
        # A loaded server's round over a large vocabulary.
        dict(name="logits_64", op="logits", req=64, nodes=8, vocab=131072, shape="tree", penalties=True, biases=300,
             allow="node", x="bf16", y="bf16"),
        # The next token of a few chats: the weights are what there is to read.
        dict(name="project_3", op="project", m=3, n=8192, k=4096, bias=False, x="bf16", y="bf16"),
        # A round of 64 requests with 8 nodes each.
        dict(name="project_512", op="project", m=512, n=6144, k=2048, bias=True, x="bf16", y="bf16"),
        # A prompt's tokens, an odd number of them.
        dict(name="project_prompt", op="project", m=8191, n=8192, k=4096, bias=False, x="bf16", y="bf16"),
    ]


# What the largest listed cases move and compute: no drawn case costs more.
_MOST = {"rope": (3.4e8, 1e15), "norm": (9.4e8, 1e15), "norm_bwd": (1.4e9, 1e15), "logits": (3.1e8, 1e15),
         "project": (2.0e8, 5.5e11)}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "norm", "norm", "norm_bwd", "norm_bwd", "logits", "logits", "project", "project"])
    if op == "rope":
        where = rng.choice(["cache", "cache", "row", "packed"])
        d = rng.choice([64, 80, 128, 128, 256])
        h_k = rng.choice([0, 1, 2, 4, 8])
        case = dict(op=op, req=1 if where == "packed" else _log(rng, 1, 64),
                    nodes=_log(rng, 1, 64) if where == "cache" else _log(rng, 100, 32768),
                    h_q=max(h_k, 1) * rng.choice([1, 2, 3, 4, 8]), h_k=h_k, d=d,
                    rot=rng.choice([d, d, d // 2, d // 4, 10]), layout=rng.choice(["half", "pairs"]),
                    scaling=rng.choice(["none", "linear", "ntk", "parts"]), where=where, far=_log(rng, 1000, 1000000),
                    inverse=rng.choice([True, False]), dtype=rng.choice(["bf16", "bf16", "f32"]))
        sizes = ("nodes", "req")
    elif op in ("norm", "norm_bwd"):
        heads = rng.random() < 0.4
        types = rng.choice([("bf16", "f32", "bf16"), ("bf16", "bf16", "bf16"), ("f32", "f32", "bf16"), ("f32", "f32", "f32")])
        post, residual = rng.choice([True, False]), not heads and rng.random() < 0.8
        case = dict(op=op, outer=_log(rng, 1, 32768), inner=rng.choice([1, 2, 5, 16, 32]) if heads else 1,
                    d=rng.choice([64, 128, 256, 100]) if heads else _log(rng, 100, 8192), post=post or heads,
                    pre=not heads and (not post or rng.random() < 0.7), gate=rng.choice(["none", "silu", "sigmoid"]),
                    layer_scale=rng.choice([True, False]) and not heads, residual=residual, x=types[0], r=types[1], y=types[2])
        if rng.random() < 0.7:
            case["d"] = max(8, case["d"] // 8 * 8)
        sizes = ("outer",)
    elif op == "logits":
        x, y = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
        case = dict(op=op, req=_log(rng, 1, 64), nodes=rng.choice([1, 1, 2, 8, 13, 24]), vocab=_log(rng, 1000, 131072),
                    shape=rng.choice(["chain", "tree"]), penalties=rng.random() < 0.8, biases=rng.choice([0, 0, 7, 300]),
                    allow=rng.choice(["none", "request", "node"]), x=x, y=y)
        sizes = ("req", "nodes")
    else:
        case = dict(op=op, m=_log(rng, 1, 8192), n=_log(rng, 64, 16384), k=_log(rng, 64, 16384), bias=rng.choice([True, False]),
                    x=rng.choice(["bf16", "bf16", "f32"]), y=rng.choice(["bf16", "bf16", "f32"]))
        if rng.random() < 0.7:
            case["n"], case["k"] = max(16, case["n"] // 16 * 16), max(64, case["k"] // 64 * 64)
        sizes = ("m", "n")
    for turn in range(80):
        w = work(case)
        if w["bytes"] <= _MOST[op][0] and w["flops"] <= _MOST[op][1]:
            break
        key = sizes[turn % len(sizes)]
        case[key] = max(1, case[key] // 2)
    return case


_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
_EPS = 1e-6


def work(case):
    op = case["op"]
    if op == "rope":
        n = case["req"] * case["nodes"] * (case["h_q"] + case["h_k"])
        return {"bytes": 2 * n * case["d"] * _SIZE[case["dtype"]], "flops": 3 * n * case["rot"]}
    if op in ("norm", "norm_bwd"):
        n = case["outer"] * case["inner"] * case["d"]
        x, r, y, gate = _SIZE[case["x"]], _SIZE[case["r"]], _SIZE[case["y"]], case["gate"] != "none"
        if op == "norm":
            return {"bytes": n * (x + y + gate * y + 2 * r * case["residual"]), "flops": 12 * n}
        return {"bytes": n * (2 * x + y + 2 * gate * y + 3 * r * case["residual"]), "flops": 30 * n}
    if op == "logits":
        R, N, V = case["req"], case["nodes"], case["vocab"]
        masks = {"none": 0, "request": R, "node": R * N}[case["allow"]]
        return {"bytes": R * N * V * (_SIZE[case["x"]] + _SIZE[case["y"]]) + 4 * R * V * case["penalties"]
                + masks * ((V + 31) // 32) * 4 + 8 * R * case["biases"], "flops": 6 * R * N * V}
    M, N, K = case["m"], case["n"], case["k"]
    return {"bytes": M * K * _SIZE[case["x"]] + N * K + M * N * _SIZE[case["y"]] + 4 * N, "flops": 2 * M * N * K}


# ------------------------------------------------------------------ what the program holds
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, dtype, *shape, std=1.0):
    return torch.empty(shape, dtype=_DT[dtype], device="cuda").normal_(0, std, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _frequencies(case):
    """Radians a position of each pair, and what the rotated elements are multiplied with.  Long
    contexts: positions divided by 8 (linear), a larger base (ntk), or divided only where a pair
    turns seldom within the original length (parts)."""
    rot, base, factor, original = case["rot"], 10000.0, 8.0, 8192.0
    if case["scaling"] == "ntk":
        base *= factor ** (rot / (rot - 2))
    w = [base ** (-2 * i / rot) for i in range(rot // 2)]
    if case["scaling"] == "linear":
        w = [f / factor for f in w]
    if case["scaling"] == "parts":
        keep = [min(max((original * f / (2 * math.pi) - 1) / 31, 0.0), 1.0) for f in w]
        w = [f * a + f / factor * (1 - a) for f, a in zip(w, keep)]
        return w, 0.1 * math.log(factor) + 1
    return w, 1.0


def _prepare_rope(case, seed):
    g, rng = _gen(seed), random.Random(seed)
    R, N, h_q, h_k, d = (case[k] for k in ("req", "nodes", "h_q", "h_k", "d"))
    w, scale = _frequencies(case)
    # fractions of a turn a position, in units of 2^-64 (as signed words)
    turns = [int(f / (2 * math.pi) * 2.0 ** 64) for f in w]
    s = dict(case=case, w=torch.tensor(w, dtype=torch.float64).cuda(), scale=scale,
             turns=torch.tensor([t - (1 << 64) if t >= 1 << 63 else t for t in turns], dtype=torch.int64).cuda(),
             slot=None, seq_len=None, pos=None)
    # q and k are parts of the rows of one projection, which holds the values too
    rows = _normal(g, case["dtype"], R, N, h_q + 2 * h_k, d)
    s["q"], s["k"] = rows[:, :, :h_q], rows[:, :, h_q:h_q + h_k] if h_k else None
    if case["where"] == "cache":   # a tree's or a block's nodes behind their sequences
        s["seq_len"] = _ints([rng.randint(case["far"] // 2, case["far"]) for _ in range(R + 3)])
        s["slot"] = _ints(rng.sample(range(R + 3), R))
        s["pos"] = _ints([[rng.randint((n + 1) // 2, n) for n in range(N)] for _ in range(R)])
    elif case["where"] == "packed":   # documents one behind the other, some of them a long file's later part
        at, pos = 0, []
        while at < N:
            n = min(rng.randint(1, 8000), N - at)
            first = rng.choice([0, rng.randint(0, case["far"])])
            pos += range(first, first + n)
            at += n
        s["pos"] = _ints([pos])
    return s


def _prepare_norm(case, seed):
    g = _gen(seed)
    A, B, d, back = case["outer"], case["inner"], case["d"], case["op"] == "norm_bwd"
    s = dict(case=case, scale=0.7 if case["layer_scale"] else 1.0)
    s["x"] = _normal(g, case["x"], A, B, d, std=1.5)
    # the gate is the second half of a projection's rows
    s["z"] = _normal(g, case["y"], A, 2, B, d)[:, 1] if case["gate"] != "none" else None
    s["r"] = _normal(g, case["r"], A, B, d, std=3.0) if case["residual"] else None   # (the new residual, for the backward)

    def weight(there):
        return 1 + 0.2 * torch.empty(d, device="cuda").normal_(generator=g) if there else None

    s["w_post"], s["w_pre"], s["layer_scale"] = weight(case["post"]), weight(case["pre"]), weight(case["layer_scale"])
    if back:
        s["dy"] = _normal(g, case["y"], A, B, d)
        s["dr"] = _normal(g, case["r"], A, B, d) if case["residual"] else None
    return s


def _prepare_logits(case, seed):
    g, rng = _gen(seed), random.Random(seed)
    R, N, V, K = case["req"], case["nodes"], case["vocab"], case["biases"]
    s = dict(case=case, logits=_normal(g, case["x"], R, N, V, std=2.5))
    s["parent"] = [[-1] + [n - 1 if case["shape"] == "chain" else rng.randint(max(0, n - 5), n - 1) for n in range(1, N)]
                   for _ in range(R)]
    words = [[0] * N for _ in range(R)]
    for r in range(R):
        for n in range(N):
            up = s["parent"][r][n]
            words[r][n] = (words[r][up] if up >= 0 else 0) | 1 << n
    s["words"] = torch.tensor(words, dtype=torch.int64).cuda()
    s["token"] = _ints([[rng.randrange(V) for _ in range(N)] for _ in range(R)])
    s["token"][:, -1] = s["token"][:, 0]   # (a token that comes twice)
    s["history"] = s["repetition"] = s["presence"] = s["frequency"] = s["bias"] = s["bias_token"] = s["allow"] = None
    s["slot"] = _ints(rng.sample(range(R + 2), R))
    if case["penalties"]:
        # some hundreds of generated tokens and thousands of prompt ones (bit 30) in each sequence
        s["history"] = torch.zeros(R + 2, V, dtype=torch.int32, device="cuda")
        said = torch.randint(V, (R + 2, 400), generator=g, device="cuda")
        s["history"].scatter_add_(1, said, torch.ones_like(said, dtype=torch.int32))
        prompt = torch.randint(V, (R + 2, 2000), generator=g, device="cuda")
        s["history"].scatter_(1, prompt, s["history"].gather(1, prompt) | 1 << 30)
        s["repetition"] = torch.tensor([(1.1, 1.0, 1.3)[r % 3] for r in range(R)], device="cuda")
        s["presence"] = torch.tensor([(0.0, 0.5)[r % 2] for r in range(R)], device="cuda")
        s["frequency"] = torch.tensor([(0.2, 0.0, -0.1)[r % 3] for r in range(R)], device="cuda")
    if K:
        s["bias_token"] = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(R)]).to(torch.int32)
        s["bias"] = torch.empty(R, K, device="cuda").normal_(0, 4, generator=g)
    if case["allow"] != "none":
        shape = (R, N if case["allow"] == "node" else 1, (V + 31) // 32)
        s["allow"] = torch.randint(-2 ** 31, 2 ** 31, shape, generator=g, device="cuda").to(torch.int32)
    return s


def _prepare_project(case, seed):
    g = _gen(seed)
    M, N, K = case["m"], case["n"], case["k"]
    s = dict(case=case, x=_normal(g, case["x"], M, K, std=1.3))
    # weights as a checkpoint holds them: rows of integers, filled up with zeros to a multiple of 128
    s["w"] = torch.zeros(N, -(-K // 128) * 128, dtype=torch.int8, device="cuda")
    s["w"][:, :K] = torch.randint(-127, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    s["w_scale"] = torch.empty(N, device="cuda").uniform_(0.5, 2, generator=g) / (73 * math.sqrt(K))
    s["bias"] = torch.empty(N, device="cuda").normal_(generator=g) if case["bias"] else None
    return s


def prepare(case, seed):
    make = {"rope": _prepare_rope, "norm": _prepare_norm, "norm_bwd": _prepare_norm, "logits": _prepare_logits,
            "project": _prepare_project}
    return make[case["op"]](case, seed)


# ------------------------------------------------------------------ one pass, plain
def _plain_rope(s):
    case = s["case"]
    R, N, rot = case["req"], case["nodes"], case["rot"]
    p = s["pos"].double() if s["pos"] is not None else torch.arange(N, device="cuda", dtype=torch.float64).expand(R, N)
    if s["seq_len"] is not None:
        p = p + s["seq_len"][s["slot"].long()].double()[:, None]
    angle = p[:, :, None, None] * s["w"]        # 64 bits: far positions
    if case["inverse"]:
        angle = -angle
    cos, sin = torch.cos(angle).float() * s["scale"], torch.sin(angle).float() * s["scale"]
    outs = []
    for x in (s["q"], s["k"]):
        if x is None:
            continue
        f = x.float()
        if case["layout"] == "half":
            a, b = f[..., :rot // 2], f[..., rot // 2:rot]
            turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        else:
            a, b = f[..., 0:rot:2], f[..., 1:rot:2]
            turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        outs.append(torch.cat([turned, f[..., rot:]], -1).to(x.dtype))
    return outs


def _act(z, kind):
    """act(z) and its derivative."""
    e = 1 / (1 + torch.exp(-z))
    return (e, e * (1 - e)) if kind == "sigmoid" else (z * e, e * (1 + z * (1 - e)))


def _plain_norm(s):
    case = s["case"]
    n = s["x"].float()
    if case["post"]:
        n = n * torch.rsqrt((n * n).mean(-1, keepdim=True) + _EPS) * s["w_post"]
    if s["z"] is not None:
        n = n * _act(s["z"].float(), case["gate"])[0]
    n = n * s["scale"]
    if case["layer_scale"]:
        n = n * s["layer_scale"]
    if s["r"] is not None:
        n = s["r"].float() + n
    y = n * torch.rsqrt((n * n).mean(-1, keepdim=True) + _EPS) * s["w_pre"] if case["pre"] else n
    y = y.to(_DT[case["y"]])
    return (y, n.to(s["r"].dtype)) if s["r"] is not None else (y,)


def _plain_norm_bwd(s):
    case = s["case"]
    rows = (0, 1)
    x, dy = s["x"].float(), s["dy"].float()
    if case["post"]:
        s1 = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
        xh = x * s1
        n = xh * s["w_post"]
    else:
        n = x
    act, slope = _act(s["z"].float(), case["gate"]) if s["z"] is not None else (None, None)
    u = n if act is None else n * act
    if s["r"] is not None:
        new = s["r"].float()
    else:
        new = u * s["scale"] * (s["layer_scale"] if case["layer_scale"] else 1)
    dw_pre = dw_post = dls = dz = None
    if case["pre"]:
        s2 = torch.rsqrt((new * new).mean(-1, keepdim=True) + _EPS)
        h = new * s2
        dw_pre = (dy * h).sum(rows)
        t = dy * s["w_pre"]
        g = s2 * (t - h * (t * h).mean(-1, keepdim=True))
    else:
        g = dy
    if s["dr"] is not None:
        g = g + s["dr"].float()
    dr = g.to(s["r"].dtype) if s["r"] is not None else None
    du = g * s["scale"]
    if case["layer_scale"]:
        dls = (du * u).sum(rows)
        du = du * s["layer_scale"]
    if act is not None:
        dz = (du * n * slope).to(s["z"].dtype)
        du = du * act
    if case["post"]:
        dw_post = (du * xh).sum(rows)
        t = du * s["w_post"]
        du = s1 * (t - xh * (t * xh).mean(-1, keepdim=True))
    return du.to(s["x"].dtype), dz, dr, dw_post, dw_pre, dls


def _plain_logits(s):
    case = s["case"]
    R, N, V = case["req"], case["nodes"], case["vocab"]
    x = s["logits"].float()
    if case["penalties"]:
        words = s["history"][s["slot"].long()]
        sees = (s["words"][:, :, None] >> torch.arange(N, device="cuda")) & 1           # [R, N, N]
        count = (words & (1 << 30) - 1)[:, None].repeat(1, N, 1)
        count.scatter_add_(2, s["token"].long()[:, None].expand(R, N, N), sees.to(torch.int32))
        seen = (count > 0) | ((words >> 30) & 1).bool()[:, None]
        rho = s["repetition"][:, None, None]
        x = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x)
        x = x - (count > 0) * s["presence"][:, None, None] - count * s["frequency"][:, None, None]
    if s["bias"] is not None:
        x = x.scatter_add(2, s["bias_token"].long()[:, None].expand(R, N, -1), s["bias"][:, None].expand(R, N, -1))
    if s["allow"] is not None:
        bit = (s["allow"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bit.flatten(-2)[..., :V].bool(), x, -math.inf)
    return x.to(_DT[case["y"]])


def _plain_project(s):
    K = s["case"]["k"]
    x = s["x"].float()
    scale = x.abs().amax(-1, keepdim=True) / 127
    q = torch.clamp(torch.round(x / scale), -127, 127)
    y = torch.matmul(q, s["w"][:, :K].float().T) * scale * s["w_scale"]
    return (y if s["bias"] is None else y + s["bias"]).to(_DT[s["case"]["y"]])


# ------------------------------------------------------------------ one pass, the framework's
def _own(s):
    import paper_2606_01774_amd as bd

    case = s["case"]
    op = case["op"]
    if op == "rope":
        out = bd.bdgdn_rope(s["q"], s["turns"], s["k"], pos=s["pos"], seq_len=s["seq_len"], slot=s["slot"],
                            layout=case["layout"], scale=s["scale"], inverse=case["inverse"])
        return [out] if s["k"] is None else list(out)
    if op == "norm":
        y, r = bd.bdgdn_norm_fwd(s["x"], z=s["z"], r=s["r"], w_post=s["w_post"], w_pre=s["w_pre"],
                                 layer_scale=s["layer_scale"], post=case["post"], pre=case["pre"],
                                 act=case["gate"], scale=s["scale"], eps=_EPS, out_dtype=_DT[case["y"]])
        return (y,) if r is None else (y, r)
    if op == "norm_bwd":
        return bd.bdgdn_norm_bwd(s["x"], s["dy"], z=s["z"], r_out=s["r"], dr_out=s["dr"], w_post=s["w_post"],
                                 w_pre=s["w_pre"], layer_scale=s["layer_scale"], post=case["post"], pre=case["pre"],
                                 act=case["gate"], scale=s["scale"], eps=_EPS)
    if op == "logits":
        return bd.bdgdn_logits(s["logits"], token=s["token"], mask=s["words"], history=s["history"], slot=s["slot"],
                               repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                               bias_token=s["bias_token"], bias=s["bias"], allow=s["allow"], out_dtype=_DT[case["y"]])
    q, scale = bd.bdgdn_quant_rows(s["x"])
    return bd.bdgdn_quant_matmul(q, scale, s["w"], s["w_scale"], bias=s["bias"], out_dtype=_DT[case["y"]])


def run(state):
    if own:
        return _own(state)
    plain = {"rope": _plain_rope, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "logits": _plain_logits,
             "project": _plain_project}
    return plain[state["case"]["op"]](state)


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_rope(s):
    """Pairs as complex numbers, multiplied by scale e^(i p w), a head at a time."""
    case = s["case"]
    R, N, rot = case["req"], case["nodes"], case["rot"]
    p = torch.arange(N, device="cuda").expand(R, N) if s["pos"] is None else s["pos"].long()
    if s["seq_len"] is not None:
        p = p + s["seq_len"].long()[s["slot"].long()].unsqueeze(1)
    turn = torch.polar(torch.full((R, N, rot // 2), s["scale"], dtype=torch.float64, device="cuda"),
                       p.double().unsqueeze(-1) * s["w"])
    if case["inverse"]:
        turn = turn.conj()
    at = torch.arange(rot, device="cuda").view(-1, 2).T if case["layout"] == "pairs" else torch.arange(rot, device="cuda").view(2, -1)
    outs = []
    for x in (s["q"], s["k"]):
        if x is not None:
            y = x.double()
            for h in range(x.shape[2]):
                c = torch.complex(y[:, :, h, at[0]], y[:, :, h, at[1]]) * turn
                y[:, :, h, at[0]], y[:, :, h, at[1]] = c.real, c.imag
            outs.append(y)
    return outs


def _exact_norm(s):
    """In pieces of rows; the backward is what differentiating the forward pass leaves."""
    case = s["case"]
    A, d, back = case["outer"], case["d"], case["op"] == "norm_bwd"
    par = {k: s[k].double().requires_grad_(back) for k in ("w_post", "w_pre", "layer_scale") if s[k] is not None}
    outs = []

    def normed(t, w):
        return t / (t.square().mean(-1, keepdim=True) + _EPS).sqrt() * w

    for a in range(0, A, 2048):
        x = s["x"][a:a + 2048].double().requires_grad_(back)
        z = None if s["z"] is None else s["z"][a:a + 2048].double().requires_grad_(back)
        u = normed(x, par["w_post"]) if case["post"] else x
        if z is not None:
            u = u * (torch.sigmoid(z) if case["gate"] == "sigmoid" else z * torch.sigmoid(z))
        u = u * s["scale"] * par.get("layer_scale", 1.0)
        if s["r"] is None:
            new = u
        elif back:   # the residual that makes the sum what the backward is given
            r = (s["r"][a:a + 2048].double() - u.detach()).requires_grad_(True)
            new = r + u
        else:
            new = s["r"][a:a + 2048].double() + u
        y = normed(new, par["w_pre"]) if case["pre"] else new
        if not back:
            outs.append((y, new) if s["r"] is not None else (y,))
            continue
        loss = (y * s["dy"][a:a + 2048].double()).sum()
        if s["dr"] is not None:
            loss = loss + (new * s["dr"][a:a + 2048].double()).sum()
        loss.backward()
        outs.append((x.grad, None if z is None else z.grad, None if s["r"] is None else r.grad))
    whole = [None if part[0] is None else torch.cat(part) for part in zip(*outs)]
    return tuple(whole) if not back else (*whole, *(par[k].grad if k in par else None for k in ("w_post", "w_pre", "layer_scale")))


def _exact_logits(s):
    """Token by token on lists of what each node has before it, on top of the untouched logits."""
    case = s["case"]
    R, N, V = case["req"], case["nodes"], case["vocab"]
    out = s["logits"].double()
    token = s["token"].tolist()
    for r in range(R):
        word = s["history"][int(s["slot"][r])].long() if case["penalties"] else None
        for n in range(N):
            row = out[r, n]
            if word is not None:
                count = word % 2 ** 30
                a = n
                while a >= 0:   # climb to the root
                    count[token[r][a]] += 1
                    a = s["parent"][r][a]
                rho = float(s["repetition"][r])
                before = (count > 0) | (word >= 2 ** 30)
                row = torch.where(before & (row > 0), row / rho, torch.where(before, row * rho, row))
                row = row - float(s["frequency"][r]) * count - float(s["presence"][r]) * (count > 0).double()
            if s["bias"] is not None:
                row[s["bias_token"][r].long()] += s["bias"][r].double()
            if s["allow"] is not None:
                v = torch.arange(V, device="cuda")
                words = s["allow"][r, n if case["allow"] == "node" else 0].long() % 2 ** 32
                row = row.masked_fill((words[v // 32] >> v % 32) % 2 == 0, -math.inf)
            out[r, n] = row
    return out


def _exact_project(s):
    x, K = s["x"].double(), s["case"]["k"]
    top = x.abs().amax(-1, keepdim=True)
    # (the steps that each number is rounded to are those of the quotient in 32 bits)
    q = torch.round(s["x"].float() / (s["x"].float().abs().amax(-1, keepdim=True) / 127)).double()
    y = torch.empty(x.shape[0], s["w"].shape[0], dtype=torch.float64, device="cuda")
    for a in range(0, y.shape[1], 2048):
        y[:, a:a + 2048] = (q @ s["w"][a:a + 2048, :K].double().T.contiguous()) * (top / 127) * s["w_scale"][a:a + 2048].double()
    return y if s["bias"] is None else y + s["bias"].double()


def exact(case, seed):
    define = {"rope": _exact_rope, "norm": _exact_norm, "norm_bwd": _exact_norm, "logits": _exact_logits,
              "project": _exact_project}
    return define[case["op"]](prepare(case, seed))
