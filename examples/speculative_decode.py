"""Speculative decoding of a small hybrid model: AR-Trust serving rounds with every call on the
device.

The model has random weights: an embedding, layers "g" (Gated DeltaNet) and "a" (softmax attention over
a paged cache), an output projection.  Its drafter is the model without its layers.  A round
drafts a chain behind each request's last token, runs the block through the layers
(bdgdn_commit_record, bdgdn_tree_attn), decides (bdgdn_verify) and keeps what was accepted
(bdgdn_accept_states, bdgdn_cache_append); nothing of it waits for the host.  Prompts are forked
several ways (bdgdn_cache_fork), a window keeps the caches short (bdgdn_cache_compact), and
finished sequences give their pages back (bdgdn_cache_truncate).  A model without "g" layers
can also draft trees (bdgdn_tree_mask).  The residual and its norms are bdgdn_norm_fwd's; on request the
attention layers turn their queries and keys by their positions (bdgdn_rope), the projections are in 8-bit
integers (bdgdn_quant_rows, bdgdn_quant_matmul), and repeated tokens are penalised (bdgdn_logits,
bdgdn_history_add).

    python examples/speculative_decode.py --prompts 8 --ways 4 --rounds 64
    python examples/speculative_decode.py --layers aa --tree 3,2,1 --temperature 0
    python examples/speculative_decode.py --rotary 10000 --eight-bit --repetition 1.1
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2606_01774_amd as bd  # noqa: E402

GDN_HEADS, GDN_DIM = 2, 128
HEADS, KV_HEADS, DIM = 4, 2, 64


def norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


def parents_of(branches):
    """The parents of a tree whose nodes at depth i have branches[i] children each, and for each
    node its place among its siblings."""
    parent, place, level = [-1], [0], [0]
    for width in branches:
        grown = []
        for n in level:
            for j in range(width):
                grown.append(len(parent))
                parent.append(n)
                place.append(j)
        level = grown
    return parent, place


class Decoder:
    """The model with the states and caches of `slots` sequences of up to max_len tokens.  rotary: the
    base of the attention layers' positions (None: they have none); eight_bit: projections in 8-bit
    integers; penalties: (repetition, presence, frequency) of tokens that a sequence holds already (the last
    two: that it has generated)."""

    def __init__(self, layers="gaga", vocab=512, width=256, slots=32, page=16, max_len=1024, pages=None, seed=0,
                 device="cuda", rotary=None, eight_bit=False, penalties=None):
        gen = torch.Generator().manual_seed(seed)

        def weight(rows, cols):
            w = torch.randn(rows, cols, generator=gen) * rows ** -0.5
            return w.to(device, torch.bfloat16)

        self.layers, self.vocab, self.device = layers, vocab, device
        self.embed = torch.randn(vocab, width, generator=gen).to(device, torch.bfloat16)
        self.out = weight(width, vocab)
        qkv = {"g": 3 * GDN_HEADS * GDN_DIM + 2 * GDN_HEADS, "a": (HEADS + 2 * KV_HEADS) * DIM}
        back = {"g": GDN_HEADS * GDN_DIM, "a": HEADS * DIM}
        self.w_in = [weight(width, qkv[x]) for x in layers]
        self.w_out = [weight(back[x], width) for x in layers]
        # rows of integers with a scale for each channel
        self.eight_bit = [[bd.bdgdn_quant_rows(w.T.contiguous()) for w in ws] for ws in (self.w_in, self.w_out)] if eight_bit else None
        self.turns = None if rotary is None else bd.make_rope_turns(DIM, rotary, device=device)[0]
        # tokens that a sequence has taken in (a window shortens its cache, not its positions)
        self.taken = torch.zeros(slots, dtype=torch.int32, device=device)
        self.penalties = penalties
        self.history = torch.zeros(slots, vocab, dtype=torch.int32, device=device) if penalties else None
        # sequences whose next anchor is a prompt's token (its last: the model has not taken it in yet)
        self.prompted = torch.zeros(slots, dtype=torch.bool, device=device) if penalties else None
        self.drafter = self.logits(self.embed.float())   # [V, V]: after each token
        self.states = [torch.zeros(slots, GDN_HEADS, GDN_DIM, GDN_DIM, device=device) if x == "g" else None
                       for x in layers]
        max_pages = -(-max_len // page)
        self.page, n_pages = page, slots * max_pages if pages is None else pages
        self.tables = bd.make_cache_tables(slots, max_pages, n_pages, device=device, page=page)
        self.pools = [torch.zeros(n_pages, page, KV_HEADS, DIM, dtype=torch.bfloat16, device=device)
                      for _ in range(2 * layers.count("a"))]   # keys, values of each "a"

    def logits(self, x):
        return (norm(x).to(torch.bfloat16) @ self.out).float()

    def project(self, x, out, i):
        """Rows [R * N, .] through the projection in front of layer i, or behind it (out 1)."""
        if self.eight_bit is None:
            return x @ (self.w_in, self.w_out)[out][i]
        return bd.bdgdn_quant_matmul(*bd.bdgdn_quant_rows(x), *self.eight_bit[out][i])

    def forward(self, token, slot, mask="causal", depth=None, n_record=0):
        """Logits [R, N, V] of a block of tokens behind the sequences in `slot`, the attention
        layers' new rows, and with n_record the recorded states of the "g" layers.  The "g"
        layers' states go forward by the whole block, the caches stay as they are.  depth: the
        nodes' positions behind the sequence (None: 0, 1, ...)."""
        R, N = token.shape
        x = self.embed[token.long()].float().view(R * N, -1)
        z, _ = bd.bdgdn_norm_fwd(x, pre=True, out_dtype=torch.bfloat16)
        rows, recorded, a = [], [], 0
        for i, kind in enumerate(self.layers):
            y = self.project(z, 0, i).view(R, N, -1)
            if kind == "g":
                q, k, v, rest = y.split([GDN_HEADS * GDN_DIM] * 3 + [2 * GDN_HEADS], dim=-1)
                q, k, v = (t.reshape(R, N, GDN_HEADS, GDN_DIM) for t in (q, k, v))
                q, k = (F.normalize(t.float(), dim=-1).to(torch.bfloat16) for t in (q, k))
                g, beta = rest.float().split(GDN_HEADS, dim=-1)
                args = (self.states[i], q, k, v.contiguous(), -F.softplus(g).contiguous(),
                        torch.sigmoid(beta).contiguous())
                if n_record:
                    kept, o = bd.bdgdn_commit_record(*args, n_record=n_record, slot=slot, want_o=True,
                                                     out_dtype=torch.bfloat16)
                    recorded.append(kept)
                else:
                    o = bd.bdgdn_commit(*args, slot=slot, want_o=True, out_dtype=torch.bfloat16)
                    recorded.append(None)
            else:
                y = y.view(R, N, HEADS + 2 * KV_HEADS, DIM)   # q, k and v as parts of its rows
                q, k, v = y.split([HEADS, KV_HEADS, KV_HEADS], dim=2)
                if self.turns is not None:
                    q, k = bd.bdgdn_rope(q, self.turns, k, pos=depth, seq_len=self.taken, slot=slot, q_out=q, k_out=k)
                o, _ = bd.bdgdn_tree_attn(q, k, v, self.pools[a], self.pools[a + 1], self.tables.page_table,
                                          self.tables.seq_len, mask=mask, slot=slot)
                rows += [k, v]
                recorded.append(None)
                a += 2
            z, x = bd.bdgdn_norm_fwd(self.project(o.reshape(R * N, -1), 1, i), r=x, pre=True, r_out=x)
        return (z @ self.out).float().view(R, N, -1), rows, recorded

    def append(self, rows, slot, count, path=None):
        """(status, how many tokens each sequence has taken in: none where the cache has refused them)."""
        if rows:
            status = bd.bdgdn_cache_append(self.tables, self.pools, rows, slot, count, path=path)
        else:
            status = torch.zeros_like(count)
        kept = torch.where(status == bd.BDGDN_CACHE_DONE, count, 0)
        self.taken.index_add_(0, slot.long(), kept)
        return status, kept

    def prefill(self, prompt, slot, block=32, whole=False):
        """Takes in prompt [R, T] but its last token, which is the first round's anchor.  whole: that token is the
        prompt's too; else it counts as generated, like the anchors behind it.  A request whose status
        is not BDGDN_CACHE_DONE has taken in a part: it is to be finished."""
        status = torch.zeros_like(slot)
        if self.penalties:
            self.prompted[slot.long()] = whole
            bd.bdgdn_history_add(self.history, (prompt if whole else prompt[:, :-1]).contiguous(), slot=slot, prompt=True)
        for t in range(0, prompt.shape[1] - 1, block):
            part = prompt[:, t:min(t + block, prompt.shape[1] - 1)]
            _, rows, _ = self.forward(part, slot)
            status |= self.append(rows, slot, torch.full_like(slot, part.shape[1]))[0]
        return prompt[:, -1], status

    def fork(self, src, dst):
        """Gives slots dst the sequences of src; a slot whose status is not BDGDN_CACHE_DONE stays as it was."""
        status = bd.bdgdn_cache_fork(self.tables, src, dst)
        done, src, dst = status == bd.BDGDN_CACHE_DONE, src.long(), dst.long()
        for t in (*self.states, self.taken, self.prompted, self.history):
            if t is not None:
                t[dst] = torch.where(done.view(-1, *[1] * (t.dim() - 1)), t[src], t[dst])
        return status

    def _draft(self, logits, temperature):
        if temperature <= 0:
            return logits.argmax(-1)
        p = torch.softmax(logits / temperature, -1)
        return (p / torch.empty_like(p).exponential_()).argmax(-1)

    def _verify(self, target, token, generated, slot, temperature, mask=None, **kw):
        R, N, V = target.shape
        if self.penalties:
            repetition, presence, frequency = (torch.full((R,), float(p), device=self.device) for p in self.penalties)
            bd.bdgdn_logits(target, token=generated, mask=mask, history=self.history, slot=slot, repetition=repetition,
                            presence=presence, frequency=frequency, out=target)
        u = torch.rand(R, N, device=self.device)
        noise = torch.empty(R, V, device=self.device).exponential_()
        T = torch.full((R,), float(temperature), device=self.device)
        return bd.bdgdn_verify(target, token, u, noise, temperature=T, want_n_path=True, **kw)

    def _generated(self, token, slot):
        """A block's tokens as the penalties count them (-1 counts for nothing: the history has marked a prompt's)."""
        if not self.penalties:
            return None
        token = token.clone()
        token[:, 0].masked_fill_(self.prompted[slot.long()], -1)
        return token

    def _keep(self, rows, recorded, generated, slot, path, n_path):
        """The sequences take in the accepted path of a block, in their caches, states and histories; those that
        the cache refuses stay as they were before it, and the block may be tried again."""
        status, kept = self.append(rows, slot, n_path, path)
        for state, states in zip(self.states, recorded):
            if states is not None:
                bd.bdgdn_accept_states(state, states, kept, block=path.shape[1], slot=slot)
        if self.penalties:
            bd.bdgdn_history_add(self.history, generated, slot=slot, path=path, count=kept)
            self.prompted[slot.long()] &= kept == 0
        return status

    def round(self, anchor, slot, drafts=7, temperature=1.0):
        """One round with a drafted chain.  Returns (tokens [R, 1 + drafts] of the block,
        n_accept, the next anchor, status).  A request whose status is not BDGDN_CACHE_DONE has taken in
        nothing: it goes on with the anchor that it came with."""
        token = [anchor]
        for _ in range(drafts):
            token.append(self._draft(self.drafter[token[-1].long()], temperature).to(torch.int32))
        token = torch.stack(token, 1)
        draft = self.drafter[token[:, :-1].long()]
        target, rows, recorded = self.forward(token, slot, n_record=1 + drafts)   # (from the state before the block on)
        generated = self._generated(token, slot)
        n_accept, path, anchor, n_path = self._verify(target, token, generated, slot, temperature, draft=draft)
        return token, n_accept, anchor, self._keep(rows, recorded, generated, slot, path, n_path)

    def tree_round(self, anchor, slot, branches, temperature=1.0):
        """One round with a tree of the drafter's most likely tokens.  Returns (tokens of the
        accepted path [R, N] (its first n_accept + 1), n_accept, the next anchor, status)."""
        if "g" in self.layers:
            raise ValueError("a Gated DeltaNet state follows one chain")
        parent, place = parents_of(branches)
        likely = self.drafter.topk(max(branches), -1).indices.to(torch.int32)
        token = [anchor]
        for p, j in zip(parent[1:], place[1:]):
            token.append(likely[token[p].long(), j])
        token = torch.stack(token, 1)
        parents = torch.tensor([parent] * len(slot), dtype=torch.int32, device=self.device)
        mask, depth = bd.bdgdn_tree_mask(parents, want_depth=True)
        target, rows, recorded = self.forward(token, slot, mask=mask, depth=depth)
        generated = self._generated(token, slot)
        n_accept, path, anchor, n_path = self._verify(target, token, generated, slot, temperature, mask=mask, parent=parents)
        status = self._keep(rows, recorded, generated, slot, path, n_path)
        return token.gather(1, path.clamp(min=0).long()), n_accept, anchor, status

    def shorten(self, slot, first, last):
        """Keeps the first and the last tokens of each cached sequence."""
        n = self.tables.seq_len[slot.long()]
        count = n.clamp(max=first + last)
        j = torch.arange(first + last, device=self.device, dtype=torch.int32)[None]
        keep = torch.where(j < first, j, j + (n - count)[:, None])
        return bd.bdgdn_cache_compact(self.tables, self.pools, slot, keep.contiguous(), count)

    def finish(self, slot):
        """The sequences end: their slots may be used again."""
        for t in (*self.states, self.taken, self.prompted, self.history):
            if t is not None:
                t[slot.long()] = 0
        bd.bdgdn_cache_truncate(self.tables, slot)


def positive(text):
    n = int(text)
    if n < 1:
        raise argparse.ArgumentTypeError(f"{n} is not above zero")
    return n


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", default="gaga", help='of "g" (Gated DeltaNet) and "a" (attention)')
    ap.add_argument("--prompts", type=positive, default=8)
    ap.add_argument("--ways", type=positive, default=4, help="continuations of each prompt")
    ap.add_argument("--length", type=positive, default=100, help="of a prompt")
    ap.add_argument("--rounds", type=positive, default=64)
    ap.add_argument("--drafts", type=int, default=7)
    ap.add_argument("--tree", help="children of a node at each depth, as 3,2,1: draft trees")
    ap.add_argument("--temperature", type=float, default=1.0)
    ap.add_argument("--window", type=int, default=256, help="cached tokens kept, from twice as many on")
    ap.add_argument("--rotary", type=float, help="base of the attention layers' rotary positions")
    ap.add_argument("--eight-bit", action="store_true", help="projections in 8-bit integers")
    ap.add_argument("--repetition", type=float, default=1.0)
    ap.add_argument("--presence", type=float, default=0.0)
    ap.add_argument("--frequency", type=float, default=0.0)
    args = ap.parse_args()
    penalties = (args.repetition, args.presence, args.frequency)
    torch.manual_seed(0)
    R, ways = args.prompts, args.ways
    branches = [int(x) for x in args.tree.split(",")] if args.tree else []
    grows = 1 + (len(branches) or args.drafts)      # tokens a round at most
    every = max(1, args.window // grows)            # rounds from one shortening to the next
    max_len = max(args.length, args.window) + (every + 1) * grows
    # (twice the pages: a shortened sequence's tokens move before their old pages are free)
    model = Decoder(args.layers, slots=R * ways, max_len=max_len, pages=2 * R * ways * -(-max_len // 16),
                    rotary=args.rotary, eight_bit=args.eight_bit, penalties=penalties if penalties != (1, 0, 0) else None)
    slot = torch.arange(R * ways, dtype=torch.int32, device=model.device)
    prompt = torch.randint(model.vocab, (R, args.length), dtype=torch.int32, device=model.device)
    anchor, status = model.prefill(prompt, slot[:R], whole=True)
    bad = status.max()
    if ways > 1:
        bad = torch.maximum(bad, model.fork(slot[:R].repeat(ways - 1), slot[R:]).max())
    anchor = anchor.repeat(ways)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    emitted = torch.zeros((), dtype=torch.int64, device=model.device)
    start.record()
    for i in range(args.rounds):
        if i == 1:   # (the first of several rounds loads kernels and fills allocators)
            start.record()
        if i and i % every == 0 and model.pools:
            bad = torch.maximum(bad, model.shorten(slot, 4, args.window - 4).max())
        step = model.tree_round(anchor, slot, branches, args.temperature) if branches else model.round(
            anchor, slot, args.drafts, args.temperature)
        _, n_accept, anchor, status = step
        emitted += (n_accept + 1).sum()
        bad = torch.maximum(bad, status.max())
    end.record()
    model.finish(slot)
    if int(bad) != bd.BDGDN_CACHE_DONE or int(model.tables.refcount.max()) != 0:
        raise SystemExit(f"the cache refused a request (status {int(bad)})")
    per_round = start.elapsed_time(end) / max(args.rounds - 1, 1)
    print(f"{R * ways} sequences, {args.rounds} rounds: {int(emitted) / (R * ways * args.rounds):.2f} tokens a "
          f"sequence and round, {per_round * 1e3:.0f} us a round")


if __name__ == "__main__":
    main()
