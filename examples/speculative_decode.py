"""Speculative decoding of a small hybrid model: AR-Trust serving rounds with every call on the
device.

The model has random weights: an embedding, layers "g" (Gated DeltaNet) and "a" (softmax attention over
a paged cache), an output projection.  Its drafter is the model without its layers.  A round
drafts a chain behind each request's last token, runs the block through the layers
(bdgdn_commit_record, bdgdn_tree_attn), decides (bdgdn_verify) and keeps what was accepted
(bdgdn_accept_states, bdgdn_cache_append); nothing of it waits for the host.  Prompts are forked
several ways (bdgdn_cache_fork), a window keeps the caches short (bdgdn_cache_compact), and
finished sequences give their pages back (bdgdn_cache_truncate).  A model without "g" layers
can also draft trees (bdgdn_tree_mask).

    python examples/speculative_decode.py --prompts 8 --ways 4 --rounds 64
    python examples/speculative_decode.py --layers aa --tree 3,2,1 --temperature 0
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
    """The model with the states and caches of `slots` sequences of up to max_len tokens."""

    def __init__(self, layers="gaga", vocab=512, width=256, slots=32, page=16, max_len=1024, pages=None, seed=0,
                 device="cuda"):
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

    def forward(self, token, slot, mask="causal", n_record=0):
        """Logits [R, N, V] of a block of tokens behind the sequences in `slot`, the attention
        layers' new rows, and with n_record the recorded states of the "g" layers.  The "g"
        layers' states go forward by the whole block, the caches stay as they are."""
        R, N = token.shape
        x = self.embed[token.long()].float()
        rows, recorded, a = [], [], 0
        for i, kind in enumerate(self.layers):
            y = norm(x).to(torch.bfloat16) @ self.w_in[i]
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
                o, _ = bd.bdgdn_tree_attn(q, k, v, self.pools[a], self.pools[a + 1], self.tables.page_table,
                                          self.tables.seq_len, mask=mask, slot=slot)
                rows += [k, v]
                recorded.append(None)
                a += 2
            x = x + (o.reshape(R, N, -1) @ self.w_out[i]).float()
        return self.logits(x), rows, recorded

    def append(self, rows, slot, count, path=None):
        if rows:
            return bd.bdgdn_cache_append(self.tables, self.pools, rows, slot, count, path=path)
        return torch.zeros_like(count)

    def prefill(self, prompt, slot, block=32):
        """Takes in prompt [R, T] but its last token, which is the first round's anchor."""
        status = torch.zeros_like(slot)
        for t in range(0, prompt.shape[1] - 1, block):
            part = prompt[:, t:min(t + block, prompt.shape[1] - 1)]
            _, rows, _ = self.forward(part, slot)
            status |= self.append(rows, slot, torch.full_like(slot, part.shape[1]))
        return prompt[:, -1], status

    def fork(self, src, dst):
        for s in self.states:
            if s is not None:
                s[dst.long()] = s[src.long()]
        return bd.bdgdn_cache_fork(self.tables, src, dst)

    def _draft(self, logits, temperature):
        if temperature <= 0:
            return logits.argmax(-1)
        p = torch.softmax(logits / temperature, -1)
        return (p / torch.empty_like(p).exponential_()).argmax(-1)

    def _verify(self, target, token, temperature, **kw):
        R, N, V = target.shape
        u = torch.rand(R, N, device=self.device)
        noise = torch.empty(R, V, device=self.device).exponential_()
        T = torch.full((R,), float(temperature), device=self.device)
        return bd.bdgdn_verify(target, token, u, noise, temperature=T, want_n_path=True, **kw)

    def round(self, anchor, slot, drafts=7, temperature=1.0):
        """One round with a drafted chain.  Returns (tokens [R, 1 + drafts] of the block,
        n_accept, the next anchor, status)."""
        token = [anchor]
        for _ in range(drafts):
            token.append(self._draft(self.drafter[token[-1].long()], temperature).to(torch.int32))
        token = torch.stack(token, 1)
        draft = self.drafter[token[:, :-1].long()]
        target, rows, recorded = self.forward(token, slot, n_record=drafts)
        n_accept, path, anchor, n_path = self._verify(target, token, temperature, draft=draft)
        for state, kept in zip(self.states, recorded):
            if kept is not None:
                bd.bdgdn_accept_states(state, kept, n_accept, block=token.shape[1], slot=slot)
        return token, n_accept, anchor, self.append(rows, slot, n_path, path)

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
        target, rows, _ = self.forward(token, slot, mask=bd.bdgdn_tree_mask(parents))
        n_accept, path, anchor, n_path = self._verify(target, token, temperature, parent=parents)
        status = self.append(rows, slot, n_path, path)
        return token.gather(1, path.clamp(min=0).long()), n_accept, anchor, status

    def shorten(self, slot, first, last):
        """Keeps the first and the last tokens of each cached sequence."""
        n = self.tables.seq_len[slot.long()]
        count = n.clamp(max=first + last)
        j = torch.arange(first + last, device=self.device, dtype=torch.int32)[None]
        keep = torch.where(j < first, j, j + (n - count)[:, None])
        return bd.bdgdn_cache_compact(self.tables, self.pools, slot, keep.contiguous(), count)

    def finish(self, slot):
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
    args = ap.parse_args()
    torch.manual_seed(0)
    R, ways = args.prompts, args.ways
    branches = [int(x) for x in args.tree.split(",")] if args.tree else []
    grows = 1 + (len(branches) or args.drafts)      # tokens a round at most
    every = max(1, args.window // grows)            # rounds from one shortening to the next
    max_len = max(args.length, args.window) + (every + 1) * grows
    # (twice the pages: a shortened sequence's tokens move before their old pages are free)
    model = Decoder(args.layers, slots=R * ways, max_len=max_len, pages=2 * R * ways * -(-max_len // 16))
    slot = torch.arange(R * ways, dtype=torch.int32, device=model.device)
    prompt = torch.randint(model.vocab, (R, args.length), dtype=torch.int32, device=model.device)
    anchor, status = model.prefill(prompt, slot[:R])
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
