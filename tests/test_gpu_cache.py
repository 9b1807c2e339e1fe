"""The pages of a cache against lists of tokens: append (copy on write), fork, compact and
truncate in long random rounds, with every refusal, at page sizes of one token and more."""
import random

import pytest
import torch

import paper_2606_01774_amd as bd

pytestmark = pytest.mark.gpu


class Model:
    """What the entry points do, on lists: a sequence is a list of pages and a length."""

    def __init__(self, n_slots, max_pages, n_pages, page):
        self.page, self.max_pages, self.n_pages = page, max_pages, n_pages
        self.cols = [[] for _ in range(n_slots)]
        self.len = [0] * n_slots
        self.refs = [0] * n_pages
        self.data = {}                       # (page, place) -> row id

    def pages(self, n):
        return -(-n // self.page)

    def tokens(self, s):
        return [self.data[self.cols[s][t // self.page], t % self.page] for t in range(self.len[s])]

    def release(self, p):
        self.refs[p] -= 1

    def _grant(self, needs):
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        out = []
        for n in needs:
            if n is None or n > len(free):
                out.append(None)
            else:
                out.append([free.pop(0) for _ in range(n)])
        return out

    def append(self, slots, counts, rows):
        refs, status, needs = list(self.refs), [], []
        for s, n in zip(slots, counts):
            if not 0 <= s < len(self.cols):
                st, need = bd.BDGDN_CACHE_BAD_SLOT, None
            elif self.len[s] + n > self.max_pages * self.page:
                st, need = bd.BDGDN_CACHE_NO_ROOM, None
            else:
                own = self.len[s] % self.page and n and refs[self.cols[s][-1]] > 1
                st, need = bd.BDGDN_CACHE_DONE, self.pages(self.len[s] + n) - self.pages(self.len[s]) + bool(own)
            status.append(st)
            needs.append(need)
        snap = dict(self.data)
        for i, (s, n, got) in enumerate(zip(slots, counts, self._grant(needs))):
            if got is None:
                if status[i] == bd.BDGDN_CACHE_DONE:
                    status[i] = bd.BDGDN_CACHE_NO_PAGES
                continue
            start = self.len[s]
            ids = list(rows[i][:n])
            if start % self.page and n and refs[self.cols[s][-1]] > 1:
                old = self.cols[s].pop()
                ids = [snap[old, t] for t in range(start % self.page)] + ids
                start -= start % self.page
                self.release(old)
            self.cols[s] += got
            for p in got:
                self.refs[p] = 1
            for j, x in enumerate(ids):
                self.data[self.cols[s][(start + j) // self.page], (start + j) % self.page] = x
            self.len[s] += n
        return status

    def fork(self, src, dst):
        status = []
        for a, b in zip(src, dst):
            if not (0 <= a < len(self.cols) and 0 <= b < len(self.cols)) or self.len[b]:
                status.append(bd.BDGDN_CACHE_BAD_SLOT)
                continue
            self.cols[b], self.len[b] = list(self.cols[a]), self.len[a]
            for p in self.cols[b]:
                self.refs[p] += 1
            status.append(bd.BDGDN_CACHE_DONE)
        return status

    def compact(self, slots, keeps):
        status, needs, plans = [], [], []
        for s, keep in zip(slots, keeps):
            plan = None
            if not 0 <= s < len(self.cols):
                st, need = bd.BDGDN_CACHE_BAD_SLOT, None
            elif any(not 0 <= t < self.len[s] for t in keep) or any(a >= b for a, b in zip(keep, keep[1:])):
                st, need = bd.BDGDN_CACHE_BAD_KEEP, None
            else:
                stay = sum(t == j for j, t in enumerate(keep))
                whole = self.pages(stay) if stay == len(keep) else stay // self.page
                st, need, plan = bd.BDGDN_CACHE_DONE, self.pages(len(keep)) - whole, whole
            status.append(st)
            needs.append(need)
            plans.append(plan)
        snap = dict(self.data)
        for i, (s, keep, got) in enumerate(zip(slots, keeps, self._grant(needs))):
            if got is None:
                if status[i] == bd.BDGDN_CACHE_DONE:
                    status[i] = bd.BDGDN_CACHE_NO_PAGES
                continue
            ids = [snap[self.cols[s][t // self.page], t % self.page] for t in keep]
            whole = plans[i]
            for p in self.cols[s][whole:]:
                self.release(p)
            self.cols[s] = self.cols[s][:whole] + got
            for p in got:
                self.refs[p] = 1
            for j in range(whole * self.page, len(keep)):
                self.data[self.cols[s][j // self.page], j % self.page] = ids[j]
            self.len[s] = len(keep)
        return status

    def truncate(self, slots, lengths):
        for s, n in zip(slots, lengths):
            if 0 <= s < len(self.cols):
                n = min(self.len[s], max(n, 0))
                for p in self.cols[s][self.pages(n):]:
                    self.release(p)
                self.cols[s], self.len[s] = self.cols[s][:self.pages(n)], n


class Cache:
    def __init__(self, n_slots, max_pages, n_pages, page, h_kv, d, dtype, pools, htd):
        self.model = Model(n_slots, max_pages, n_pages, page)
        self.tables = bd.make_cache_tables(n_slots, max_pages, n_pages)
        self.page, self.next = page, 1
        self.shape, self.dtype = (h_kv, d), dtype
        shape = (n_pages, h_kv, page, d) if htd else (n_pages, page, h_kv, d)
        self.pools = [torch.full(shape, float("nan"), dtype=dtype, device="cuda") for _ in range(pools)]
        self.pools = [p.transpose(1, 2) if htd else p for p in self.pools]

    def rows(self, R, N):
        """Rows whose elements tell the row, the pool and the head."""
        ids = torch.arange(self.next, self.next + R * N).view(R, N)
        self.next += R * N
        out = []
        for i in range(len(self.pools)):
            x = torch.zeros(R, N, *self.shape)
            x[..., 0] = (ids % 251)[..., None].float()
            x[..., 1] = (ids // 251)[..., None].float()
            x[..., 2] = i
            x[..., -1] = torch.arange(self.shape[0]).float()
            out.append(x.to(self.dtype).cuda())
        return ids.tolist(), out

    def check(self):
        m, (table, seq, refs, bits) = self.model, [t.cpu() for t in self.tables]
        for s, cols in enumerate(m.cols):
            assert table[s].tolist() == cols + [-1] * (m.max_pages - len(cols)), s
        assert seq.tolist() == m.len and refs.tolist() == m.refs
        free = [bool(int(bits[p // 32]) >> p % 32 & 1) for p in range(len(bits) * 32)]
        assert free == [p < m.n_pages and m.refs[p] == 0 for p in range(len(free))]
        for i, pool in enumerate(self.pools):
            host = pool.cpu().float()
            for s in range(len(m.cols)):
                n = m.len[s]
                if not n:
                    continue
                t = torch.arange(n)
                got = host[torch.tensor(m.cols[s])[t // self.page], t % self.page]
                ids = torch.tensor(m.tokens(s))
                assert torch.equal(got[:, 0, 0], (ids % 251).float()) and torch.equal(got[:, -1, 1], (ids // 251).float())
                assert (got[:, :, 2] == i).all() and not got[:, :, 3:-1].any()
                assert torch.equal(got[0, :, -1], torch.arange(self.shape[0]).float())


def _ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("page,h_kv,d,dtype,pools,htd,n_pages", [
    (1, 1, 64, torch.float32, 1, False, 90),
    (7, 3, 64, torch.bfloat16, 2, True, 40),
    (16, 2, 128, torch.bfloat16, 3, False, 33),
    (64, 8, 128, torch.bfloat16, 2, False, 1100),
    (24, 1, 256, torch.float32, 2, True, 64),
])
def test_random_rounds(page, h_kv, d, dtype, pools, htd, n_pages):
    rng = random.Random(page)
    n_slots, max_pages = 12, max(4, 60 // page)
    c = Cache(n_slots, max_pages, n_pages, page, h_kv, d, dtype, pools, htd)
    seen = set()
    for step in range(60):
        what = rng.choice(["append", "append", "append", "fork", "compact", "truncate"])
        k = rng.randint(1, n_slots)
        slots = rng.sample(range(n_slots), k)
        if rng.random() < 0.1:
            slots[0] = rng.choice([-1, n_slots, 2 ** 31 - 1])
        if what == "append":
            N = rng.choice([1, 5, page, 3 * page + 1])
            ids, rows = c.rows(k, N)
            counts = [rng.choice([0, 1, N, rng.randint(0, N)]) for _ in slots]
            path = None
            picked = ids
            if rng.random() < 0.6:
                path = [sorted(rng.sample(range(N), n)) + [-1] * (N - n) for n in counts]
                picked = [[ids[i][j] for j in path[i][:n]] for i, n in enumerate(counts)]
            want = c.model.append(slots, counts, picked)
            got = bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints(slots), _ints(counts),
                                        path=None if path is None else _ints(path))
        elif what == "fork":
            src = [s for s in range(n_slots) if c.model.len[s]] or [0]
            dst = [s for s in slots if s not in src][:4] or [src[0]]
            src = [rng.choice([s for s in src if s not in dst] or [0]) for _ in dst]
            if set(src) & set(dst):
                continue
            want = c.model.fork(src, dst)
            got = bd.bdgdn_cache_fork(c.tables, _ints(src), _ints(dst), page=page)
        elif what == "compact":
            keeps = []
            for s in slots:
                n = c.model.len[s] if 0 <= s < n_slots else 3
                lead = rng.choice([0, n // 2, n])
                keep = list(range(lead)) + sorted(rng.sample(range(lead, n), rng.randint(0, n - lead)))
                if rng.random() < 0.1:
                    keep = keep + [n]
                if rng.random() < 0.1 and len(keep) > 1:
                    keep[-1] = keep[-2]
                keeps.append(keep)
            M = max(max(len(x) for x in keeps), 1) + rng.randint(0, 3)
            want = c.model.compact(slots, keeps)
            got = bd.bdgdn_cache_compact(c.tables, c.pools, _ints(slots), _ints([x + [-9] * (M - len(x)) for x in keeps]),
                                         _ints([len(x) for x in keeps]))
        else:
            lengths = [rng.choice([-2, 0, 1, page, 10 ** 6, rng.randint(0, page * max_pages)]) for _ in slots]
            c.model.truncate(slots, lengths)
            bd.bdgdn_cache_truncate(c.tables, _ints(slots), _ints(lengths), page=page)
            want = got = None
        if want is not None:
            assert got.tolist() == want, (step, what)
            seen |= set(want)
        c.check()
    assert {bd.BDGDN_CACHE_DONE, bd.BDGDN_CACHE_BAD_SLOT} <= seen
    bd.bdgdn_cache_truncate(c.tables, _ints(list(range(n_slots))), page=page)
    c.model.truncate(range(n_slots), [0] * n_slots)
    c.check()
    assert not any(c.model.refs)


def test_too_few_pages_go_to_whom_they_suffice():
    c = Cache(6, 8, 9, 4, 1, 64, torch.float32, 1, False)
    ids, rows = c.rows(6, 20)
    counts = [16, 20, 8, 9, 4, 1]      # 4, 5, 2, 3, 1, 1 pages of 9
    want = c.model.append(range(6), counts, ids)
    got = bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints(range(6)), _ints(counts))
    assert got.tolist() == want == [0, 0, 1, 1, 1, 1]
    c.check()
    ids, rows = c.rows(2, 20)
    bd.bdgdn_cache_truncate(c.tables, _ints([0]), _ints([7]), page=4)
    c.model.truncate([0], [7])
    want = c.model.append([2, 3], [12, 8], ids)
    got = bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints([2, 3]), _ints([12, 8]))
    assert got.tolist() == want == [1, 0]
    c.check()
    want = c.model.append([1], [20], ids)
    got = bd.bdgdn_cache_append(c.tables, c.pools, [rows[0][:1]], _ints([1]), _ints([20]))
    assert got.tolist() == want == [2]
    c.check()


def test_many_requests_and_many_pages():
    """More requests and more words of free bits than a workgroup has threads."""
    n = 1500
    c = Cache(n, 4, 70000, 2, 1, 64, torch.bfloat16, 1, False)
    c.model.refs[:66000] = [1] * 66000             # low pages that somebody else holds
    c.tables.refcount[:66000] = 1
    c.tables.free_bits[:66000 // 32] = 0
    c.tables.free_bits[66000 // 32] &= ~((1 << 66000 % 32) - 1)
    ids, rows = c.rows(n, 3)
    counts = [(i * 7) % 4 for i in range(n)]
    slots = list(range(n))[::-1]
    want = c.model.append(slots, counts, ids)
    got = bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints(slots), _ints(counts))
    assert got.tolist() == want
    c.check()


@pytest.mark.parametrize("R,tokens,page,max_pages,n_pages,pools", [
    (3, 700, 16, 50, 200, 1),        # planned by one workgroup
    (300, 11, 2, 8, 3000, 1),        # by many: requests,
    (2, 17000, 64, 300, 900, 1),     # positions,
    (4, 300, 16, 5000, 160, 2),      # columns of the table
    (2, 100, 8, 20, 60, 17),         # more pools than a small launch takes
    (2, 40, 8, 20, 40, 100),         # more than any launch takes
])
def test_compactions_of_few_and_of_many(R, tokens, page, max_pages, n_pages, pools):
    rng = random.Random(R * tokens)
    c = Cache(R + 1, max_pages, n_pages, page, 1, 64, torch.bfloat16, pools, False)
    slots, counts = list(range(R)), [tokens - i % 3 for i in range(R)]
    ids, rows = c.rows(R, tokens)
    want = c.model.append(slots, counts, ids)
    assert bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints(slots), _ints(counts)).tolist() == want
    c.model.fork([0], [R])
    bd.bdgdn_cache_fork(c.tables, _ints([0]), _ints([R]), page=page)
    for turn in range(3):
        keeps = []
        for i in range(R):
            n = c.model.len[i]
            first = rng.randrange(n + 1) if i % 2 else 0     # some keep their beginnings
            keeps.append([t for t in range(n) if t < first or rng.random() < 0.6])
        asked = list(slots)
        if turn == 1:
            keeps[-1] = []
            asked[0] = R + 7
        if turn == 2 and len(keeps[0]) > 1:
            keeps[0][1] = keeps[0][0]                        # does not rise
        keep = torch.zeros(R, max(map(len, keeps)), dtype=torch.int32)
        for i, k in enumerate(keeps):
            keep[i, :len(k)] = torch.tensor(k, dtype=torch.int32)
        want = c.model.compact(asked, keeps)
        got = bd.bdgdn_cache_compact(c.tables, c.pools, _ints(asked), keep.cuda(), _ints([len(k) for k in keeps]))
        assert got.tolist() == want
        c.check()


def test_nodes_that_are_none_and_rows_of_a_projection():
    c = Cache(2, 4, 8, 4, 2, 64, torch.bfloat16, 2, False)
    whole = torch.randn(2, 3, 6, 64, device="cuda").to(torch.bfloat16)
    rows = [whole[:, :, 2:4], whole[:, :, 4:]]
    bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints([1, 0]), _ints([3, 2]), path=_ints([[2, -1, 0], [3, 1, 9]]))
    table = c.tables.page_table.cpu()
    for i, rows_i in enumerate(rows):
        got = c.pools[i][int(table[1, 0])]
        assert torch.equal(got[0], rows_i[0, 2]) and not got[1].any() and torch.equal(got[2], rows_i[0, 0])
        got = c.pools[i][int(table[0, 0])]
        assert not got[0].any() and torch.equal(got[1], rows_i[1, 1])
    assert c.tables.seq_len.tolist() == [2, 3]


def test_a_missing_last_page_is_replaced():
    """A table entry that holds no page (its tokens were dropped by the caller) takes a new one."""
    c = Cache(1, 4, 8, 4, 1, 64, torch.float32, 1, False)
    ids, rows = c.rows(1, 6)
    bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints([0]), _ints([6]))
    c.tables.page_table[0, 1] = -1
    ids, rows = c.rows(1, 6)
    assert bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints([0]), _ints([3])).tolist() == [0]
    assert c.tables.page_table[0].tolist() == [0, 2, 3, -1] and c.tables.seq_len.tolist() == [9]
    assert torch.equal(c.pools[0][2, 2:], rows[0][0, :2]) and torch.equal(c.pools[0][3, 0], rows[0][0, 2])


def test_a_replayed_graph_of_a_round():
    """append, fork, append to both, compact, truncate: captured once, replayed three times."""
    def round_(c, rows, one):
        bd.bdgdn_cache_append(c.tables, c.pools, rows, s0, n5)
        bd.bdgdn_cache_fork(c.tables, s0, s1, page=4)
        bd.bdgdn_cache_append(c.tables, c.pools, one, both, ones)
        bd.bdgdn_cache_compact(c.tables, c.pools, s1, keep, three)
        bd.bdgdn_cache_truncate(c.tables, s0, two, page=4)

    s0, s1, both, n5 = _ints([0]), _ints([1]), _ints([1, 0]), _ints([5])
    ones, keep, three, two = _ints([1, 1]), _ints([[0, 2, 5]]), _ints([3]), _ints([2])
    made = [Cache(2, 6, 20, 4, 1, 64, torch.float32, 2, False) for _ in range(2)]
    rows, one = [torch.randn(1, 5, 1, 64, device="cuda") for _ in range(2)], [torch.randn(2, 1, 1, 64, device="cuda")] * 2
    for c in made:
        for p in c.pools:
            p.zero_()
        round_(c, rows, one)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_(made[1], rows, one)
    for _ in range(3):
        for c in made:
            bd.bdgdn_cache_truncate(c.tables, _ints([0, 1]), page=4)
        for t in rows:
            t.mul_(1.5)
        round_(made[0], rows, one)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*made[0].tables, *made[0].pools), (*made[1].tables, *made[1].pools)):
            assert torch.equal(a, b)


def test_expanded_rows_are_refused():
    """One first row for all ways of a fork: refused, and taken as a copy."""
    c = Cache(3, 4, 8, 4, 1, 64, torch.float32, 1, False)
    row = torch.randn(1, 1, 1, 64, device="cuda")
    with pytest.raises(ValueError, match="must have"):
        bd.bdgdn_cache_append(c.tables, c.pools, [row.expand(3, 1, 1, 64)], _ints([0, 1, 2]), _ints([1, 1, 1]))
    c.check()
    bd.bdgdn_cache_append(c.tables, c.pools, [row.expand(3, 1, 1, 64).contiguous()], _ints([0, 1, 2]), _ints([1, 1, 1]))
    for page in c.tables.page_table[:, 0].tolist():
        assert torch.equal(c.pools[0][page, 0], row[0, 0])


@pytest.mark.parametrize("page,old,htd,pools", [(4, 6, False, 1), (16, 47, True, 2), (64, 1, False, 17)])
def test_a_replaced_page_holds_nothing_of_its_last_owner(page, old, htd, pools):
    """The new page in place of a missing one: the tokens before the appended ones, which now have a page
    again, are rows of zeros, not what the page held before."""
    c = Cache(2, 8, 12, page, 2, 64, torch.bfloat16, pools, htd)
    ids, rows = c.rows(1, old)
    assert bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints([0]), _ints([old])).tolist() == [0]
    last = (old - 1) // page
    c.tables.page_table[0, last] = 12 if pools == 2 else -1
    ids, rows = c.rows(1, page + 1)
    path = None if pools == 1 else _ints([list(range(page + 1))])
    assert bd.bdgdn_cache_append(c.tables, c.pools, rows, _ints([0]), _ints([page + 1]), path=path).tolist() == [0]
    cols, n = c.tables.page_table[0].tolist(), old + page + 1
    assert 0 <= cols[last] < 12 and c.tables.seq_len.tolist() == [n, 0]
    for pool, new in zip(c.pools, rows):
        got = torch.stack([pool[cols[t // page], t % page] for t in range(last * page, n)])
        assert not got[:old - last * page].any() and torch.equal(got[old - last * page:], new[0])


def test_pools_of_another_page_are_refused():
    t = bd.make_cache_tables(2, 4, 8, page=16)
    rows, one = [torch.zeros(1, 2, 1, 64, device="cuda")], _ints([0])
    other = [torch.zeros(8, 8, 1, 64, device="cuda")]
    with pytest.raises(ValueError, match="pages of 16"):
        bd.bdgdn_cache_append(t, other, rows, one, _ints([2]))
    with pytest.raises(ValueError, match="pages of 16"):
        bd.bdgdn_cache_compact(t, other, one, _ints([[0]]), _ints([1]))
    pools = [torch.zeros(8, 16, 1, 64, device="cuda")]
    assert bd.bdgdn_cache_append(t, pools, rows, one, _ints([2])).tolist() == [0]
    assert bd.bdgdn_cache_fork(t, one, _ints([1])).tolist() == [0] and t.refcount.tolist()[:2] == [2, 0]
    bd.bdgdn_cache_truncate(t, _ints([0, 1]))
    assert not t.refcount.any() and not t.seq_len.any()
