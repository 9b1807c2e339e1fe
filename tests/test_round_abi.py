"""Host-side validation of the entry points that serve the softmax half of a round (no GPU is
touched: every call here fails validation, or has no requests)."""
import copy
import ctypes

import pytest
import torch

import paper_2606_01774_amd as bd
from paper_2606_01774_amd import rounds

FAKE = 0x1000   # never dereferenced: validation fails first


def _cache(**kw):
    d = dict(n_pages=10, page=16, n_slots=4, max_pages=5, h_kv=2, d=128, dtype=bd.BDGDN_BF16, page_stride=16 * 256,
             token_stride=256, head_stride=128)
    d.update(kw)
    return rounds.CacheDesc(**d)


def _attn(**kw):
    d = dict(num_req=2, nodes=8, h_q=8, h_kv=2, d=128, scale=0.1, dtype=bd.BDGDN_BF16, out_dtype=bd.BDGDN_BF16,
             mask=bd.BDGDN_MASK_CAUSAL)
    d.update(kw)
    return rounds.AttnDesc(**d)


def _call_attn(desc, cache, bytes_=1 << 40, ptr=None, mask=None, slot=None):
    p = dict(q=FAKE, k=FAKE, v=FAKE, kp=FAKE, vp=FAKE, table=FAKE, len=FAKE, o=FAKE, ws=FAKE)
    p.update(ptr or {})
    return bd.load_library().bdgdn_tree_attn(desc, cache, p["q"], p["k"], p["v"], p["kp"], p["vp"], p["table"], p["len"],
                                             slot, None, mask, p["o"], None, p["ws"], bytes_, None)


INV, UNS, WS = bd.BDGDN_ERR_INVALID_ARG, bd.BDGDN_ERR_UNSUPPORTED, bd.BDGDN_ERR_WORKSPACE


@pytest.mark.parametrize("attn,cache,status", [
    (dict(num_req=-1), {}, INV), (dict(nodes=0), {}, INV), (dict(nodes=65), {}, UNS), (dict(h_q=7), {}, INV),
    (dict(h_kv=4), {}, INV), (dict(d=64), {}, INV), (dict(d=96), dict(d=96, head_stride=96), UNS),
    (dict(scale=float("inf")), {}, INV), (dict(mask=3), {}, INV), (dict(dtype=5), dict(dtype=5), UNS),
    (dict(dtype=bd.BDGDN_F32, out_dtype=bd.BDGDN_BF16), dict(dtype=bd.BDGDN_F32), UNS),
    (dict(q_stride=8), {}, INV), (dict(k_stride=260), {}, INV), (dict(v_stride=-256), {}, INV),
    ({}, dict(n_pages=0), INV), ({}, dict(page=0), INV), ({}, dict(page=65537), UNS), ({}, dict(max_pages=1 << 30), UNS),
    ({}, dict(token_stride=100), INV), ({}, dict(head_stride=130), INV), ({}, dict(page_stride=0), INV),
    ({}, dict(page_stride=1 << 40), UNS), ({}, dict(n_slots=1), INV), ({}, dict(dtype=bd.BDGDN_F32), INV),
])
def test_attention_rejects_bad_descriptors(attn, cache, status):
    a, c = _attn(**attn), _cache(**cache)
    assert _call_attn(a, c) == status
    if cache != dict(n_slots=1):
        assert bd.bdgdn_tree_attn_workspace(a, c) == 0


@pytest.mark.parametrize("ptr,status", [
    (dict(q=None), INV), (dict(kp=None), INV), (dict(table=None), INV), (dict(o=None), INV), (dict(q=0x1008), INV),
    (dict(vp=0x1004), INV), (dict(o=0x1008), INV), (dict(ws=0x1010), INV), (dict(ws=None), WS),
])
def test_attention_rejects_bad_pointers(ptr, status):
    assert _call_attn(_attn(), _cache(), ptr=ptr) == status


def test_attention_limits():
    """Rows of tokens further apart than 32-bit offsets within a page allow, more tiles of keys
    or more workgroups than 31 bits count."""
    token = 1 << 25                                 # bf16 elements: 2^26 bytes
    far = dict(n_pages=1, page=1, page_stride=token, max_pages=5)
    assert bd.bdgdn_tree_attn_workspace(_attn(), _cache(token_stride=token, **far)) > 0
    assert _call_attn(_attn(), _cache(token_stride=token + 8, **far)) == UNS
    for page, columns, want in ((65536, 32767, bd.BDGDN_OK), (1, 0x7fff0001, UNS), (1, 0x7fffffff, UNS)):
        cache = _cache(page=page, max_pages=columns)
        got = bd.bdgdn_tree_attn_workspace(_attn(num_req=1), cache) > 0
        assert got == (want == bd.BDGDN_OK) and (got or _call_attn(_attn(num_req=1), cache) == want)
    # 65535 requests of 32764 tiles: 2^31 is passed by what their nodes count for
    many = dict(num_req=65535, nodes=64, h_q=2)
    assert bd.bdgdn_tree_attn_workspace(_attn(**many), _cache(n_slots=65535, max_pages=2 * 32700)) > 0
    assert _call_attn(_attn(**many), _cache(n_slots=65535, max_pages=2 * 32764)) == UNS
    assert _call_attn(_attn(num_req=65535, nodes=64, h_q=512), _cache(n_slots=65535)) == UNS
    for h_kv, want in ((256, bd.BDGDN_OK), (257, UNS)):
        cache = _cache(n_slots=65535, h_kv=h_kv, token_stride=128 * h_kv, page_stride=128 * h_kv * 16)
        attn = _attn(num_req=65535, nodes=1, h_q=h_kv, h_kv=h_kv)
        assert (bd.bdgdn_tree_attn_workspace(attn, cache) > 0) == (want == bd.BDGDN_OK)
        assert want == bd.BDGDN_OK or _call_attn(attn, cache) == want


def test_attention_checks_mask_and_workspace():
    assert _call_attn(_attn(), _cache(), mask=FAKE) == INV
    assert _call_attn(_attn(mask=bd.BDGDN_MASK_BITS), _cache()) == INV
    assert _call_attn(_attn(mask=bd.BDGDN_MASK_BITS), _cache(), mask=0x1004) == INV
    need = bd.bdgdn_tree_attn_workspace(_attn(), _cache())
    assert need > 0 and _call_attn(_attn(), _cache(), bytes_=need - 1) == WS
    assert _call_attn(_attn(num_req=0), _cache()) == bd.BDGDN_OK and bd.bdgdn_tree_attn_workspace(_attn(num_req=0), _cache()) == 0


def test_tree_mask_rejects():
    f = bd.load_library().bdgdn_tree_mask
    assert f(1, 0, FAKE, FAKE, None, None) == INV and f(-1, 4, FAKE, FAKE, None, None) == INV
    assert f(1, 65, FAKE, FAKE, None, None) == UNS and f(1, 4, None, FAKE, None, None) == INV
    assert f(1, 4, FAKE, 0x1004, None, None) == INV and f(0, 4, None, None, None, None) == bd.BDGDN_OK


def _verify(**kw):
    d = dict(num_req=2, nodes=4, vocab=100, dtype=bd.BDGDN_F32, target_req_stride=400, target_row_stride=100,
             draft_req_stride=400, draft_row_stride=100, noise_stride=100)
    d.update(kw)
    return rounds.VerifyDesc(**d)


def _call_verify(desc, bytes_=1 << 40, **ptr):
    p = dict(target=FAKE, draft=FAKE, token=FAKE, u=FAKE, noise=FAKE, acc=FAKE, path=FAKE, nxt=FAKE, ws=FAKE)
    p.update(ptr)
    return bd.load_library().bdgdn_verify(desc, p["target"], p["draft"], p["token"], None, None, None, p["u"], p["noise"],
                                          p["acc"], None, p["path"], p["nxt"], p["ws"], bytes_, None)


@pytest.mark.parametrize("kw,status", [
    (dict(num_req=-1), INV), (dict(nodes=0), INV), (dict(nodes=65), UNS), (dict(vocab=0), INV), (dict(dtype=2), UNS),
    (dict(target_row_stride=-1), INV), (dict(noise_stride=-4), INV), (dict(num_req=70000), UNS),
])
def test_verify_rejects_bad_descriptors(kw, status):
    assert _call_verify(_verify(**kw)) == status and bd.bdgdn_verify_workspace(_verify(**kw)) == 0


def test_verify_rejects_bad_pointers():
    for name in ("target", "token", "u", "noise", "acc", "path", "nxt"):
        assert _call_verify(_verify(), **{name: None}) == INV, name
    assert _call_verify(_verify(), target=0x1002) == INV and _call_verify(_verify(), draft=0x1001) == INV
    assert _call_verify(_verify(dtype=bd.BDGDN_BF16), draft=0x1001) == INV
    need = bd.bdgdn_verify_workspace(_verify())
    assert _call_verify(_verify(), bytes_=need - 1) == WS and _call_verify(_verify(), ws=None) == WS
    assert _call_verify(_verify(), ws=0x1040) == INV
    assert _call_verify(_verify(num_req=0)) == bd.BDGDN_OK


def test_cache_calls_reject():
    lib = bd.load_library()
    t = rounds._Tables(FAKE, FAKE, FAKE, FAKE)
    hole = rounds._Tables(FAKE, FAKE, None, FAKE)
    ptrs, none = (ctypes.c_void_p * 2)(FAKE, FAKE), (ctypes.c_void_p * 2)(FAKE, None)
    odd = (ctypes.c_void_p * 2)(FAKE, 0x1008)

    def append(c=None, tables=t, pools=ptrs, rows=ptrs, R=2, N=4, stride=0, slot=FAKE, count=FAKE, ws=FAKE, size=1 << 30):
        return lib.bdgdn_cache_append(c or _cache(), tables, pools, rows, 2, R, N, stride, slot, None, count, None, ws,
                                      size, None)

    def compact(c=None, tables=t, pools=ptrs, R=2, M=4, slot=FAKE, keep=FAKE, count=FAKE, ws=FAKE, size=1 << 30):
        return lib.bdgdn_cache_compact(c or _cache(), tables, pools, 2, R, M, slot, keep, count, None, ws, size, None)

    for call in (append, compact):
        assert call(_cache(page=0)) == INV and call(_cache(d=80, head_stride=80)) == UNS
        assert call(tables=hole) == INV and call(pools=none) == INV and call(pools=odd) == INV and call(pools=None) == INV
        assert call(slot=None) == INV and call(count=None) == INV and call(R=-1) == INV and call(R=70000) == UNS
        assert call(ws=None) == WS and call(ws=0x1010) == INV
        assert call(size=bd.bdgdn_cache_workspace(_cache(), 2, 4) - 1) == WS and call(R=0) == bd.BDGDN_OK
    assert append(rows=none) == INV and append(rows=odd) == INV and append(stride=100) == INV and append(N=-1) == INV
    assert append(stride=257) == INV and compact(keep=None) == INV and compact(M=-1) == INV
    assert lib.bdgdn_cache_fork(_cache(), t, 1, None, FAKE, None, None) == INV
    assert lib.bdgdn_cache_fork(_cache(), hole, 1, FAKE, FAKE, None, None) == INV
    assert lib.bdgdn_cache_fork(_cache(), t, -1, FAKE, FAKE, None, None) == INV
    assert lib.bdgdn_cache_truncate(_cache(), t, 1, None, None, None) == INV
    assert lib.bdgdn_cache_truncate(_cache(max_pages=0), t, 1, FAKE, None, None) == INV
    assert bd.bdgdn_cache_workspace(_cache(), 0, 4) == 0 and bd.bdgdn_cache_workspace(_cache(), 2, -1) == 0


def test_cache_limits():
    """More pages in one call than 32 bits count, more requests than a grid has room for."""
    lib, one = bd.load_library(), _cache(page=1, max_pages=1 << 20, page_stride=256)
    tables = rounds._Tables(FAKE, FAKE, FAKE, FAKE)
    pools = (ctypes.c_void_p * 1)(FAKE)
    for R, rows, want in ((65535, 16382, WS), (65535, 16384, UNS), (65536, 1, UNS), (1024, 0x7fffffff, UNS)):
        assert (bd.bdgdn_cache_workspace(one, R, rows) > 0) == (want == WS)
        assert lib.bdgdn_cache_append(one, tables, pools, pools, 1, R, rows, 0, FAKE, None, FAKE, None, FAKE, 16,
                                      None) == want
        assert lib.bdgdn_cache_compact(one, tables, pools, 1, R, rows, FAKE, FAKE, FAKE, None, FAKE, 16, None) == want


def test_tables_of_an_empty_cache():
    for n in (1, 31, 32, 33, 64, 95):
        t = bd.make_cache_tables(2, 3, n, device="cpu")
        assert (t.page_table == -1).all() and not t.seq_len.any() and not t.refcount.any()
        bits = [bool(int(t.free_bits[p // 32]) >> p % 32 & 1) for p in range(32 * t.free_bits.numel())]
        assert bits == [p < n for p in range(len(bits))]


def test_binding_refuses():
    x = torch.zeros(1, 2, 2, 64)
    with pytest.raises(ValueError, match="device tensor"):
        bd.bdgdn_tree_attn(x, x, x, x, x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        bd.bdgdn_verify(torch.zeros(1, 2, 3), x, x, x)
    with pytest.raises(ValueError, match="at least one pool"):
        bd.bdgdn_cache_append(bd.make_cache_tables(1, 1, 1, device="cpu"), [], [], x, x)


_EXPANDED = [((1, 1), (64, 1)), ((1, 1), (16, 4)), ((1, 1), (1, 4)), ((1, 4), (3, 4)), ((3, 1), (3, 4))]


@pytest.mark.parametrize("made,seen", _EXPANDED)
@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_attention_refuses_expanded_inputs(name, made, seen):
    """Rows that share memory have no stride that the library knows: its 0 stands for contiguous rows."""
    (R, N), d = seen, 128
    x = dict(q=torch.zeros(R, N, 8, d), k=torch.zeros(R, N, 2, d), v=torch.zeros(R, N, 2, d))

    def plan():
        pool = torch.zeros(3, 16, 2, d)
        args = [y for t in (x["q"], x["k"], x["v"], pool, pool) for y in (t.shape, t.stride())]
        return rounds._attn_plan(*args, (R, 4), R, None, torch.float32, torch.float32, bd.BDGDN_MASK_FULL)

    assert plan()[2] > 0
    x[name] = torch.zeros(*made, *x[name].shape[2:]).expand(x[name].shape)
    with pytest.raises(ValueError, match=f"{name} must have"):
        plan()


@pytest.mark.parametrize("made,seen", _EXPANDED)
def test_append_refuses_expanded_rows(made, seen):
    pool, table = torch.zeros(3, 16, 2, 64), (80, 4)

    def plan(rows):
        return rounds._pools_plan(table, 3, pool.shape, pool.stride(), torch.float32, *seen, rows.shape, rows.stride())

    assert plan(torch.zeros(*seen, 2, 64))[2] == 0
    with pytest.raises(ValueError, match=r"rows\[0\] must have"):
        plan(torch.zeros(*made, 2, 64).expand(*seen, 2, 64))


def test_rows_closer_than_their_heads_are_refused():
    base = torch.zeros(4096)
    with pytest.raises(ValueError, match="q must have"):
        x = base.as_strided((2, 3, 2, 64), (3 * 64, 64, 64, 1))
        rounds._row_stride(x.shape, x.stride(), "q")
    # dimensions of one say nothing, whatever their strides
    for shape, strides in (((1, 1, 2, 64), (0, 0, 64, 1)), ((1, 3, 2, 64), (0, 128, 64, 1)), ((3, 1, 1, 64), (64, 0, 0, 1))):
        x = base.as_strided(shape, strides)
        assert rounds._row_stride(x.shape, x.stride(), "q") == 0


def test_tables_that_know_their_page_refuse_another():
    """The tables say nothing of their page by themselves, and a call with another one would give back pages that are in use."""
    t = bd.make_cache_tables(2, 3, 40, device="cpu", page=16)
    assert t.page == 16 and len(t) == 4 and copy.copy(t).page == 16 and t._replace(seq_len=t.seq_len).page == 16
    slot = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="pages of 16"):
        bd.bdgdn_cache_fork(t, slot, slot, page=8)
    with pytest.raises(ValueError, match="pages of 16"):
        bd.bdgdn_cache_truncate(t, slot, page=64)
    with pytest.raises(ValueError, match="pages of 16"):
        rounds._page_of(t, 24)
    assert rounds._page_of(t, None) == rounds._page_of(t, 16) == 16
    unknown = bd.CacheTables(*t)
    assert unknown.page is None and rounds._page_of(unknown, 24) == 24 and rounds._page_of(tuple(t), 24) == 24
    for call in (lambda: bd.bdgdn_cache_fork(unknown, slot, slot), lambda: bd.bdgdn_cache_truncate(unknown, slot)):
        with pytest.raises(ValueError, match="page must be given"):
            call()
    with pytest.raises(ValueError, match="page must be"):
        bd.make_cache_tables(2, 3, 40, device="cpu", page=0)
