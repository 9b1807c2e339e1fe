// round_api.hip -- the C ABI of the softmax half of a serving round: validation and dispatch
// of attention over the paged cache, verification, and the cache's pages.
#include <math.h>

#include "bdgdn.h"
#include "round.hpp"

using namespace bdgdn;

namespace {

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

int size_of(int dtype) { return dtype == BDGDN_BF16 ? 2 : 4; }

// A pool's geometry (shape: the parts that only the tables need are checked alone).
int check_tables(const bdgdn_cache_desc_t *c)
{
    if (!c) return BDGDN_ERR_INVALID_ARG;
    if (c->n_pages <= 0 || c->page <= 0 || c->n_slots <= 0 || c->max_pages <= 0) return BDGDN_ERR_INVALID_ARG;
    if (c->page > 65536 || (long)c->max_pages * c->page > 0x7fffffffL) return BDGDN_ERR_UNSUPPORTED;
    return BDGDN_OK;
}

int check_pools(const bdgdn_cache_desc_t *c)
{
    int st = check_tables(c);
    if (st != BDGDN_OK) return st;
    if (c->h_kv <= 0 || c->d <= 0) return BDGDN_ERR_INVALID_ARG;
    if (c->dtype != BDGDN_BF16 && c->dtype != BDGDN_F32) return BDGDN_ERR_UNSUPPORTED;
    if (!head_dim_ok(c->d) || c->h_kv > 65536) return BDGDN_ERR_UNSUPPORTED;
    const int64_t unit = 16 / size_of(c->dtype);
    if (c->page_stride <= 0 || c->token_stride < c->d || c->head_stride < c->d) return BDGDN_ERR_INVALID_ARG;
    if (c->page_stride % unit || c->token_stride % unit || c->head_stride % unit) return BDGDN_ERR_INVALID_ARG;
    // offsets within a tile of 32 tokens are 32-bit bytes, those within a pool 32-bit 16-byte units
    if (c->token_stride * size_of(c->dtype) > (1L << 26)) return BDGDN_ERR_UNSUPPORTED;
    const double bytes = ((double)c->n_pages * (double)c->page_stride + (double)c->page * (double)c->token_stride +
                          (double)c->h_kv * (double)c->head_stride) * size_of(c->dtype);
    if (bytes > 68719476736.0) return BDGDN_ERR_UNSUPPORTED;
    return BDGDN_OK;
}

int check_attn(const bdgdn_attn_desc_t *d, const bdgdn_cache_desc_t *c)
{
    if (!d) return BDGDN_ERR_INVALID_ARG;
    int st = check_pools(c);
    if (st != BDGDN_OK) return st;
    if (d->num_req < 0 || d->nodes <= 0 || d->h_q <= 0 || d->h_kv <= 0 || d->d <= 0) return BDGDN_ERR_INVALID_ARG;
    if (d->h_q % d->h_kv != 0 || !isfinite(d->scale)) return BDGDN_ERR_INVALID_ARG;
    if (d->h_kv != c->h_kv || d->d != c->d || d->dtype != c->dtype) return BDGDN_ERR_INVALID_ARG;
    if (d->mask != BDGDN_MASK_FULL && d->mask != BDGDN_MASK_CAUSAL && d->mask != BDGDN_MASK_BITS)
        return BDGDN_ERR_INVALID_ARG;
    const bool types = (d->dtype == BDGDN_BF16 && (d->out_dtype == BDGDN_BF16 || d->out_dtype == BDGDN_F32)) ||
                       (d->dtype == BDGDN_F32 && d->out_dtype == BDGDN_F32);
    if (!types || d->nodes > 64 || d->h_q > 65536 || d->num_req > 65535) return BDGDN_ERR_UNSUPPORTED;
    const int64_t unit = 16 / size_of(d->dtype);
    const int64_t least[3] = {(int64_t)d->h_q * d->d, (int64_t)d->h_kv * d->d, (int64_t)d->h_kv * d->d};
    const int64_t stride[3] = {d->q_stride, d->k_stride, d->v_stride};
    for (int i = 0; i < 3; ++i)
        if (stride[i] != 0 && (stride[i] < least[i] || stride[i] % unit)) return BDGDN_ERR_INVALID_ARG;
    // token numbers up to some tiles past a sequence's end
    if ((long)c->max_pages * c->page > 0x7fff0000L) return BDGDN_ERR_UNSUPPORTED;
    // workgroups of 256 threads, of which a launch has 2^32; tiles of all requests, their nodes
    // counting as eight at most
    const long rows = (long)d->nodes * (d->h_q / d->h_kv);
    if ((long)d->num_req * d->nodes * d->h_q > 0x40000000L || (long)d->num_req * d->h_kv * ((rows + 15) / 16) >= (1L << 24) ||
        (long)d->num_req * ((long)c->max_pages * c->page / 32 + 9) > 0x7fff0000L)
        return BDGDN_ERR_UNSUPPORTED;
    return BDGDN_OK;
}

// Requests are a grid's second dimension, and the pages that a call may take a 32-bit count.
bool countable(const bdgdn_cache_desc_t *c, int32_t num_req, int32_t rows_max)
{
    return num_req <= 65535 && (long)num_req * (((long)rows_max + c->page - 1) / c->page + 1) <= 0x40000000L;
}

int check_verify(const bdgdn_verify_desc_t *d)
{
    if (!d) return BDGDN_ERR_INVALID_ARG;
    if (d->num_req < 0 || d->nodes <= 0 || d->vocab <= 0) return BDGDN_ERR_INVALID_ARG;
    if (d->dtype != BDGDN_BF16 && d->dtype != BDGDN_F32) return BDGDN_ERR_UNSUPPORTED;
    if (d->nodes > 64 || d->num_req > 65535 || d->vocab > 0x40000000) return BDGDN_ERR_UNSUPPORTED;
    if (d->target_req_stride < 0 || d->target_row_stride < 0 || d->draft_req_stride < 0 || d->draft_row_stride < 0 ||
        d->noise_stride < 0)
        return BDGDN_ERR_INVALID_ARG;
    return BDGDN_OK;
}

int status_of(hipError_t e) { return e == hipSuccess ? BDGDN_OK : BDGDN_ERR_LAUNCH; }

CacheArgs cache_args(const bdgdn_cache_desc_t *c, const bdgdn_cache_tables_t *t, int R, const int32_t *slot,
                     int32_t *status)
{
    CacheArgs a = {};
    a.table = t->page_table; a.len = t->seq_len; a.ref = t->refcount; a.bits = t->free_bits;
    a.n_pages = c->n_pages; a.page = c->page; a.n_slots = c->n_slots; a.max_pages = c->max_pages;
    a.R = R; a.slot = slot; a.status = status;
    return a;
}

bool tables_there(const bdgdn_cache_tables_t *t)
{
    return t && t->page_table && t->seq_len && t->refcount && t->free_bits;
}

hipError_t move_pools(bool append, const bdgdn_cache_desc_t *c, const CacheArgs &ca, void *const *pools,
                      const void *const *rows, int n_pools, int64_t row_stride, hipStream_t s)
{
    const long size = size_of(c->dtype);
    MoveShape m = {};
    m.c = ca;
    m.row16 = (int)(c->h_kv * c->d * size / 16);
    while ((16L << m.head16_log) < c->d * size) ++m.head16_log;
    m.page_stride = c->page_stride * size;
    m.token_stride = c->token_stride * size;
    m.head_stride = c->head_stride * size;
    m.row_stride = (row_stride ? row_stride : (int64_t)c->h_kv * c->d) * size;
    m.head_bytes = c->d * size;
    return launch_cache_move(append, m, pools, rows, n_pools, s);
}

size_t cache_workspace(const bdgdn_cache_desc_t *c, int32_t num_req, int32_t rows_max)
{
    return (cache_plan(num_req, rows_max, c->page, c->max_pages).ints * 4 + 255) & ~(size_t)255;
}

// The parts of a workspace.
void place_workspace(CacheArgs &a, const bdgdn_cache_desc_t *c, void *workspace)
{
    const CachePlan p = cache_plan(a.R, a.rows_max, c->page, c->max_pages);
    a.meta = static_cast<int32_t *>(workspace);
    a.alloc = a.meta + p.alloc_at;
    a.saved = p.one ? a.meta + p.saved_at : nullptr;
}

int check_pool_list(void *const *pools, const void *const *rows, bool with_rows, int n_pools)
{
    if (n_pools < 0 || (n_pools > 0 && (!pools || (with_rows && !rows)))) return BDGDN_ERR_INVALID_ARG;
    for (int i = 0; i < n_pools; ++i) {
        if (!pools[i] || !aligned(pools[i], 16)) return BDGDN_ERR_INVALID_ARG;
        if (with_rows && (!rows[i] || !aligned(rows[i], 16))) return BDGDN_ERR_INVALID_ARG;
    }
    return BDGDN_OK;
}

}  // namespace

extern "C" {

size_t bdgdn_tree_attn_workspace(const bdgdn_attn_desc_t *desc, const bdgdn_cache_desc_t *cache)
{
    if (check_attn(desc, cache) != BDGDN_OK || desc->num_req == 0) return 0;
    return attn_plan(desc->dtype == BDGDN_BF16, desc->d, cache->page, (long)cache->max_pages * cache->page, desc->num_req, desc->nodes, desc->h_q, desc->h_kv).bytes;
}

int bdgdn_tree_attn(const bdgdn_attn_desc_t *desc, const bdgdn_cache_desc_t *cache, const void *q,
                    const void *k, const void *v, const void *k_pages, const void *v_pages,
                    const int32_t *page_table, const int32_t *seq_len, const int32_t *slot,
                    const int32_t *count, const uint64_t *mask, void *o, float *lse,
                    void *workspace, size_t workspace_bytes, void *stream)
{
    int st = check_attn(desc, cache);
    if (st != BDGDN_OK) return st;
    if (desc->num_req == 0) return BDGDN_OK;
    if (!q || !k || !v || !k_pages || !v_pages || !page_table || !seq_len || !o) return BDGDN_ERR_INVALID_ARG;
    if ((desc->mask == BDGDN_MASK_BITS) != (mask != nullptr)) return BDGDN_ERR_INVALID_ARG;
    if (!slot && desc->num_req > cache->n_slots) return BDGDN_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) ||
        !aligned(o, 16) || !aligned(mask, 8))
        return BDGDN_ERR_INVALID_ARG;
    const bool bf16 = desc->dtype == BDGDN_BF16;
    const AttnPlan p = attn_plan(bf16, desc->d, cache->page, (long)cache->max_pages * cache->page, desc->num_req, desc->nodes, desc->h_q, desc->h_kv);
    if (!aligned(workspace, 256)) return BDGDN_ERR_INVALID_ARG;
    if (workspace_bytes < p.bytes || !workspace) return BDGDN_ERR_WORKSPACE;
    const long size = size_of(desc->dtype);
    AttnArgs a = {};
    a.q = q; a.k = k; a.v = v; a.kp = k_pages; a.vp = v_pages;
    a.table = page_table; a.len = seq_len; a.slot = slot; a.count = count; a.mask = mask;
    a.o = o; a.lse = lse;
    a.R = desc->num_req; a.N = desc->nodes; a.h_q = desc->h_q; a.h_kv = desc->h_kv; a.G = desc->h_q / desc->h_kv;
    a.page = cache->page; a.max_pages = cache->max_pages; a.n_slots = cache->n_slots; a.n_pages = cache->n_pages;
    // tok / page for tok < 2^31: with 2^(l-1) < page <= 2^l, m = ceil(2^(31+l) / page) < 2^32 and
    // tok m >> (31 + l) is exact (m page - 2^(31+l) < 2^l)
    if (cache->page > 1) {
        int l = 1;
        while ((1 << l) < cache->page) ++l;
        a.page_mul = (uint32_t)(((1ull << (31 + l)) + cache->page - 1) / cache->page);
        a.page_shift = l - 1;
    }
    a.mask_kind = desc->mask;
    a.q_stride = (desc->q_stride ? desc->q_stride : (int64_t)desc->h_q * desc->d) * size;
    a.k_stride = (desc->k_stride ? desc->k_stride : (int64_t)desc->h_kv * desc->d) * size;
    a.v_stride = (desc->v_stride ? desc->v_stride : (int64_t)desc->h_kv * desc->d) * size;
    a.head_stride = cache->head_stride * size;
    a.page16 = (uint32_t)(cache->page_stride * size / 16);
    a.token16 = (uint32_t)(cache->token_stride * size / 16);
    // scale s: the sign goes into q's (exactly), so that the largest score is the largest
    // product; scale 0 makes every product 0
    a.c = desc->scale == 0.f ? 1.f : fminf(fabsf(desc->scale) * 1.4426950408889634f, 3.402823466e38f);
    a.q_and = desc->scale == 0.f ? 0u : ~0u;
    a.q_xor = desc->scale < 0.f ? (bf16 ? 0x80008000u : 0x80000000u) : 0u;
    return status_of(launch_tree_attn(bf16, desc->out_dtype == BDGDN_F32, desc->d, p, a, workspace,
                                      static_cast<hipStream_t>(stream)));
}

int bdgdn_tree_mask(int32_t num_req, int32_t nodes, const int32_t *parent, uint64_t *mask, int32_t *depth, void *stream)
{
    if (num_req < 0 || nodes <= 0) return BDGDN_ERR_INVALID_ARG;
    if (nodes > 64) return BDGDN_ERR_UNSUPPORTED;
    if (num_req == 0) return BDGDN_OK;
    if (!parent || !mask || !aligned(mask, 8)) return BDGDN_ERR_INVALID_ARG;
    return status_of(launch_tree_mask(num_req, nodes, parent, mask, depth, static_cast<hipStream_t>(stream)));
}

size_t bdgdn_verify_workspace(const bdgdn_verify_desc_t *desc)
{
    if (check_verify(desc) != BDGDN_OK || desc->num_req == 0) return 0;
    return verify_plan(desc->num_req, desc->nodes, desc->vocab).bytes;
}

int bdgdn_verify(const bdgdn_verify_desc_t *desc, const void *target, const void *draft,
                 const int32_t *token, const int32_t *parent, const int32_t *count,
                 const float *temperature, const float *u, const float *noise, int32_t *n_accept,
                 int32_t *n_path, int32_t *path, int32_t *next_token, void *workspace,
                 size_t workspace_bytes, void *stream)
{
    int st = check_verify(desc);
    if (st != BDGDN_OK) return st;
    if (desc->num_req == 0) return BDGDN_OK;
    if (!target || !token || !u || !noise || !n_accept || !path || !next_token) return BDGDN_ERR_INVALID_ARG;
    const size_t size = size_of(desc->dtype);
    if (!aligned(target, size) || !aligned(draft, size) || !aligned(workspace, 256)) return BDGDN_ERR_INVALID_ARG;
    const VerifyPlan plan = verify_plan(desc->num_req, desc->nodes, desc->vocab);
    if (workspace_bytes < plan.bytes || !workspace) return BDGDN_ERR_WORKSPACE;
    VerifyArgs a = {};
    a.target = target; a.draft = draft; a.token = token; a.parent = parent; a.count = count;
    a.temperature = temperature; a.u = u; a.noise = noise;
    a.n_accept = n_accept; a.n_path = n_path; a.path = path; a.next = next_token;
    a.R = desc->num_req; a.N = desc->nodes; a.V = desc->vocab;
    a.t_req = desc->target_req_stride; a.t_row = desc->target_row_stride;
    a.d_req = desc->draft_req_stride; a.d_row = desc->draft_row_stride;
    a.noise_stride = desc->noise_stride;
    return status_of(launch_verify(desc->dtype == BDGDN_BF16, a, plan, workspace, static_cast<hipStream_t>(stream)));
}

size_t bdgdn_cache_workspace(const bdgdn_cache_desc_t *cache, int32_t num_req, int32_t rows_max)
{
    if (check_tables(cache) != BDGDN_OK || num_req <= 0 || rows_max < 0 || !countable(cache, num_req, rows_max)) return 0;
    return cache_workspace(cache, num_req, rows_max);
}

int bdgdn_cache_append(const bdgdn_cache_desc_t *cache, const bdgdn_cache_tables_t *tables, void *const *pools,
                       const void *const *rows, int32_t n_pools, int32_t num_req, int32_t nodes,
                       int64_t row_stride, const int32_t *slot, const int32_t *path, const int32_t *count,
                       int32_t *status, void *workspace, size_t workspace_bytes, void *stream)
{
    int st = check_pools(cache);
    if (st != BDGDN_OK) return st;
    if (num_req < 0 || nodes < 0) return BDGDN_ERR_INVALID_ARG;
    const int64_t unit = 16 / size_of(cache->dtype);
    if (row_stride != 0 && (row_stride < (int64_t)cache->h_kv * cache->d || row_stride % unit)) return BDGDN_ERR_INVALID_ARG;
    if (!countable(cache, num_req, nodes)) return BDGDN_ERR_UNSUPPORTED;
    if (num_req == 0) return BDGDN_OK;
    if (!tables_there(tables) || !slot || !count) return BDGDN_ERR_INVALID_ARG;
    st = check_pool_list(pools, rows, nodes > 0, n_pools);
    if (st != BDGDN_OK) return st;
    if (!aligned(workspace, 256)) return BDGDN_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < cache_workspace(cache, num_req, nodes)) return BDGDN_ERR_WORKSPACE;
    CacheArgs a = cache_args(cache, tables, num_req, slot, status);
    a.rows_max = nodes; a.path = path; a.count = count;
    place_workspace(a, cache, workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = launch_cache_plan(true, a, s);
    if (e == hipSuccess && nodes > 0) e = move_pools(true, cache, a, pools, rows, n_pools, row_stride, s);
    return status_of(e);
}

int bdgdn_cache_fork(const bdgdn_cache_desc_t *cache, const bdgdn_cache_tables_t *tables, int32_t num_req,
                     const int32_t *src, const int32_t *dst, int32_t *status, void *stream)
{
    int st = check_tables(cache);
    if (st != BDGDN_OK) return st;
    if (num_req < 0) return BDGDN_ERR_INVALID_ARG;
    if (num_req == 0) return BDGDN_OK;
    if (!tables_there(tables) || !src || !dst) return BDGDN_ERR_INVALID_ARG;
    return status_of(launch_cache_fork(cache_args(cache, tables, num_req, nullptr, status), src, dst,
                                       static_cast<hipStream_t>(stream)));
}

int bdgdn_cache_compact(const bdgdn_cache_desc_t *cache, const bdgdn_cache_tables_t *tables, void *const *pools,
                        int32_t n_pools, int32_t num_req, int32_t keep_max, const int32_t *slot,
                        const int32_t *keep, const int32_t *count, int32_t *status, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    int st = check_pools(cache);
    if (st != BDGDN_OK) return st;
    if (num_req < 0 || keep_max < 0) return BDGDN_ERR_INVALID_ARG;
    if (!countable(cache, num_req, keep_max)) return BDGDN_ERR_UNSUPPORTED;
    if (num_req == 0) return BDGDN_OK;
    if (!tables_there(tables) || !slot || !count || (keep_max > 0 && !keep)) return BDGDN_ERR_INVALID_ARG;
    st = check_pool_list(pools, nullptr, false, n_pools);
    if (st != BDGDN_OK) return st;
    if (!aligned(workspace, 256)) return BDGDN_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < cache_workspace(cache, num_req, keep_max)) return BDGDN_ERR_WORKSPACE;
    CacheArgs a = cache_args(cache, tables, num_req, slot, status);
    a.rows_max = keep_max; a.path = keep; a.count = count;
    place_workspace(a, cache, workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = launch_cache_plan(false, a, s);
    if (e == hipSuccess && keep_max > 0) e = move_pools(false, cache, a, pools, nullptr, n_pools, 0, s);
    if (e == hipSuccess && !a.saved) e = launch_cache_finish(a, s);
    return status_of(e);
}

int bdgdn_cache_truncate(const bdgdn_cache_desc_t *cache, const bdgdn_cache_tables_t *tables, int32_t num_req,
                         const int32_t *slot, const int32_t *length, void *stream)
{
    int st = check_tables(cache);
    if (st != BDGDN_OK) return st;
    if (num_req < 0) return BDGDN_ERR_INVALID_ARG;
    if (num_req == 0) return BDGDN_OK;
    if (!tables_there(tables) || !slot) return BDGDN_ERR_INVALID_ARG;
    CacheArgs a = cache_args(cache, tables, num_req, slot, nullptr);
    a.count = length;
    return status_of(launch_cache_truncate(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
