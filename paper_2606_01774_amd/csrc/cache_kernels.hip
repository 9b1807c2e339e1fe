// cache_kernels.hip -- the pages of a cache of keys and values: append (copy on write), fork,
// compact, truncate.  The tables are integers on the device, so that a server's round needs
// no trip to the host; the lowest free pages are taken in the order of the requests, so that
// the tables do not depend on the order in which workgroups run.  A plan kernel of one
// workgroup takes the pages, move kernels copy rows in 16-byte chunks.
//
// What bounds it: the copies memory, the rest launches.  Compacting 8 sequences of up to 4096
// tokens to their halves in 4 pools: move 40 us (5.4 TB/s read and written), keep 5.5, plan 7.8,
// finish 4.7.  Appending to 64 sequences in 8 pools: plan 5.5, move 5.0; to 64 that share their
// last page with others: plan 7.7, move 12.9 (5.6 TB/s).  A fork is 3.4 us, a truncation 3.6.
// Small calls are bound by the host's launches, about 3 us each.  An append's plan gives a request's
// new pages out one after the other, a quarter of a microsecond each: a prompt of 4096 tokens takes 26 us in
// pages of 64, 71 in pages of 16, 1.02 ms in pages of one.
#include "kernels.hpp"
#include "round.hpp"

namespace bdgdn {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kOneRequests = 256;   // of a compaction that one workgroup plans
enum { kDone = 0, kNoPages = 1, kNoRoom = 2, kBadSlot = 3, kBadKeep = 4 };

typedef unsigned int u32x4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int pages_of(int tokens, int page) { return (int)(((unsigned)tokens + page - 1) / (unsigned)page); }

__device__ __forceinline__ int seq_of(const CacheArgs &a, int slot)
{
    return min(max(a.len[slot], 0), a.max_pages * a.page);
}

// Sum of x over the threads before this one, and over all of them (every thread calls it).
__device__ __forceinline__ int block_scan(int x, int &total, int *lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int inc = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(inc, o);
        if (lane >= o) inc += y;
    }
    if (lane == 63) lds[wave] = inc;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        const int y = lds[w];
        if (w < wave) before += y;
        total += y;
    }
    __syncthreads();
    return before + inc - x;
}

__device__ __forceinline__ void give_back(const CacheArgs &a, int page)
{
    if ((unsigned)page < (unsigned)a.n_pages && atomicSub(&a.ref[page], 1) == 1)
        atomicOr(&a.bits[page >> 5], 1u << (page & 31));
}

// What request f needs: its words of meta but kOff.  Returns the pages it needs.
template <bool APPEND> __device__ int plan_request(const CacheArgs &a, int f)
{
    int32_t *m = a.meta + (long)f * kMeta;
    const int slot = a.slot[f];
    int st = kDone, n = min(max(a.count[f], 0), a.rows_max), old = 0, cow = -1, start = 0, need = 0;
    if ((unsigned)slot >= (unsigned)a.n_slots) {
        st = kBadSlot;
    } else {
        old = seq_of(a, slot);
        if (APPEND) {
            if (n > a.max_pages * a.page - old) {
                st = kNoRoom;
            } else if (n > 0) {
                start = pages_of(old, a.page);
                if (old % a.page) {
                    const int last = a.table[(long)slot * a.max_pages + start - 1];
                    const bool there = (unsigned)last < (unsigned)a.n_pages;
                    if (!there || a.ref[last] > 1) {
                        --start;
                        cow = there ? last : -2;   // -2: a new page for one that is not there
                    }
                }
                need = pages_of(old + n, a.page) - start;
            }
        } else {
            const int stay = m[kStay];
            if (stay < 0) st = kBadKeep;
            else {
                start = stay == n ? pages_of(stay, a.page) : stay / a.page;
                need = pages_of(n, a.page) - start;
            }
        }
    }
    m[kOld] = old;
    m[kNew] = st == kDone ? n : -1;
    m[kCow] = cow;
    m[kStart] = start;
    m[kNeed] = need;
    if (a.status) a.status[f] = st;
    return need;
}

// Do the positions of each request rise, are they there, how many stay in place (-1: they are
// bad); and the tables as they are.  By the plan kernel's workgroup, 512 positions to a wave's turn.
__device__ void look_at_keeps(const CacheArgs &a)
{
    __shared__ int s_stay[kOneRequests], s_bad[kOneRequests];
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < a.R) s_stay[tid] = s_bad[tid] = 0;
    __syncthreads();
    const int turns = (a.rows_max + 511) / 512;
    for (int x = tid >> 6; x < a.R * turns; x += kPlanThreads / 64) {
        const int f = x / turns, j0 = (x - f * turns) * 512, slot = a.slot[f], n = min(max(a.count[f], 0), a.rows_max);
        const int old = (unsigned)slot < (unsigned)a.n_slots ? seq_of(a, slot) : 0;
        const int32_t *keep = a.path + (long)f * a.rows_max;
        int stay = 0;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = j0 + 64 * i + lane;
            if (j < n) {
                const int t = keep[j], before = j > 0 ? keep[j - 1] : -1;
                stay += t == j;
                bad |= t < 0 || t >= old || before >= t;
            }
        }
        if (stay) atomicAdd(&s_stay[f], stay);
        if (bad) s_bad[f] = 1;
    }
    for (int x = tid; x < a.R * a.max_pages; x += kPlanThreads) {
        const int f = x / a.max_pages, i = x - f * a.max_pages, slot = a.slot[f];
        if ((unsigned)slot < (unsigned)a.n_slots && i < pages_of(seq_of(a, slot), a.page))
            a.saved[x] = a.table[(long)slot * a.max_pages + i];
    }
    __syncthreads();
    if (tid < a.R) a.meta[(long)tid * kMeta + kStay] = s_bad[tid] ? -1 : s_stay[tid];
    __syncthreads();
}

template <bool APPEND> __global__ void __launch_bounds__(kPlanThreads) bdgdn_cache_plan_kernel(CacheArgs a)
{
    __shared__ int lds[kPlanThreads / 64];
    __shared__ int s_granted;
    const int tid = threadIdx.x;
    if (!APPEND && a.saved) look_at_keeps(a);
    int want = 0;
    for (int f0 = 0; f0 < a.R; f0 += kPlanThreads) {
        const int f = f0 + tid;
        const int need = f < a.R ? plan_request<APPEND>(a, f) : 0;
        int total;
        const int before = block_scan(need, total, lds);
        if (f < a.R) a.meta[(long)f * kMeta + kOff] = want + before;
        want += total;
    }
    // the lowest `want` free pages
    const int words = (a.n_pages + 31) >> 5;
    int found = 0;
    for (int w0 = 0; w0 < words && found < want; w0 += kPlanThreads) {
        const int w = w0 + tid;
        unsigned x = w < words ? a.bits[w] : 0u;
        if (w == words - 1 && (a.n_pages & 31)) x &= (1u << (a.n_pages & 31)) - 1;
        int total;
        int at = found + block_scan(__popc(x), total, lds);
        while (x && at < want) {
            a.alloc[at++] = (w << 5) + __ffs(x) - 1;
            x &= x - 1;
        }
        found += total;
    }
    if (tid == 0) s_granted = want;
    __syncthreads();
    if (found < want && tid == 0) {   // too few: in order, whoever still fits
        int used = 0;
        for (int f = 0; f < a.R; ++f) {
            int32_t *m = a.meta + (long)f * kMeta;
            if (m[kNeed] > found - used) {
                m[kNew] = -1;
                m[kNeed] = 0;
                m[kCow] = -1;
                if (a.status) a.status[f] = kNoPages;
            }
            m[kOff] = used;
            used += m[kNeed];
        }
        s_granted = used;
    }
    __syncthreads();
    const int granted = s_granted;
    for (int i = tid; i < granted; i += kPlanThreads) {
        const int p = a.alloc[i];
        atomicAnd(&a.bits[p >> 5], ~(1u << (p & 31)));
        a.ref[p] = 1;
    }
    if (!APPEND) {
        if (!a.saved) return;
        // the compacted sequences' tables: the rows' moves go by the saved ones
        for (int x = tid; x < a.R * a.max_pages; x += kPlanThreads) {
            const int f = x / a.max_pages, i = x - f * a.max_pages;
            const int32_t *m = a.meta + (long)f * kMeta;
            if (m[kNew] < 0 || i < m[kStart] || i >= pages_of(m[kOld], a.page)) continue;
            give_back(a, a.saved[x]);
            a.table[(long)a.slot[f] * a.max_pages + i] = i < m[kStart] + m[kNeed] ? a.alloc[m[kOff] + i - m[kStart]] : -1;
        }
        for (int f = tid; f < a.R; f += kPlanThreads) {
            const int n = a.meta[(long)f * kMeta + kNew];
            if (n >= 0) a.len[a.slot[f]] = n;
        }
        return;
    }
    for (int f = tid; f < a.R; f += kPlanThreads) {
        const int32_t *m = a.meta + (long)f * kMeta;
        if (m[kNew] <= 0) continue;
        const int slot = a.slot[f];
        int32_t *row = a.table + (long)slot * a.max_pages + m[kStart];
        for (int i = 0; i < m[kNeed]; ++i) row[i] = a.alloc[m[kOff] + i];
        if (m[kCow] >= 0) give_back(a, m[kCow]);
        a.len[slot] = m[kOld] + m[kNew];
    }
}

// One workgroup per request: do its positions rise, are they there, how many stay in place.
__global__ void __launch_bounds__(256) bdgdn_cache_keep_kernel(CacheArgs a)
{
    __shared__ int s_stay, s_bad;
    const int f = blockIdx.x, slot = a.slot[f];
    if (threadIdx.x == 0) s_stay = s_bad = 0;
    __syncthreads();
    const int n = min(max(a.count[f], 0), a.rows_max);
    const int old = (unsigned)slot < (unsigned)a.n_slots ? seq_of(a, slot) : 0;
    const int32_t *keep = a.path + (long)f * a.rows_max;
    int stay = 0, bad = 0;
    for (int j = threadIdx.x; j < n; j += 256) {
        const int t = keep[j];
        stay += t == j;
        bad |= t < 0 || t >= old || (j > 0 && keep[j - 1] >= t);
    }
    if (stay) atomicAdd(&s_stay, stay);
    if (bad) s_bad = 1;
    __syncthreads();
    if (threadIdx.x == 0) a.meta[(long)f * kMeta + kStay] = s_bad ? -1 : s_stay;
}

// The compacted sequences' tables, after their rows have moved.
__global__ void __launch_bounds__(256) bdgdn_cache_finish_kernel(CacheArgs a)
{
    const int f = blockIdx.x;
    const int32_t *m = a.meta + (long)f * kMeta;
    if (m[kNew] < 0) return;
    const int slot = a.slot[f], start = m[kStart], need = m[kNeed], had = pages_of(m[kOld], a.page);
    int32_t *row = a.table + (long)slot * a.max_pages;
    for (int i = start + threadIdx.x; i < had; i += 256) {
        give_back(a, row[i]);
        row[i] = i < start + need ? a.alloc[m[kOff] + i - start] : -1;
    }
    if (threadIdx.x == 0) a.len[slot] = m[kNew];
}

template <int POOLS> struct MoveArgs : MoveShape {
    unsigned char *pool[POOLS];
    const unsigned char *rows[POOLS];
};

// Copies 16-byte chunks: grid (chunks, requests, pools).
template <bool APPEND, int POOLS> __global__ void __launch_bounds__(256) bdgdn_cache_move_kernel(MoveArgs<POOLS> a)
{
    const CacheArgs &c = a.c;
    const int f = blockIdx.y;
    const int32_t *m = c.meta + (long)f * kMeta;
    const int n = m[kNew];
    if (n <= 0) return;
    const int slot = c.slot[f], old = m[kOld];
    const int32_t *row = !APPEND && c.saved ? c.saved + (long)f * c.max_pages : c.table + (long)slot * c.max_pages;
    // append: tokens from `first` on, of which the first `copied` come from a shared page or, where
    // there is none, are zeros (the new page may hold another sequence's rows);
    // compact: tokens from `first` on come from the positions kept
    const int copied = APPEND && m[kCow] != -1 ? old % c.page : 0;
    const int first = APPEND ? old - copied : min(m[kStart] * c.page, n);
    const int rows = APPEND ? n + copied : n - first;
    unsigned char *pool = a.pool[blockIdx.z];
    const long chunks = (long)rows * a.row16;
    for (long x = (long)blockIdx.x * 256 + threadIdx.x; x < chunks; x += (long)gridDim.x * 256) {
        const int j = (int)(x / a.row16), ch = (int)(x - (long)j * a.row16);
        const int h = ch >> a.head16_log, e = (ch - (h << a.head16_log)) * 16;
        const int t = first + j;
        const long head = h * a.head_stride + e;
        u32x4v val = {0, 0, 0, 0};
        int to;
        if (APPEND) {
            to = row[t / c.page];
            if (j < copied) {
                if (m[kCow] >= 0)
                    val = *reinterpret_cast<const u32x4v *>(pool + m[kCow] * a.page_stride + j * a.token_stride + head);
            } else {
                const int i = j - copied;
                const int node = c.path ? c.path[(long)f * c.rows_max + i] : i;
                if ((unsigned)node < (unsigned)c.rows_max)
                    val = *reinterpret_cast<const u32x4v *>(a.rows[blockIdx.z] + ((long)f * c.rows_max + node) * a.row_stride +
                                                            h * a.head_bytes + e);
            }
        } else {
            const int s = c.path[(long)f * c.rows_max + t], from = row[s / c.page];
            to = c.alloc[m[kOff] + t / c.page - m[kStart]];
            if ((unsigned)from < (unsigned)c.n_pages)
                val = *reinterpret_cast<const u32x4v *>(pool + from * a.page_stride + (s % c.page) * a.token_stride + head);
        }
        if ((unsigned)to < (unsigned)c.n_pages)
            *reinterpret_cast<u32x4v *>(pool + to * a.page_stride + (t % c.page) * a.token_stride + head) = val;
    }
}

__global__ void __launch_bounds__(256) bdgdn_cache_fork_kernel(CacheArgs a, const int32_t *src, const int32_t *dst)
{
    const int f = blockIdx.x, s = src[f], d = dst[f];
    const bool ok = (unsigned)s < (unsigned)a.n_slots && (unsigned)d < (unsigned)a.n_slots && a.len[d] == 0;
    __syncthreads();   // every thread has seen the length that thread 0 sets
    if (threadIdx.x == 0 && a.status) a.status[f] = ok ? kDone : kBadSlot;
    if (!ok) return;
    const int n = seq_of(a, s), pages = pages_of(n, a.page);
    for (int i = threadIdx.x; i < pages; i += 256) {
        const int p = a.table[(long)s * a.max_pages + i];
        a.table[(long)d * a.max_pages + i] = p;
        if ((unsigned)p < (unsigned)a.n_pages) atomicAdd(&a.ref[p], 1);
    }
    if (threadIdx.x == 0) a.len[d] = n;
}

__global__ void __launch_bounds__(256) bdgdn_cache_truncate_kernel(CacheArgs a)
{
    const int f = blockIdx.x, slot = a.slot[f];
    if ((unsigned)slot >= (unsigned)a.n_slots) return;
    const int old = seq_of(a, slot), n = a.count ? min(max(a.count[f], 0), old) : 0;
    __syncthreads();   // as above
    int32_t *row = a.table + (long)slot * a.max_pages;
    for (int i = pages_of(n, a.page) + threadIdx.x; i < pages_of(old, a.page); i += 256) {
        give_back(a, row[i]);
        row[i] = -1;
    }
    if (threadIdx.x == 0) a.len[slot] = n;
}

}  // namespace

// One workgroup plans a small compaction (it looks at the positions and tables itself and sets the
// tables: two launches in all).  For others a kernel of a workgroup per request comes before it and
// another after the moves.  Fork, truncate and compact of 1 to 64 sequences with up to 6400
// positions to keep: 31 to 33 us with one, 37 to 40 with all; with 16384 positions 63 and 63, with
// 32768 68 and 59.
CachePlan cache_plan(int R, int rows_max, int page, int max_pages)
{
    CachePlan p;
    p.one = R <= kOneRequests && (long)R * rows_max <= 8192 && (long)R * max_pages <= 8192;
    p.alloc_at = (size_t)R * kMeta;
    p.saved_at = p.alloc_at + (size_t)R * (((size_t)rows_max + page - 1) / page + 1);
    p.ints = p.saved_at + (p.one ? (size_t)R * max_pages : 0);
    return p;
}

hipError_t launch_cache_plan(bool append, const CacheArgs &a, hipStream_t s)
{
    if (append) {
        bdgdn_cache_plan_kernel<true><<<1, kPlanThreads, 0, s>>>(a);
    } else {
        if (!a.saved) bdgdn_cache_keep_kernel<<<a.R, 256, 0, s>>>(a);
        bdgdn_cache_plan_kernel<false><<<1, kPlanThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

namespace {

// Moves in `n` <= POOLS pools.
template <int POOLS> hipError_t move_some(bool append, const MoveShape &m, void *const *pools, const void *const *rows, int n, hipStream_t s)
{
    MoveArgs<POOLS> a;
    static_cast<MoveShape &>(a) = m;
    for (int i = 0; i < n; ++i) {
        a.pool[i] = static_cast<unsigned char *>(pools[i]);
        a.rows[i] = rows ? static_cast<const unsigned char *>(rows[i]) : nullptr;
    }
    const long most = (long)m.c.rows_max + (append ? m.c.page - 1 : 0);
    const long blocks = (most * m.row16 + 1023) / 1024;
    const dim3 grid((unsigned)(blocks < 1 ? 1 : blocks > 256 ? 256 : blocks), m.c.R, n);
    if (append) bdgdn_cache_move_kernel<true, POOLS><<<grid, 256, 0, s>>>(a);
    else bdgdn_cache_move_kernel<false, POOLS><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

// (what a launch's arguments weigh costs the host: an append to 8 pools takes 30.6 us with room for
// 16 pools' addresses, 31.3 with room for 96)
hipError_t launch_cache_move(bool append, const MoveShape &m, void *const *pools, const void *const *rows, int n_pools, hipStream_t s)
{
    if (n_pools <= 16) return n_pools > 0 ? move_some<16>(append, m, pools, rows, n_pools, s) : hipSuccess;
    for (int p0 = 0; p0 < n_pools; p0 += 96) {
        const int n = n_pools - p0 < 96 ? n_pools - p0 : 96;
        const hipError_t e = move_some<96>(append, m, pools + p0, rows ? rows + p0 : nullptr, n, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_cache_finish(const CacheArgs &a, hipStream_t s)
{
    bdgdn_cache_finish_kernel<<<a.R, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_cache_fork(const CacheArgs &a, const int32_t *src, const int32_t *dst, hipStream_t s)
{
    bdgdn_cache_fork_kernel<<<a.R, 256, 0, s>>>(a, src, dst);
    return hipGetLastError();
}

hipError_t launch_cache_truncate(const CacheArgs &a, hipStream_t s)
{
    bdgdn_cache_truncate_kernel<<<a.R, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace bdgdn
