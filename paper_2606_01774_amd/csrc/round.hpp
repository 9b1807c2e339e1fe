// round.hpp -- argument blocks and host-side launchers of the kernels that serve the softmax
// half of a serving round: attention over a paged cache, verification of drafts, the cache's
// pages.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bdgdn {

// ------------------------------------------------------------------ attention (attn_kernels.hip)
struct AttnArgs {
    const void *q, *k, *v, *kp, *vp;
    const int32_t *table, *len, *slot, *count;
    const uint64_t *mask;
    void *o;
    float *lse;
    int32_t *info;             // tiles of a range; [R][2]: a request's first tile among all, its tiles
    float *part_o, *part_ml;   // the pieces' results: [range][2][h_kv][rows_padded][d], [..][2]
    int R, N, h_q, h_kv, G;    // G = h_q / h_kv query heads to a key head
    int page, max_pages, n_slots, n_pages;
    uint32_t page_mul;         // tok / page = mulhi(tok, page_mul) >> page_shift, or tok for 0 (pages of one)
    int page_shift;
    int mask_kind;             // bdgdn_mask_t
    long q_stride, k_stride, v_stride;   // bytes between nodes' rows
    long head_stride;                    // bytes between a pool's heads
    uint32_t page16, token16;            // strides of a pool in units of 16 bytes
    float c;                   // |scale| log2(e), or 1 for scale 0
    uint32_t q_and, q_xor;     // applied to the words of q: the scale's sign, or zero
    int RW, RG;                // waves of a workgroup, and workgroups, with other rows of a key head
    int rows_padded;           // rows of a key head, filled up to those of RW x RG waves
    int node_units;            // tiles that a request's nodes, queries and output count as
    int ranges, least;         // ranges that the keys are cut into, at most, and their tiles, at least
    int uncut;                 // a range is a request
};

// How a call is cut: 16-row groups of a wave, the above, workgroups, and the workspace.
struct AttnPlan {
    bool staged;               // the kernel that stages tiles in LDS
    bool uncut;                // every request is one piece
    int mt, RW, RG, rows_padded, ranges, least, grid;
    size_t ml_at, o_at, bytes;
};
AttnPlan attn_plan(bool bf16, int d, int page, long most, int R, int N, int h_q, int h_kv);
hipError_t launch_tree_attn(bool bf16, bool f32_out, int d, const AttnPlan &p, AttnArgs &a, void *workspace, hipStream_t s);
hipError_t launch_tree_attn_staged(bool f32_out, int d, int grid, const AttnArgs &a, hipStream_t s);
hipError_t launch_tree_mask(int R, int N, const int32_t *parent, uint64_t *mask, int32_t *depth, hipStream_t s);

// ------------------------------------------------------------------ verification (verify_kernels.hip)
struct VerifyArgs {
    const void *target, *draft;
    const int32_t *token, *parent, *count;
    const float *temperature, *u, *noise;
    int32_t *n_accept, *n_path, *path, *next;
    float *stats;              // [2][R * N][splits][4]: max, sum, index of the max
    void *walked, *best;       // the walks' results and the races' parts
    int R, N, V;
    int splits, part;          // parts of a row for its statistics, logits of a part
    int race_splits, race_part;
    long t_req, t_row, d_req, d_row, noise_stride;   // elements
};
struct VerifyPlan {
    int splits, part, race_splits, race_part;
    size_t walked_at, best_at, bytes;   // offsets into the workspace, its size
};
VerifyPlan verify_plan(int R, int N, int V);
hipError_t launch_verify(bool bf16, VerifyArgs &a, const VerifyPlan &p, void *workspace, hipStream_t s);

// ------------------------------------------------------------------ the cache's pages (cache_kernels.hip)

struct CacheArgs {
    int32_t *table, *len, *ref;
    uint32_t *bits;
    int n_pages, page, n_slots, max_pages;
    int R, rows_max;           // requests; rows that one may add (append) or keep (compact)
    const int32_t *slot, *path, *count;   // path: append's path or compact's positions
    int32_t *status;
    int32_t *meta, *alloc;     // workspace: kMeta ints per request, then the pages taken
    int32_t *saved;            // and, for a compaction that one workgroup plans, the tables before it
};

// Per-request words of the workspace.
enum { kOld = 0, kNew, kCow, kStart, kNeed, kOff, kStay, kMeta = 8 };

struct MoveShape {
    CacheArgs c;
    int row16, head16_log;     // 16-byte chunks of a token's row; log2 of those of a head
    long page_stride, token_stride, head_stride, row_stride;   // bytes
    long head_bytes;           // of a head in the rows to append
};

// Ints of the workspace: where each part of CacheArgs' begins, how many there are.
struct CachePlan {
    size_t alloc_at, saved_at, ints;
    bool one;                  // one workgroup plans a compaction
};

CachePlan cache_plan(int R, int rows_max, int page, int max_pages);
hipError_t launch_cache_plan(bool append, const CacheArgs &a, hipStream_t s);
hipError_t launch_cache_move(bool append, const MoveShape &m, void *const *pools, const void *const *rows, int n_pools, hipStream_t s);
hipError_t launch_cache_finish(const CacheArgs &a, hipStream_t s);
hipError_t launch_cache_fork(const CacheArgs &a, const int32_t *src, const int32_t *dst, hipStream_t s);
hipError_t launch_cache_truncate(const CacheArgs &a, hipStream_t s);

}  // namespace bdgdn
