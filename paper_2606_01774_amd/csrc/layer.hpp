// layer.hpp -- argument blocks and host-side launchers of the kernels around a hybrid layer's
// mixers: rotary positions, norms with gate and residual, logits, products of 8-bit integers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bdgdn {

// ------------------------------------------------------------------ rotary positions (rope_kernels.hip)
struct RopeArgs {
    const unsigned char *x[2];
    unsigned char *y[2];
    long xs[2][3], ys[2][3];   // bytes between requests, rows, heads
    const uint64_t *turns;
    const int32_t *pos, *len, *slot, *count;
    int R, N, h_q, h;          // h: heads of q and k
    int d, rot, n_slots;
    int in_place;
    float scale, sine;         // sine: +-scale
    // how the work is cut: 2^item_log lanes to the pieces of a head, 2^sub_log head-lanes to a row of
    // a workgroup, 2^row_log rows to a workgroup
    int items, turned, item_log, sub_log, row_log;   // items: pieces, of which the first `turned` turn
};
hipError_t launch_rope(bool bf16, bool pairs, RopeArgs &a, hipStream_t s);

// ------------------------------------------------------------------ norms (norm_kernels.hip, norm_bwd_kernels.hip)
struct RowStride {
    long outer, inner;         // elements
};
struct NormArgs {
    const void *x, *z, *r;     // backward: r is the stored sum
    const float *w_post, *w_pre, *ls;
    void *r_out, *y;
    const void *dy, *dr_out;
    void *dx, *dz, *dr;
    float *dw[3];              // post, pre, layer scale
    float *part;               // [workgroups][3][d], backward
    RowStride sx, sz, sr, sro, sy, sdx, sdz, sdr, sdro, sdy;
    int rows, inner, d;
    int post, pre, act;
    float scale, eps, inv_d;
    int groups;
};
// Types of x, of the residual, of the gate and y: fp32 (true) or bf16.
hipError_t launch_norm_fwd(bool xf, bool rf, bool yf, NormArgs &a, hipStream_t s);
hipError_t launch_norm_bwd(bool xf, bool rf, bool yf, NormArgs &a, hipStream_t s);
int norm_bwd_groups(int rows, int d);   // workgroups of the backward pass, each of which leaves partial sums

// ------------------------------------------------------------------ logits (logits_kernels.hip)
struct LogitsArgs {
    const void *x;
    void *y;
    const int32_t *history, *slot, *token, *count, *bias_token;
    const uint64_t *mask;
    const float *repetition, *presence, *frequency, *bias;
    const uint32_t *allow;
    int R, N, V, n_slots, n_bias;
    long x_req, x_row, y_req, y_row, h_row, a_req, a_row;   // elements
    int group;                 // nodes to a workgroup
};
hipError_t launch_logits(bool bf16, bool f32_out, LogitsArgs &a, hipStream_t s);
hipError_t launch_history_add(int R, int N, int V, int n_slots, long row, int32_t *history, const int32_t *slot,
                              const int32_t *token, const int32_t *path, const int32_t *count, int prompt, hipStream_t s);

// ------------------------------------------------------------------ 8-bit products (quant_kernels.hip)
struct QuantArgs {
    const void *x;
    int8_t *q;
    float *scale;
    int rows, cols, width;
    long xs, qs;
};
struct QuantMatmulArgs {
    const int8_t *a, *w;
    const float *as, *ws, *bias;
    void *y;
    int32_t *part;
    int m, n, k;
    long lda, ldw, ldy;
    int split;
};
struct QuantPlan {
    int kind, split;
    size_t bytes;
};
QuantPlan quant_plan(int m, int n, int k);
hipError_t launch_quant_rows(bool bf16, const QuantArgs &a, hipStream_t s);
hipError_t launch_quant_matmul(bool f32_out, const QuantPlan &p, QuantMatmulArgs &a, hipStream_t s);

}  // namespace bdgdn
