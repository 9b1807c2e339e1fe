// layer_api.hip -- the C ABI of what a hybrid layer does around its mixers: validation and
// dispatch of rotary positions, norms with gate and residual, logits, products of 8-bit integers.
#include <math.h>

#include "bdgdn.h"
#include "layer.hpp"

using namespace bdgdn;

namespace {

constexpr int64_t kFarthest = 1ll << 44;   // elements: strides and their products with sizes stay in 64 bits

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Arrays of 32-bit numbers (NULL is aligned).
template <typename... P> bool words(const P *...p) { return (aligned(p, 4) && ...); }

int size_of(int dtype) { return dtype == BDGDN_BF16 ? 2 : 4; }

bool type_ok(int dtype) { return dtype == BDGDN_BF16 || dtype == BDGDN_F32; }

int status_of(hipError_t e) { return e == hipSuccess ? BDGDN_OK : BDGDN_ERR_LAUNCH; }

bool stride_ok(int64_t s) { return s >= 0 && s <= kFarthest; }

// Rows of `inner` elements, n dimensions of them, share no memory (dimensions that are not nested in
// each other are not looked into and count as sharing).
bool disjoint(int64_t inner, int n, const int64_t *size, const int64_t *stride)
{
    for (int i = 0; i < n; ++i)
        if (size[i] == 0) return true;
    bool done[3] = {};
    double span = (double)inner;
    for (int turn = 0; turn < n; ++turn) {
        int next = -1;
        for (int i = 0; i < n; ++i)
            if (!done[i] && (next < 0 || stride[i] < stride[next] || (stride[i] == stride[next] && size[i] < size[next]))) next = i;
        done[next] = true;
        if (size[next] <= 1) continue;
        if ((double)stride[next] < span) return false;
        span += (double)stride[next] * (double)(size[next] - 1);
    }
    return true;
}

// ------------------------------------------------------------------ rotary positions
int check_rope(const bdgdn_rope_desc_t *d)
{
    if (!d) return BDGDN_ERR_INVALID_ARG;
    if (d->num_req < 0 || d->nodes < 0 || d->h_q <= 0 || d->h_k < 0 || d->d <= 0 || d->rot <= 0) return BDGDN_ERR_INVALID_ARG;
    if (d->rot % 2 || d->rot > d->d || !isfinite(d->scale)) return BDGDN_ERR_INVALID_ARG;
    if (d->layout != BDGDN_ROPE_HALF && d->layout != BDGDN_ROPE_PAIRS) return BDGDN_ERR_INVALID_ARG;
    if (d->inverse != 0 && d->inverse != 1) return BDGDN_ERR_INVALID_ARG;
    if (!type_ok(d->dtype) || d->d > 4096 || d->h_q > 65536 || d->h_k > 65536) return BDGDN_ERR_UNSUPPORTED;
    if ((long)d->num_req * d->nodes > 0x7fffffffL) return BDGDN_ERR_UNSUPPORTED;
    const bdgdn_heads_t *s[4] = {&d->q, &d->q_out, &d->k, &d->k_out};
    for (int i = 0; i < (d->h_k ? 4 : 2); ++i) {
        if (!stride_ok(s[i]->req) || !stride_ok(s[i]->row) || !stride_ok(s[i]->head)) return BDGDN_ERR_INVALID_ARG;
        const int64_t size[3] = {d->num_req, d->nodes, i < 2 ? d->h_q : d->h_k}, stride[3] = {s[i]->req, s[i]->row, s[i]->head};
        if (i % 2 && !disjoint(d->d, 3, size, stride)) return BDGDN_ERR_INVALID_ARG;
    }
    return BDGDN_OK;
}

// Two descriptions of one tensor (strides of single rows say nothing).
bool same(const bdgdn_rope_desc_t *d, int heads, const bdgdn_heads_t &a, const bdgdn_heads_t &b)
{
    return (d->num_req <= 1 || a.req == b.req) && (d->nodes <= 1 || a.row == b.row) && (heads <= 1 || a.head == b.head);
}

// ------------------------------------------------------------------ norms
int check_rows(const bdgdn_norm_desc_t *d, const bdgdn_rows_t &s, bool out)
{
    if (!stride_ok(s.outer) || !stride_ok(s.inner)) return BDGDN_ERR_INVALID_ARG;
    const int64_t size[2] = {d->outer, d->inner}, stride[2] = {s.outer, s.inner};
    return !out || disjoint(d->d, 2, size, stride) ? BDGDN_OK : BDGDN_ERR_INVALID_ARG;
}

int check_norm(const bdgdn_norm_desc_t *d)
{
    if (!d) return BDGDN_ERR_INVALID_ARG;
    if (d->outer < 0 || d->inner < 0 || d->d <= 0) return BDGDN_ERR_INVALID_ARG;
    if ((d->post != 0 && d->post != 1) || (d->pre != 0 && d->pre != 1)) return BDGDN_ERR_INVALID_ARG;
    if (d->act != BDGDN_ACT_NONE && d->act != BDGDN_ACT_SILU && d->act != BDGDN_ACT_SIGMOID) return BDGDN_ERR_INVALID_ARG;
    if (!isfinite(d->scale) || !isfinite(d->eps) || d->eps < 0.f) return BDGDN_ERR_INVALID_ARG;
    if (!type_ok(d->x_dtype) || !type_ok(d->r_dtype) || !type_ok(d->dtype)) return BDGDN_ERR_UNSUPPORTED;
    if (d->dtype == BDGDN_F32 && (d->x_dtype != BDGDN_F32 || d->r_dtype != BDGDN_F32)) return BDGDN_ERR_UNSUPPORTED;
    if (d->d > 16384 || (long)d->outer * d->inner > 0x7fffffffL) return BDGDN_ERR_UNSUPPORTED;
    return BDGDN_OK;
}

struct NormTensor {
    const void *p;
    const bdgdn_rows_t *s;
    RowStride *to;
    int dtype;
    bool out;
};

// Checks the tensors that are there.
int check_tensors(const bdgdn_norm_desc_t *d, const NormTensor *t, int n, const float *const *weights, int n_weights)
{
    for (int i = 0; i < n; ++i) {
        if (!t[i].p) continue;
        const int st = check_rows(d, *t[i].s, t[i].out);
        if (st != BDGDN_OK) return st;
        if (!aligned(t[i].p, size_of(t[i].dtype))) return BDGDN_ERR_INVALID_ARG;
        t[i].to->outer = t[i].s->outer;
        t[i].to->inner = t[i].s->inner;
    }
    for (int i = 0; i < n_weights; ++i)
        if (!aligned(weights[i], 4)) return BDGDN_ERR_INVALID_ARG;
    return BDGDN_OK;
}

bool same_rows(const bdgdn_norm_desc_t *d, const bdgdn_rows_t &a, const bdgdn_rows_t &b)
{
    return (d->outer <= 1 || a.outer == b.outer) && (d->inner <= 1 || a.inner == b.inner);
}

NormArgs norm_args(const bdgdn_norm_desc_t *d, const float *w_post, const float *w_pre, const float *layer_scale)
{
    NormArgs a = {};
    a.w_post = d->post ? w_post : nullptr;
    a.w_pre = d->pre ? w_pre : nullptr;
    a.ls = layer_scale;
    a.rows = d->outer * d->inner;
    a.inner = d->inner;
    a.d = d->d;
    a.post = d->post;
    a.pre = d->pre;
    a.act = d->act;
    a.scale = d->scale;
    a.eps = d->eps;
    a.inv_d = 1.f / (float)d->d;
    return a;
}

size_t norm_workspace(const bdgdn_norm_desc_t *d)
{
    return ((size_t)norm_bwd_groups(d->outer * d->inner, d->d) * 3 * d->d * 4 + 255) & ~(size_t)255;
}

// ------------------------------------------------------------------ logits
int check_logits(const bdgdn_logits_desc_t *d)
{
    if (!d) return BDGDN_ERR_INVALID_ARG;
    if (d->num_req < 0 || d->nodes <= 0 || d->vocab <= 0 || d->n_bias < 0 || d->n_slots < 0) return BDGDN_ERR_INVALID_ARG;
    if (!type_ok(d->dtype) || !type_ok(d->out_dtype) || (d->dtype == BDGDN_F32 && d->out_dtype == BDGDN_BF16))
        return BDGDN_ERR_UNSUPPORTED;
    if (d->nodes > 64 || d->num_req > 65535 || d->vocab > 0x40000000 || d->n_bias > 0x40000000) return BDGDN_ERR_UNSUPPORTED;
    if (!stride_ok(d->req_stride) || !stride_ok(d->row_stride) || !stride_ok(d->out_req_stride) ||
        !stride_ok(d->out_row_stride) || !stride_ok(d->history_stride) || !stride_ok(d->allow_req_stride) ||
        !stride_ok(d->allow_row_stride))
        return BDGDN_ERR_INVALID_ARG;
    const int64_t size[2] = {d->num_req, d->nodes}, stride[2] = {d->out_req_stride, d->out_row_stride};
    if (!disjoint(d->vocab, 2, size, stride)) return BDGDN_ERR_INVALID_ARG;
    return BDGDN_OK;
}

// ------------------------------------------------------------------ 8-bit products
int check_quant(const bdgdn_quant_desc_t *d)
{
    if (!d) return BDGDN_ERR_INVALID_ARG;
    if (d->rows < 0 || d->cols <= 0 || d->width <= 0 || !stride_ok(d->x_stride) || !stride_ok(d->q_stride)) return BDGDN_ERR_INVALID_ARG;
    if (d->cols > 0x40000000 || d->rows >= (1 << 24)) return BDGDN_ERR_UNSUPPORTED;   // (a launch has 2^32 threads)
    if (d->width != (d->cols + 127) / 128 * 128 || d->q_stride % 16 || (d->rows > 1 && d->q_stride < d->width)) return BDGDN_ERR_INVALID_ARG;
    return type_ok(d->dtype) ? BDGDN_OK : BDGDN_ERR_UNSUPPORTED;
}

int check_quant_matmul(const bdgdn_quant_matmul_desc_t *d)
{
    if (!d) return BDGDN_ERR_INVALID_ARG;
    if (d->m < 0 || d->n <= 0 || d->k <= 0 || d->k % 128) return BDGDN_ERR_INVALID_ARG;
    if (!stride_ok(d->a_stride) || !stride_ok(d->w_stride) || !stride_ok(d->out_stride)) return BDGDN_ERR_INVALID_ARG;
    if (d->a_stride % 16 || d->w_stride % 16 || (d->m > 1 && d->out_stride < d->n)) return BDGDN_ERR_INVALID_ARG;
    // 32-bit sums of products of up to 2^14, and workgroups of 512 threads, of which a launch has 2^32
    if (!type_ok(d->out_dtype) || d->k > 130944 || d->n > (1 << 26) || d->m > (1 << 30)) return BDGDN_ERR_UNSUPPORTED;
    if (((long)d->m + 127) / 128 * (((long)d->n + 127) / 128) > (1 << 22)) return BDGDN_ERR_UNSUPPORTED;
    return BDGDN_OK;
}

}  // namespace

extern "C" {

int bdgdn_rope_freqs(const bdgdn_rope_freq_t *f, uint64_t *turns_host)
{
    if (!f || !turns_host || f->rot <= 0 || f->rot % 2) return BDGDN_ERR_INVALID_ARG;
    if (!(f->base >= 1) || !isfinite(f->base) || !(f->factor > 0) || !isfinite(f->factor)) return BDGDN_ERR_INVALID_ARG;
    if (f->scaling < BDGDN_ROPE_PLAIN || f->scaling > BDGDN_ROPE_PARTS) return BDGDN_ERR_INVALID_ARG;
    if (f->scaling == BDGDN_ROPE_PARTS &&
        (!(f->original > 0) || !isfinite(f->original) || !(f->slow >= 0) || !(f->fast > f->slow) || !isfinite(f->fast)))
        return BDGDN_ERR_INVALID_ARG;
    if (f->scaling == BDGDN_ROPE_NTK && f->rot == 2) return BDGDN_ERR_INVALID_ARG;
    const long double two_pi = 6.283185307179586476925286766559L;
    long double base = f->base;
    if (f->scaling == BDGDN_ROPE_NTK) base *= powl(f->factor, (long double)f->rot / (f->rot - 2));
    for (int i = 0; i < f->rot / 2; ++i) {
        long double w = powl(base, -2.0L * i / f->rot);
        if (f->scaling == BDGDN_ROPE_LINEAR) w /= f->factor;
        if (f->scaling == BDGDN_ROPE_PARTS) {
            long double keep = (f->original * w / two_pi - f->slow) / ((long double)f->fast - f->slow);
            keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
            w = w * keep + w / f->factor * (1 - keep);
        }
        const long double part = fmodl(w / two_pi, 1.0L) * 18446744073709551616.0L;
        turns_host[i] = part < 18446744073709551615.0L ? (uint64_t)(part + 0.5L) : 0;   // (all but a whole turn: none)
    }
    return BDGDN_OK;
}

int bdgdn_rope(const bdgdn_rope_desc_t *desc, const void *q, const void *k, const uint64_t *turns,
               const int32_t *pos, const int32_t *seq_len, const int32_t *slot, const int32_t *count,
               void *q_out, void *k_out, void *stream)
{
    const int st = check_rope(desc);
    if (st != BDGDN_OK) return st;
    if (desc->num_req == 0 || desc->nodes == 0) return BDGDN_OK;
    const bool with_k = desc->h_k > 0;
    if (!q || !q_out || !turns || with_k != (k != nullptr) || with_k != (k_out != nullptr)) return BDGDN_ERR_INVALID_ARG;
    if (seq_len && (desc->n_slots <= 0 || (!slot && desc->num_req > desc->n_slots))) return BDGDN_ERR_INVALID_ARG;
    const size_t size = size_of(desc->dtype);
    if (!aligned(q, size) || !aligned(k, size) || !aligned(q_out, size) || !aligned(k_out, size) || !aligned(turns, 8) ||
        !words(pos, seq_len, slot, count))
        return BDGDN_ERR_INVALID_ARG;
    if ((q == q_out && !same(desc, desc->h_q, desc->q, desc->q_out)) || (with_k && k == k_out && !same(desc, desc->h_k, desc->k, desc->k_out)))
        return BDGDN_ERR_INVALID_ARG;
    RopeArgs a = {};
    a.x[0] = static_cast<const unsigned char *>(q);
    a.x[1] = static_cast<const unsigned char *>(k);
    a.y[0] = static_cast<unsigned char *>(q_out);
    a.y[1] = static_cast<unsigned char *>(k_out);
    const bdgdn_heads_t *s[2][2] = {{&desc->q, &desc->q_out}, {&desc->k, &desc->k_out}};
    for (int w = 0; w <= (with_k ? 1 : 0); ++w) {
        for (int o = 0; o < 2; ++o) {
            const int64_t stride[3] = {s[w][o]->req, s[w][o]->row, s[w][o]->head};
            for (int i = 0; i < 3; ++i) (o ? a.ys : a.xs)[w][i] = stride[i] * (long)size;
        }
    }
    a.turns = turns; a.pos = pos; a.len = seq_len; a.slot = slot; a.count = count;
    a.R = desc->num_req; a.N = desc->nodes; a.h_q = desc->h_q; a.h = desc->h_q + desc->h_k;
    a.d = desc->d; a.rot = desc->rot; a.n_slots = desc->n_slots;
    a.in_place = q == q_out && (!with_k || k == k_out);
    a.scale = desc->scale;
    a.sine = desc->inverse ? -desc->scale : desc->scale;
    return status_of(launch_rope(desc->dtype == BDGDN_BF16, desc->layout == BDGDN_ROPE_PAIRS, a, static_cast<hipStream_t>(stream)));
}

int bdgdn_norm_fwd(const bdgdn_norm_desc_t *desc, const void *x, const void *z, const void *r,
                   const float *w_post, const float *w_pre, const float *layer_scale, void *r_out,
                   void *y, void *stream)
{
    int st = check_norm(desc);
    if (st != BDGDN_OK) return st;
    if (desc->outer == 0 || desc->inner == 0) return BDGDN_OK;
    if (!x || (!r_out && !y)) return BDGDN_ERR_INVALID_ARG;
    if (r && r == r_out && !same_rows(desc, desc->r, desc->r_out)) return BDGDN_ERR_INVALID_ARG;
    NormArgs a = norm_args(desc, w_post, w_pre, layer_scale);
    const NormTensor t[5] = {{x, &desc->x, &a.sx, desc->x_dtype, false}, {z, &desc->z, &a.sz, desc->dtype, false},
                             {r, &desc->r, &a.sr, desc->r_dtype, false}, {r_out, &desc->r_out, &a.sro, desc->r_dtype, true},
                             {y, &desc->y, &a.sy, desc->dtype, true}};
    const float *weights[3] = {a.w_post, a.w_pre, a.ls};
    st = check_tensors(desc, t, 5, weights, 3);
    if (st != BDGDN_OK) return st;
    a.x = x; a.z = z; a.r = r; a.r_out = r_out; a.y = y;
    return status_of(launch_norm_fwd(desc->x_dtype == BDGDN_F32, desc->r_dtype == BDGDN_F32, desc->dtype == BDGDN_F32, a,
                                     static_cast<hipStream_t>(stream)));
}

size_t bdgdn_norm_bwd_workspace(const bdgdn_norm_desc_t *desc)
{
    if (check_norm(desc) != BDGDN_OK || desc->outer == 0 || desc->inner == 0) return 0;
    return norm_workspace(desc);
}

int bdgdn_norm_bwd(const bdgdn_norm_desc_t *desc, const void *x, const void *z, const void *r_out,
                   const float *w_post, const float *w_pre, const float *layer_scale, const void *dy,
                   const void *dr_out, void *dx, void *dz, void *dr, float *dw_post, float *dw_pre,
                   float *dlayer_scale, void *workspace, size_t workspace_bytes, void *stream)
{
    int st = check_norm(desc);
    if (st != BDGDN_OK) return st;
    const bool any = desc->outer > 0 && desc->inner > 0, sums = dw_post || dw_pre || dlayer_scale;
    if ((dw_post && !desc->post) || (dw_pre && !desc->pre)) return BDGDN_ERR_INVALID_ARG;
    if (!aligned(dw_post, 4) || !aligned(dw_pre, 4) || !aligned(dlayer_scale, 4)) return BDGDN_ERR_INVALID_ARG;
    if (any && (!x || (!dy && !dr_out) || (dz && !z) || (!dx && !dz && !dr && !sums))) return BDGDN_ERR_INVALID_ARG;
    if (any && dr && dr == dr_out && !same_rows(desc, desc->dr, desc->dr_out)) return BDGDN_ERR_INVALID_ARG;
    NormArgs a = norm_args(desc, w_post, w_pre, layer_scale);
    if (any) {
        const NormTensor t[8] = {{x, &desc->x, &a.sx, desc->x_dtype, false}, {z, &desc->z, &a.sz, desc->dtype, false},
                                 {r_out, &desc->r_out, &a.sro, desc->r_dtype, false}, {dy, &desc->dy, &a.sdy, desc->dtype, false},
                                 {dr_out, &desc->dr_out, &a.sdro, desc->r_dtype, false}, {dx, &desc->dx, &a.sdx, desc->x_dtype, true},
                                 {dz, &desc->dz, &a.sdz, desc->dtype, true}, {dr, &desc->dr, &a.sdr, desc->r_dtype, true}};
        const float *weights[3] = {a.w_post, a.w_pre, a.ls};
        st = check_tensors(desc, t, 8, weights, 3);
        if (st != BDGDN_OK) return st;
        if (sums) {
            if (!aligned(workspace, 256)) return BDGDN_ERR_INVALID_ARG;
            if (!workspace || workspace_bytes < norm_workspace(desc)) return BDGDN_ERR_WORKSPACE;
        }
        a.groups = norm_bwd_groups(a.rows, a.d);
    } else if (!sums) {
        return BDGDN_OK;
    }
    a.x = x; a.z = z; a.dy = dy; a.dr_out = dr_out;
    a.r = desc->pre ? r_out : nullptr;   // (nothing else asks for it)
    a.dx = dx; a.dz = dz; a.dr = dr;
    a.dw[0] = dw_post; a.dw[1] = dw_pre; a.dw[2] = dlayer_scale;
    a.part = static_cast<float *>(workspace);
    return status_of(launch_norm_bwd(desc->x_dtype == BDGDN_F32, desc->r_dtype == BDGDN_F32, desc->dtype == BDGDN_F32, a,
                                     static_cast<hipStream_t>(stream)));
}

int bdgdn_logits(const bdgdn_logits_desc_t *desc, const void *logits, const int32_t *history,
                 const int32_t *slot, const int32_t *token, const uint64_t *mask, const int32_t *count,
                 const float *repetition, const float *presence, const float *frequency,
                 const int32_t *bias_token, const float *bias, const uint32_t *allow, void *out, void *stream)
{
    const int st = check_logits(desc);
    if (st != BDGDN_OK) return st;
    if (desc->num_req == 0) return BDGDN_OK;
    if (!logits || !out || (mask && !token)) return BDGDN_ERR_INVALID_ARG;
    if ((desc->n_bias > 0) != (bias_token != nullptr) || (desc->n_bias > 0) != (bias != nullptr)) return BDGDN_ERR_INVALID_ARG;
    if (history && (desc->n_slots <= 0 || (!slot && desc->num_req > desc->n_slots))) return BDGDN_ERR_INVALID_ARG;
    if (history && desc->n_slots > 1 && desc->history_stride < desc->vocab) return BDGDN_ERR_INVALID_ARG;
    if (!aligned(logits, size_of(desc->dtype)) || !aligned(out, size_of(desc->out_dtype)) || !aligned(mask, 8) ||
        !words(history, allow, slot, token, count, repetition, presence, frequency, bias_token, bias))
        return BDGDN_ERR_INVALID_ARG;
    if (logits == out && (desc->dtype != desc->out_dtype || (desc->num_req > 1 && desc->req_stride != desc->out_req_stride) ||
                          (desc->nodes > 1 && desc->row_stride != desc->out_row_stride)))
        return BDGDN_ERR_INVALID_ARG;
    LogitsArgs a = {};
    a.x = logits; a.y = out;
    a.history = history; a.slot = slot; a.token = token; a.mask = mask; a.count = count;
    a.repetition = repetition; a.presence = presence; a.frequency = frequency;
    a.bias_token = bias_token; a.bias = bias; a.allow = allow;
    a.R = desc->num_req; a.N = desc->nodes; a.V = desc->vocab; a.n_slots = desc->n_slots; a.n_bias = desc->n_bias;
    a.x_req = desc->req_stride; a.x_row = desc->row_stride;
    a.y_req = desc->out_req_stride; a.y_row = desc->out_row_stride;
    a.h_row = desc->history_stride; a.a_req = desc->allow_req_stride; a.a_row = desc->allow_row_stride;
    return status_of(launch_logits(desc->dtype == BDGDN_BF16, desc->out_dtype == BDGDN_F32, a, static_cast<hipStream_t>(stream)));
}

int bdgdn_history_add(int32_t num_req, int32_t nodes, int32_t vocab, int32_t n_slots, int64_t history_stride,
                      int32_t *history, const int32_t *slot, const int32_t *token, const int32_t *path,
                      const int32_t *count, int32_t prompt, void *stream)
{
    if (num_req < 0 || nodes < 0 || vocab <= 0 || n_slots <= 0 || !stride_ok(history_stride)) return BDGDN_ERR_INVALID_ARG;
    if ((n_slots > 1 && history_stride < vocab) || (prompt != 0 && prompt != 1)) return BDGDN_ERR_INVALID_ARG;
    if (num_req == 0 || nodes == 0) return BDGDN_OK;
    if (!history || !token || !words(history, slot, token, path, count) || (!slot && num_req > n_slots)) return BDGDN_ERR_INVALID_ARG;
    return status_of(launch_history_add(num_req, nodes, vocab, n_slots, history_stride, history, slot, token, path, count,
                                        prompt, static_cast<hipStream_t>(stream)));
}

int bdgdn_quant_rows(const bdgdn_quant_desc_t *desc, const void *x, int8_t *q, float *scale, void *stream)
{
    const int st = check_quant(desc);
    if (st != BDGDN_OK) return st;
    if (desc->rows == 0) return BDGDN_OK;
    if (!x || !q || !scale || !aligned(x, size_of(desc->dtype)) || !aligned(q, 16) || !aligned(scale, 4)) return BDGDN_ERR_INVALID_ARG;
    QuantArgs a = {x, q, scale, desc->rows, desc->cols, desc->width, desc->x_stride, desc->q_stride};
    return status_of(launch_quant_rows(desc->dtype == BDGDN_BF16, a, static_cast<hipStream_t>(stream)));
}

size_t bdgdn_quant_matmul_workspace(const bdgdn_quant_matmul_desc_t *desc)
{
    if (check_quant_matmul(desc) != BDGDN_OK || desc->m == 0) return 0;
    return quant_plan(desc->m, desc->n, desc->k).bytes;
}

int bdgdn_quant_matmul(const bdgdn_quant_matmul_desc_t *desc, const int8_t *a, const float *a_scale,
                       const int8_t *w, const float *w_scale, const float *bias, void *out, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    const int st = check_quant_matmul(desc);
    if (st != BDGDN_OK) return st;
    if (desc->m == 0) return BDGDN_OK;
    if (!a || !a_scale || !w || !w_scale || !out) return BDGDN_ERR_INVALID_ARG;
    if (!aligned(a, 16) || !aligned(w, 16) || !aligned(a_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) ||
        !aligned(out, size_of(desc->out_dtype)) || !aligned(workspace, 256))
        return BDGDN_ERR_INVALID_ARG;
    const QuantPlan p = quant_plan(desc->m, desc->n, desc->k);
    if (p.bytes > 0 && (!workspace || workspace_bytes < p.bytes)) return BDGDN_ERR_WORKSPACE;
    QuantMatmulArgs g = {a, w, a_scale, w_scale, bias, out, static_cast<int32_t *>(workspace), desc->m, desc->n, desc->k,
                         desc->a_stride, desc->w_stride, desc->out_stride, p.split};
    return status_of(launch_quant_matmul(desc->out_dtype == BDGDN_F32, p, g, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
