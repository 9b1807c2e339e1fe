/*
 * bdgdn.h -- C ABI of the block-diffusion Gated DeltaNet library (libbdgdn.so) for
 * AMD MI355X (gfx950).
 *
 * The library computes the Gated Delta Rule (GDR) layer of FLARE's hybrid backbone
 * (arXiv 2606.01774) under the block-diffusion clean/noisy schedule:
 *
 *   clean stream (Sec. 3.1, eq. gdn-recurrence; Appendix eq. per-step-fwd):
 *     S_t = exp(g_t) (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T,
 *     o_t = scale * S_t^T q_t                                (S is d_k x d_v)
 *   noisy stream (Sec. 3.2, eq. flare-gdn-schedule; Appendix eq. noisy-block-fwd):
 *     block b of L positions is seeded with the clean state after the last clean
 *     position before the block, applies its own L noisy updates, and every
 *     position of the block reads the block-end noisy state:
 *     on_l = scale * Sn_end^T qn_l.
 *   document packing (Appendix "Document-packed training"): documents start on
 *     block boundaries, each starts from a zero state, the last block of a document
 *     may be partial (treated as padded with identity positions).
 *   serving (Appendix "Diffusion-Trust Sampling", "Differences between the denoise
 *     pass and the state-update pass"): a denoise pass reads the cached state and
 *     never writes it; a commit pass runs the token-causal update and writes it back.
 *
 * Conventions shared by every entry point
 *   - Pointers named *_dev / tensors are device pointers (HIP device memory); the
 *     only host pointers are the descriptors and cu_seqlens_host.
 *   - Token tensors are token-major and contiguous:
 *       q, k : [rows][h_qk][d_k]      v, o : [rows][h_v][d_v]     g, beta : [rows][h_v]
 *     where rows = batch*seqlen (training) or num_req*block (serving).
 *     q, k, v have the descriptor's dtype and o its out_dtype; g (the LOG gate,
 *     alpha = exp(g)) and beta are fp32 and used as given.  g must be <= 0 (alpha in
 *     (0, 1], a decay): the bf16 kernels evaluate every decay exponent as non-positive,
 *     and a positive g gives unspecified (finite) results there.
 *   - Arithmetic: states and all accumulations are fp32.  With bf16 inputs the MFMA
 *     operands are fp16 (the bf16 values converted exactly; every rounded
 *     intermediate keeps 11 significant bits), so inputs and intermediates must stay
 *     within fp16 range: |q|, |k|, |v| and state entries below 2^15 (q and k are
 *     normally L2-normalised); magnitudes below 2^-14 lose relative precision
 *     (absolute error under 2^-25).  With fp32 inputs everything is fp32.
 *   - v-head h reads q/k head h / (h_v / h_qk) (consecutive grouping).
 *   - States are fp32 [unit][h_v][d_k][d_v], row-major (paper orientation).
 *   - All work is enqueued on `stream` (a hipStream_t; NULL = default stream); no
 *     call synchronises the host or allocates device memory.  Outputs are valid
 *     once the stream reaches that point.
 *   - Every argument is validated on the host before anything is launched.  On
 *     any error return nothing is launched and no output is touched.
 *   - q, k, v and the dtype outputs must be 16-byte aligned (BDGDN_ERR_INVALID_ARG).
 *   - The caller owns every buffer.  Outputs must not alias inputs.
 *   - Calls are thread-safe; the library keeps no mutable global state besides a
 *     once-initialised table of kernel attributes.
 *
 * Supported: d_k, d_v in {64, 128}; 1 <= block <= 64; (dtype, out_dtype) in
 * {(bf16, fp32), (bf16, bf16), (fp32, fp32)}, fp32 inputs with block <= 32.
 * Anything else returns BDGDN_ERR_UNSUPPORTED.  fp32 outputs for bf16 inputs are the
 * accuracy-grade choice: rounding an output to bf16 alone perturbs it by up to
 * 2^-9 of its magnitude.
 */
#ifndef BDGDN_H
#define BDGDN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BDGDN_OK               0
#define BDGDN_ERR_INVALID_ARG -1 /* NULL required pointer, non-positive size, h_v % h_qk != 0,
                                    non-finite scale, inconsistent cu_seqlens */
#define BDGDN_ERR_UNSUPPORTED -2 /* (dtype, d_k, d_v, block) outside the supported set */
#define BDGDN_ERR_UNALIGNED   -3 /* a document start cu_seqlens[i] (i < N) is not a multiple
                                    of block (Appendix "Document-packed training") */
#define BDGDN_ERR_WORKSPACE   -4 /* workspace smaller than bdgdn_fwd_train_workspace() */
#define BDGDN_ERR_LAUNCH      -5 /* the HIP runtime reported an error for a launch */
#define BDGDN_ERR_SCRATCH     -6 /* the input needs more than the fixed scratch of a
                                    no-allocation entry point (nothing is launched) */

typedef enum { BDGDN_BF16 = 0, BDGDN_F32 = 1 } bdgdn_dtype_t;

/* How the training forward is scheduled; every route gives the same result up to
 * floating-point summation order.
 *  FUSED:   the fused two-stream schedule (Appendix "Route II"): one workgroup per
 *           (sequence, v-head, d_v tile) scans the blocks in order with the clean state
 *           on chip and evaluates each noisy block from the in-register boundary state.
 *           With bf16 inputs and blocks of at most 32 positions this is one kernel whose
 *           workgroups also compute each block's UT transform and masked Q K^T a block
 *           ahead (no workspace); when (sequences or documents) x v-heads reach the
 *           GPU's 256 compute units and d_k = d_v, one workgroup per (sequence, v-head)
 *           covers all d_v columns instead (CHUNKED's output pass with one segment per
 *           chain; no workspace).  Blocks of an even 34 .. 64 positions run the one
 *           kernel on sub-blocks of half the block, each noisy block carrying its state
 *           across its two halves (no workspace).  Blocks of 1, 2, 4 or 8 positions run
 *           it on 32-position clean chunks that hold 32 / block noisy blocks each, every
 *           noisy block seeded on chip with the clean state at its own start (no
 *           workspace).  Otherwise it is the RECORDS schedule.
 *  SPLIT:   boundary states through HBM and a separate noisy-block kernel (Appendix
 *           "Route I"): the clean scan writes the clean state before every block (the
 *           seed of that noisy block) into the workspace, fp32 [block][h_v][d_k][d_v]
 *           (blocks of all sequences, or of the packed axis, in order), then every
 *           noisy block is evaluated in parallel from its seed.  The clean outputs and
 *           ht equal FUSED's bit for bit.  bf16 inputs, d_k = d_v = 128 and blocks of at
 *           most 32 positions only (else BDGDN_ERR_UNSUPPORTED).
 *  ONEPASS: one kernel per (sequence, v-head, d_v tile) that recomputes the UT
 *           transform of each block itself, without overlap.  No workspace.
 *  RECORDS: two kernels: the UT transform and masked Q K^T of every (block, v-head)
 *           in parallel into the workspace, then the scan of FUSED reading them.
 *           Needs a workspace (bdgdn_fwd_train_workspace).
 *  CHUNKED: the chunk-parallel schedule (Appendix "Route II" with the chunk-state pass
 *           of eq. chunk-state): every (sequence or document, v-head) chain is cut into
 *           segments of G blocks, G a power of two >= 16 chosen from the descriptor so
 *           that the (chain, segment) pairs cover the GPU's compute units; a state pass
 *           computes the clean state at every later segment start (with the blocks'
 *           clean UT transforms computed in parallel before it), then one workgroup per
 *           (chain, segment) evaluates the segment's blocks for all d_v columns at once.
 *           Needs a workspace (bdgdn_fwd_train_workspace): a clean UT record per
 *           (block, v-head) and an fp32 state per (later segment start, v-head).  bf16
 *           inputs, d_k = d_v in {64, 128}, blocks of at most 32 positions, at most 512
 *           packed documents (else BDGDN_ERR_UNSUPPORTED). */
typedef enum {
    BDGDN_ROUTE_FUSED = 0,
    BDGDN_ROUTE_SPLIT = 1,
    BDGDN_ROUTE_ONEPASS = 2,
    BDGDN_ROUTE_RECORDS = 3,
    BDGDN_ROUTE_CHUNKED = 4
} bdgdn_route_t;

typedef struct {
    int32_t batch;     /* B sequences; must be 1 when packed (num_seqs > 0)            */
    int32_t seqlen;    /* T tokens per sequence, or total packed tokens                 */
    int32_t num_seqs;  /* N packed documents, 0 when not packed                         */
    int32_t h_qk, h_v; /* q/k heads and v heads; h_v % h_qk == 0                        */
    int32_t d_k, d_v;  /* head dimensions                                               */
    int32_t block;     /* diffusion block size L                                        */
    float scale;       /* output scale s (the paper uses 1/sqrt(d_k))                   */
    int32_t dtype;     /* bdgdn_dtype_t of q, k, v                                      */
    int32_t route;     /* bdgdn_route_t                                                 */
    int32_t out_dtype; /* bdgdn_dtype_t of o, on                                        */
} bdgdn_fwd_desc_t;

typedef struct {
    int32_t num_req;   /* R requests, one block of `block` tokens each                  */
    int32_t h_qk, h_v, d_k, d_v;
    int32_t block;     /* L                                                             */
    float scale;
    int32_t dtype;     /* bdgdn_dtype_t of q, k, v                                      */
    int32_t out_dtype; /* bdgdn_dtype_t of o / o_causal                                 */
} bdgdn_serve_desc_t;

/* Library version, (major << 16) | minor. */
int32_t bdgdn_version(void);

/* Human-readable text of a status code (static storage). */
const char *bdgdn_status_string(int status);

/* Bytes of device workspace bdgdn_fwd_train needs for this descriptor (0 when the
 * route runs without one), or 0 for a descriptor that bdgdn_fwd_train would reject. */
size_t bdgdn_fwd_train_workspace(const bdgdn_fwd_desc_t *desc);

/*
 * Two-stream training forward (clean + noisy), Sec. 3.2 and Appendix "Gated Delta
 * Rule: two-stream training".
 *
 *   q, k, v, g, beta       clean stream   ([B*T] rows, layouts above)
 *   qn, kn, vn, gn, betan  noisy stream   (same shapes; gn/betan are the noisy
 *                                          stream's own gates)
 *   cu_seqlens_dev/_host   both NULL (B sequences of T tokens) or both [N+1] int32
 *                          offsets into the packed axis (B == 1, cu[0] == 0,
 *                          cu[N] == T, non-decreasing, cu[i] % block == 0 for i < N).
 *                          The two copies must hold the same values.
 *   h0                     [B or N][h_v][d_k][d_v] fp32 initial clean state, or NULL
 *                          for zero.  Each sequence's first noisy block is seeded
 *                          with the same state.
 *   o, on                  [B*T][h_v][d_v] outputs of out_dtype (clean causal readout,
 *                          noisy block-end readout); every row is written.
 *   ht                     [B or N][h_v][d_k][d_v] fp32 final clean state, or NULL.
 *   workspace              device memory of at least bdgdn_fwd_train_workspace(desc)
 *                          bytes, 256-byte aligned (may be NULL when that is 0); its
 *                          contents are scratch owned by the call until the stream
 *                          passes it.
 * Returns BDGDN_OK or a negative status.
 */
int bdgdn_fwd_train(const bdgdn_fwd_desc_t *desc,
                    const void *q, const void *k, const void *v,
                    const float *g, const float *beta,
                    const void *qn, const void *kn, const void *vn,
                    const float *gn, const float *betan,
                    const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host,
                    const float *h0, void *o, void *on, float *ht,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * Complementary-view training forward (Sec. 3.3 "Training Objective and Mask Design": each
 * block is trained under two complementary noisy views, both conditioned on the same clean
 * context): one clean scan, whose boundary states seed every block of every noisy view.
 * Each view is a noisy stream of its own (inputs, gates, block-end readout); view i's output
 * equals the `on` of bdgdn_fwd_train with the same clean stream and view i as the noisy
 * stream.  desc->route picks the schedule:
 *   FUSED  one pass of the one-kernel forward per view, the clean scan recomputed with each
 *          view and every noisy block evaluated from the on-chip boundary state (no
 *          workspace);
 *   SPLIT  one pass of the one-kernel forward over the clean stream and view 0 that also
 *          writes the seed state of every (block, v-head) to the workspace, then the
 *          noisy-block pass from the seeds for every further view (the clean scan runs once;
 *          the seeds make a round trip through device memory).
 * Other routes give BDGDN_ERR_UNSUPPORTED.
 */
typedef struct {
    const void *q, *k, *v;   /* [B*T][h_qk or h_v][d] of desc->dtype, 16-byte aligned */
    const float *g, *beta;   /* [B*T][h_v] fp32: the view's log-gates and step sizes  */
    void *o;                 /* [B*T][h_v][d_v] of desc->out_dtype: its readout       */
} bdgdn_noisy_view_t;

/* Bytes of workspace bdgdn_fwd_train_views needs: the seed states for the SPLIT route, 0
 * for FUSED or for a descriptor it would reject. */
size_t bdgdn_fwd_train_views_workspace(const bdgdn_fwd_desc_t *desc);

/* Clean inputs, h0, o, ht and cu_seqlens as for bdgdn_fwd_train; views[0 .. n_views-1],
 * 1 <= n_views <= 16.  bf16 inputs; FUSED takes the blocks the one-kernel forward takes (at
 * most 32 positions, or an even 34 .. 64), SPLIT needs d_k = d_v = 128 and blocks of at most
 * 32 positions (else BDGDN_ERR_UNSUPPORTED). */
int bdgdn_fwd_train_views(const bdgdn_fwd_desc_t *desc,
                          const void *q, const void *k, const void *v,
                          const float *g, const float *beta,
                          const bdgdn_noisy_view_t *views, int32_t n_views,
                          const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host,
                          const float *h0, void *o, float *ht,
                          void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of device workspace bdgdn_bwd_train needs.  Block-form shapes (bf16 inputs,
 * d_k = d_v = 128, blocks of at most 32 positions), per (block, v-head): the recomputed
 * clean seed state (fp16), the part of the clean state gradient at the block's start that
 * does not depend on the gradient at its end (fp16; overwritten by the gradient at the
 * block's end once the reverse scan has read it), the block's U K (32 x d_k fp16) and
 * gamma_n; plus 2.3 KB for the range pass.  Per-step shapes: two states per (block, v-head)
 * (fp32), at least (and where that is over 2 GiB, only) what the serial schedule needs: the
 * clean state before every eighth block of every chain (fp32) and eight block-start states
 * per (chain, 16-column tile) (fp32).  0 for a descriptor it would reject. */
size_t bdgdn_bwd_train_workspace(const bdgdn_fwd_desc_t *desc);

/* Bytes of device workspace bdgdn_bwd_train (and bdgdn_bwd_train_views) needs when run in
 * `segments` time segments (Appendix "Backward primitives": the strided clean-state
 * checkpoints of the checkpoint build, with the stride chosen as in "Choosing the stride"):
 * every chain's clean blocks (sub-blocks of half the block for blocks of 34 .. 64) are cut
 * into segments of ceil(longest chain's blocks / segments) (even for sub-blocks), the clean
 * state at each segment start after the first is kept (fp32, one per (sequence, v-head)),
 * and the segments run last first, each recomputing its own seeds from its checkpoint, so
 * that the per-block workspace above holds the first segment's blocks only (for every
 * sequence, min(its blocks, the segment length)), plus the checkpoints, one fp32
 * state-gradient carry per (sequence, v-head) and the segment tables.
 *   cu_seqlens_host   [N+1] document offsets when desc->num_seqs > 0, else NULL
 *   segments          >= 1; 1 gives bdgdn_bwd_train_workspace(desc); more than the longest
 *                     chain's blocks count as that many
 * Per-step shapes need no more than bdgdn_bwd_train_workspace(desc) and are never segmented
 * (that value for any segments).  0 for a descriptor it would reject or missing packing. */
size_t bdgdn_bwd_train_workspace_segmented(const bdgdn_fwd_desc_t *desc, const int32_t *cu_seqlens_host,
                                           int segments);

/*
 * Backward of bdgdn_fwd_train (Appendix "Backward primitives": the noisy block-end
 * readout backward, eq. noisy-readout-bwd; the block-level chain rule,
 * eq. dh-block-recursion; the clean chunk backward): the gradients of
 *     sum <do, o> + sum <don, on> + <dht, ht>
 * with respect to every input of the forward, for the same descriptor and inputs
 * (desc->route is not used; desc->out_dtype is the dtype of do and don).
 *
 *   do, don              [B*T][h_v][d_v] upstream gradients of o and on (out_dtype)
 *   dht                  [B or N][h_v][d_k][d_v] fp32 gradient of ht, or NULL for zero
 *   dq, dk, dqn, dkn     [B*T][h_qk][d_k] fp32 (summed over the v-heads of a q/k head)
 *   dv, dvn              [B*T][h_v][d_v] fp32
 *   dg, dbeta, dgn, dbetan  [B*T][h_v] fp32 (gradients of the log-gates and step sizes)
 *   dh0                  [B or N][h_v][d_k][d_v] fp32 gradient of h0, or NULL
 *   workspace            256-byte aligned, owned by the call until the stream passes it;
 *                        at least bdgdn_bwd_train_workspace(desc) bytes runs the blocks of
 *                        every chain at once.  A smaller one runs the block-form shapes in
 *                        the fewest time segments s >= 2 with
 *                        bdgdn_bwd_train_workspace_segmented(desc, cu_seqlens_host, s) <=
 *                        workspace_bytes (the same results bit for bit: the checkpoints
 *                        and the carry are the fp32 values the one-pass call keeps on
 *                        chip; one more clean-scan pass over all but the last segment and
 *                        more, smaller launches); BDGDN_ERR_WORKSPACE if none fits
 * Every gradient row is overwritten.  bf16 inputs with d_k = d_v = 128 and blocks of at
 * most 32 positions, or an even 34 .. 64, run the block-form kernels (blocks of 1, 2, 4, 8 or
 * 16 positions with one noisy view on clean chunks of 32 that hold several, segmented by
 * chunks, where a chain saves seven steps by them or they halve more units than the chip has
 * CUs, and where that fits the workspace, else block by block, which rounds differently);
 * fp32 inputs (blocks of at most 32), d_k or
 * d_v of 64, and odd bf16 blocks of 33 .. 63 positions run the per-step fp32 backward (at
 * most 512 packed documents and four views): all blocks in parallel between two serial walks
 * of the clean state and its gradient, or, with less workspace than two states per (block,
 * v-head) or where these are over 2 GiB, one wave per (chain, 16-column tile) walking the
 * steps backwards from strided clean checkpoints.  Anything else is BDGDN_ERR_UNSUPPORTED.  The block-form kernels and the
 * parallel per-step ones are deterministic, grouped value heads included (dq, dk of a q/k
 * head summed over its v-heads in a fixed order).  The serial per-step walk sums dq, dk, dg
 * and dbeta over its column tiles with floating-point atomics (summation order not fixed).
 * Range: do, don and the state gradients enter the products as fp16 operands.  Every result
 * is linear in do, don and dht, so the call first finds the largest |entry| of do, don (of
 * every view) and dht on the device, multiplies them by the power of two sigma that puts it
 * in [4, 8) as they are converted, and divides every fp32 result by sigma (exact): upstream
 * gradients of any magnitude (a loss averaged over many tokens, or a large one) keep the
 * fp16 operands' relative precision, and scaling the upstream gradients by a power of two
 * scales every result by exactly that factor.  Non-finite upstream gradients give sigma = 1.
 */
int bdgdn_bwd_train(const bdgdn_fwd_desc_t *desc,
                    const void *q, const void *k, const void *v,
                    const float *g, const float *beta,
                    const void *qn, const void *kn, const void *vn,
                    const float *gn, const float *betan,
                    const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host,
                    const float *h0, const void *do_, const void *don, const float *dht,
                    float *dq, float *dk, float *dv, float *dg, float *dbeta,
                    float *dqn, float *dkn, float *dvn, float *dgn, float *dbetan, float *dh0,
                    void *workspace, size_t workspace_bytes, void *stream);

/* One noisy view of the complementary-view backward: its inputs (as bdgdn_noisy_view_t),
 * the upstream gradient of its readout and its gradients (as dqn .. dbetan of
 * bdgdn_bwd_train). */
typedef struct {
    const void *q, *k, *v;   /* [B*T][h_qk or h_v][d] of desc->dtype, 16-byte aligned      */
    const float *g, *beta;   /* [B*T][h_v] fp32                                              */
    const void *do_;         /* [B*T][h_v][d_v] of desc->out_dtype, 16-byte aligned          */
    float *dq, *dk;          /* [B*T][h_qk][d_k] fp32                                        */
    float *dv;               /* [B*T][h_v][d_v] fp32                                         */
    float *dg, *dbeta;       /* [B*T][h_v] fp32                                              */
} bdgdn_noisy_view_grad_t;

/* Bytes of device workspace bdgdn_bwd_train_views needs (that of bdgdn_bwd_train: the views
 * share it). */
size_t bdgdn_bwd_train_views_workspace(const bdgdn_fwd_desc_t *desc);

/*
 * Backward of bdgdn_fwd_train_views (the complementary-view objective of Sec. 3.3 "Training
 * Objective and Mask Design": several noisy views, each block seeded from the same clean
 * state): the gradients of
 *     sum <do, o> + sum_i sum <views[i].do_, o_i> + <dht, ht>
 * for 1 <= n_views <= 16.  Every view's noisy block b sends its seed's gradient into the
 * clean state gradient at the end of clean block b - 1 (eq. dh-block-recursion, summed over
 * the views).  Clean inputs, h0, do, dht, dq .. dbeta, dh0 and the workspace as for
 * bdgdn_bwd_train; each view's gradients go to its own arrays.  The same support and
 * errors as bdgdn_bwd_train; deterministic except for the grouped-head atomics described
 * there.
 */
int bdgdn_bwd_train_views(const bdgdn_fwd_desc_t *desc,
                          const void *q, const void *k, const void *v,
                          const float *g, const float *beta,
                          const bdgdn_noisy_view_grad_t *views, int32_t n_views,
                          const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host,
                          const float *h0, const void *do_, const float *dht,
                          float *dq, float *dk, float *dv, float *dg, float *dbeta, float *dh0,
                          void *workspace, size_t workspace_bytes, void *stream);

/*
 * One Diffusion-Trust denoise pass over R blocks (Appendix "Per-block denoise loop",
 * "Differences between the denoise pass and the state-update pass").  Request r's
 * block is seeded with state_pool[slot[r]] (slot == NULL means slot[r] = r) and every
 * position reads the block-end state.  state_pool is only read.
 *
 *   state_pool  [n_slots][h_v][d_k][d_v] fp32 (device)
 *   slot        [R] int32 device array of pool indices, or NULL
 *   q, k, v     [R*L][h][d] (dtype); g, beta [R*L][h_v] fp32
 *   o           [R*L][h_v][d_v] block-end readout (out_dtype)
 * Slot indices are not range-checked on the device; they must be valid.
 */
int bdgdn_denoise_step(const bdgdn_serve_desc_t *desc, const float *state_pool,
                       const int32_t *slot, const void *q, const void *k, const void *v,
                       const float *g, const float *beta, void *o, void *stream);

/*
 * Token-causal state-update pass over R blocks (Appendix Algorithm "Diffusion-Trust
 * serving loop", the forward that writes S back): state_pool[slot[r]] is advanced by
 * the L tokens of request r, in place.  o_causal ([R*L][h_v][d_v], out_dtype) receives the
 * causal readout when not NULL.  Slots must be distinct (calls with repeated slots
 * race) and valid.
 */
int bdgdn_commit(const bdgdn_serve_desc_t *desc, float *state_pool, const int32_t *slot,
                 const void *q, const void *k, const void *v,
                 const float *g, const float *beta, void *o_causal, void *stream);

/*
 * The AR-Trust verify pass with its state cache (Appendix "Serving-system machinery for
 * the hybrid backbone", cache-and-scatter; Algorithm "AR-Trust serving round"): the
 * commit pass of bdgdn_commit over each request's block of L = desc->block positions
 * (e.g. the anchor and K draft tokens, L = K + 1), which also writes, for the block's
 * last n_record positions p = L - n_record + i (i = 0 .. n_record-1), the state before
 * position p:
 *
 *   states      [R][n_record][h_v][d_k][d_v] fp32 (device, 16-byte aligned), written
 *               whole; states[r][i] is the state after the first L - n_record + i
 *               positions of request r (the cached state itself when that is 0).
 *
 * The pool then holds the state after all L positions, exactly as after bdgdn_commit
 * (o_causal as there).  1 <= n_record <= block.  Available for bf16 inputs with
 * d_k = d_v = 128 and blocks of at most 32 positions (else BDGDN_ERR_UNSUPPORTED).
 */
int bdgdn_commit_record(const bdgdn_serve_desc_t *desc, float *state_pool, const int32_t *slot,
                        const void *q, const void *k, const void *v,
                        const float *g, const float *beta, void *o_causal,
                        int32_t n_record, float *states, void *stream);

/*
 * The accept step after a verify decision: request r keeps the state at its accepted
 * offset, state_pool[slot[r]][h] = states[r][accept[r]][h] for every v-head h, in one
 * launch (one workgroup per (request, v-head)).
 *
 *   accept      [R] int32 device array; accept[r] == n_record keeps the state already in
 *               the pool (the verify pass's final state); values outside [0, n_record]
 *               also leave the slot untouched (they are not checked on the host).
 *   states      as written by bdgdn_commit_record with the same n_record and desc.
 * state_pool and states must be 16-byte aligned.  Any supported (d_k, d_v).
 */
int bdgdn_accept_states(const bdgdn_serve_desc_t *desc, float *state_pool, const int32_t *slot,
                        const float *states, int32_t n_record, const int32_t *accept, void *stream);

/*
 * The two-stream 1D causal ShortConv in front of the GDR inputs (Appendix "ShortConv under
 * two-stream training", eq. short-conv-clean and eq. short-conv-noisy, computed in the fused
 * form that picks each lag's stream in place), per channel c with filter w[c][0..W-1]:
 *
 *   y[t]   = act(bias[c] + sum_i w[c][i] x[t-i])
 *   yn[t]  = act(bias[c] + sum_i w[c][i] z(t, t-i)),  z(t, s) = xn[s] if s lies in t's
 *            diffusion block, else x[s]
 *
 * with diffusion blocks of `block` rows counted from each sequence's (or document's) start,
 * and rows before that start read as zero (Appendix "Document-packed training", the
 * ShortConv lag mask).  act is the identity or silu.
 *
 *   x, xn, y, yn   [B*T][channels] of dtype (the clean and noisy streams), 8-byte aligned
 *   w              [channels][width] fp32, w[c][i] the weight of lag i
 *   bias           [channels] fp32, or NULL for none
 *   cu_seqlens_*   both NULL (B sequences of T rows) or both [N+1] int32 offsets into the
 *                  packed rows (B == 1, cu[0] == 0, cu[N] == T, non-decreasing; any
 *                  document lengths).  The two copies must hold the same values.
 * Supported: dtype bf16 or fp32, 1 <= width <= 4, channels a multiple of 4 (bf16) or 2
 * (fp32); else BDGDN_ERR_UNSUPPORTED.  The token tensors may be NULL when B*T == 0.
 * Results are deterministic.
 */
/* (the ShortConv takes the first two) */
typedef enum { BDGDN_ACT_NONE = 0, BDGDN_ACT_SILU = 1, BDGDN_ACT_SIGMOID = 2 } bdgdn_act_t;

typedef struct {
    int32_t batch;      /* B sequences; must be 1 when packed (num_seqs > 0)           */
    int32_t seqlen;     /* T rows per sequence, or total packed rows                    */
    int32_t num_seqs;   /* N packed documents, 0 when not packed                        */
    int32_t channels;   /* D, the row length of every token tensor                      */
    int32_t width;      /* W filter taps                                                */
    int32_t block;      /* diffusion block size L                                       */
    int32_t activation; /* bdgdn_act_t                                                  */
    int32_t dtype;      /* bdgdn_dtype_t of x, xn, y, yn, dy, dyn, dx, dxn              */
} bdgdn_conv_desc_t;

/* Forward: writes every row of y and yn. */
int bdgdn_shortconv_fwd(const bdgdn_conv_desc_t *desc, const void *x, const void *xn, const float *w,
                        const float *bias, const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host,
                        void *y, void *yn, void *stream);

/* Bytes of device workspace bdgdn_shortconv_bwd needs (0 when there are no rows, or for a
 * descriptor it would reject). */
size_t bdgdn_shortconv_bwd_workspace(const bdgdn_conv_desc_t *desc);

/*
 * Backward of bdgdn_shortconv_fwd for the upstream gradients dy, dyn ([B*T][channels],
 * dtype): writes dx, dxn (dtype, every row), dw ([channels][width] fp32) and, when not
 * NULL, dbias ([channels] fp32); all are overwritten, not accumulated into.  Each noisy
 * output's gradient flows to the stream it read at each lag.  workspace: device memory
 * of at least bdgdn_shortconv_bwd_workspace(desc) bytes, 256-byte aligned, scratch owned
 * by the call until the stream passes it.
 */
int bdgdn_shortconv_bwd(const bdgdn_conv_desc_t *desc, const void *x, const void *xn, const float *w,
                        const float *bias, const void *dy, const void *dyn, const int32_t *cu_seqlens_dev,
                        const int32_t *cu_seqlens_host, void *dx, void *dxn, float *dw, float *dbias,
                        void *workspace, size_t workspace_bytes, void *stream);

/*
 * bdgdn_shortconv_bwd without a workspace argument, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving or training loops, harnesses that
 * forbid allocation).  It computes exactly what bdgdn_shortconv_bwd computes, with the same
 * kernels and the same summation order (bit-identical results), and calls no allocating
 * routine: its dw / dbias partials live in a scratch array of BDGDN_NOALLOC_SCRATCH_BYTES
 * that the library holds on each GPU it runs on until the process ends (looked up on the
 * first call on a device; the stream's device, or the current device for a NULL stream).
 * Inputs needing more than that (bdgdn_shortconv_bwd_workspace(desc) bytes: 4 (width + 1)
 * channels bytes per started group of 1024 rows, e.g. 1.9 MiB for 16384 rows of 6144
 * channels at width 4) return BDGDN_ERR_SCRATCH before anything is launched.  Every call on one GPU
 * shares that GPU's scratch: calls whose execution overlaps on one GPU (different streams,
 * or threads launching concurrently) race and give undefined dw / dbias; serialise them
 * on one stream.  The caller still owns every input and output buffer.
 */
#define BDGDN_NOALLOC_SCRATCH_BYTES (32u << 20)
int bdgdn_shortconv_bwd_noalloc(const bdgdn_conv_desc_t *desc, const void *x, const void *xn, const float *w,
                                const float *bias, const void *dy, const void *dyn,
                                const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, void *dx,
                                void *dxn, float *dw, float *dbias, void *stream);

/*
 * ------------------------------------------------------------------------------------
 * The softmax half of a serving round.  In a hybrid backbone the layers between the Gated
 * DeltaNet ones attend over a cache of keys and values.  The entry points below serve them
 * beside bdgdn_denoise_step / bdgdn_commit / bdgdn_commit_record: attention of a block of new
 * nodes over the cache (bdgdn_tree_attn), the verify decision of an AR-Trust round
 * (bdgdn_verify), whose counts bdgdn_accept_states takes, and the pages of the cache
 * (bdgdn_cache_append, _fork, _compact, _truncate).
 *
 * The cache.  A pool holds the keys, or the values, of one layer in n_pages pages of `page`
 * tokens; element e of head h of token t of page p lies at
 *     p * page_stride + t * token_stride + h * head_stride + e        (elements)
 * so that [n_pages][page][h_kv][d], [n_pages][h_kv][page][d] and slices of larger arrays are
 * all pools.  The sequence in slot s has seq_len[s] tokens; token t lies in page
 * page_table[s][t / page] at place t % page.  Slots are rows of page_table; a `slot` array
 * [R] names the slot of each request (attention takes NULL for slot[r] = r).
 * Slot numbers outside [0, n_slots) count as empty sequences; a table entry outside
 * [0, n_pages) is a page that is not there: its tokens are attended to by nobody.
 */
typedef struct {
    int32_t n_pages;        /* pages of every pool                                        */
    int32_t page;           /* tokens of a page, 1 .. 65536                               */
    int32_t n_slots;        /* rows of page_table, entries of seq_len                     */
    int32_t max_pages;      /* columns of page_table; max_pages * page < 2^31 (for
                               attention at most 2^31 - 2^16)                             */
    int32_t h_kv, d;        /* heads and head dimension of the pools                      */
    int32_t dtype;          /* bdgdn_dtype_t of the pools                                 */
    int64_t page_stride, token_stride, head_stride;   /* elements, multiples of 16 bytes;
                               a token's at most 2^26 bytes                               */
} bdgdn_cache_desc_t;

typedef enum {
    BDGDN_MASK_FULL = 0,    /* every node sees every node (a diffusion block)             */
    BDGDN_MASK_CAUSAL = 1,  /* node n sees nodes 0 .. n (a chain: anchor and drafts)      */
    BDGDN_MASK_BITS = 2     /* node n sees node j where bit j of mask[r][n] is set        */
} bdgdn_mask_t;

typedef struct {
    int32_t num_req;        /* R                                                          */
    int32_t nodes;          /* N new nodes per request, 1 .. 64                           */
    int32_t h_q, h_kv, d;   /* h_q % h_kv == 0; d in {64, 128, 256}                       */
    float scale;
    int32_t dtype;          /* bdgdn_dtype_t of q, k, v and the pools                     */
    int32_t out_dtype;      /* bdgdn_dtype_t of o                                         */
    int32_t mask;           /* bdgdn_mask_t                                               */
    int64_t q_stride, k_stride, v_stride;   /* elements between the rows of two nodes, 0 for
                               contiguous ones; multiples of 16 bytes (q, k, v may be parts
                               of the rows of one projection)                             */
} bdgdn_attn_desc_t;

/* Bytes of device workspace bdgdn_tree_attn needs, 0 for descriptors that it rejects (more
 * than R (max_pages page / 32 + 9) = 2^31 - 2^16 tiles, R N h_q = 2^30 rows or, in groups of 16 to
 * a key head, 2^24 groups of rows among them). */
size_t bdgdn_tree_attn_workspace(const bdgdn_attn_desc_t *desc, const bdgdn_cache_desc_t *cache);

/*
 * Attention of N new nodes per request over the request's cached tokens and over the nodes
 * themselves.  Node n of request r sees every cached token that is there and the nodes j <
 * count[r] that the mask lets it see (itself only where the mask says so):
 *     s_x = scale <q_n, k_x>,  o = sum_x exp(s_x) v_x / sum_x exp(s_x),  lse = log sum_x exp(s_x)
 * A node that sees nothing, and a node n >= count[r], has o = 0 and lse = -inf.  What a node
 * does not see has no part in its result, not even a NaN or an infinity.
 *   q               [R][N][h_q][d] of dtype (head h reads key head h / (h_q / h_kv))
 *   k, v            [R][N][h_kv][d] of dtype: the nodes' own keys and values
 *   k_pages, v_pages  pools as described above, 16-byte aligned, of at most 2^36 bytes
 *   page_table, seq_len   the cache's tables (read only; lengths beyond the table's columns
 *                   count as max_pages * page)
 *   slot            [R] int32, or NULL for slot[r] = r (then R <= n_slots)
 *   count           [R] int32 nodes of each request, or NULL for N
 *   mask            [R][N] 64-bit words (BDGDN_MASK_BITS), else NULL
 *   o               [R][N][h_q][d] of out_dtype, every row written
 *   lse             [R][N][h_q] fp32, or NULL
 *   workspace       256-byte aligned, owned by the call until the stream passes it
 * Scores, the softmax's statistics and all sums are fp32.  With bf16 inputs the products are
 * exact in fp32 and the weights exp(s - m) enter the product with v in two bf16 parts (16
 * significant bits); their sum, and lse with it, is that of the unrounded ones.  Results are
 * deterministic.  (dtype, out_dtype) as for the other entry
 * points: (bf16, bf16), (bf16, fp32), (fp32, fp32).
 */
int bdgdn_tree_attn(const bdgdn_attn_desc_t *desc, const bdgdn_cache_desc_t *cache, const void *q,
                    const void *k, const void *v, const void *k_pages, const void *v_pages,
                    const int32_t *page_table, const int32_t *seq_len, const int32_t *slot,
                    const int32_t *count, const uint64_t *mask, void *o, float *lse,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * The mask words of drafted trees: bit j of mask[r][n] is set for n itself and for its
 * ancestors.  parent is [R][N] int32 with parent[r][n] < n; any other value makes n a root.
 * depth ([R][N] int32, or NULL) receives the number of ancestors, by which a node's position
 * follows the sequence's length.  1 <= nodes <= 64.
 */
int bdgdn_tree_mask(int32_t num_req, int32_t nodes, const int32_t *parent, uint64_t *mask,
                    int32_t *depth, void *stream);

typedef struct {
    int32_t num_req;        /* R                                                          */
    int32_t nodes;          /* N nodes: the anchor (node 0) and N - 1 drafts, 1 .. 64     */
    int32_t vocab;          /* V                                                          */
    int32_t dtype;          /* bdgdn_dtype_t of target and draft                          */
    int64_t target_req_stride, target_row_stride;   /* elements; rows are contiguous      */
    int64_t draft_req_stride, draft_row_stride;
    int64_t noise_stride;                           /* elements between requests' noise   */
} bdgdn_verify_desc_t;

/* Bytes of device workspace bdgdn_verify needs, 0 for a descriptor that it rejects. */
size_t bdgdn_verify_workspace(const bdgdn_verify_desc_t *desc);

/*
 * Verification of drafted tokens (the exact rejection rule of AR-Trust decoding, for chains
 * and trees of drafts), with the random numbers given.  Row n of target holds the target's
 * logits after node n, p = softmax(target / T); row n of draft those that the children of n
 * were drawn from, q = softmax(draft / T), each child by itself (two children may carry the
 * same token).  The walk begins at node 0 and tries the children of the node that it is on
 * in index order.  After j refusals the law of the next token is
 *     (p - c q)+ / W,   c = 0, W = 1 at first; each refusal: c += W, W = sum (p - c q)+
 * ((x/W - q)+ = (x - W q)+ / W, so the residuals of all refusals have this form), and the
 * child with token d is accepted where u W q(d) < (p(d) - c q(d))+.  Without a draft the
 * proposals are certain (a draft's most likely tokens): a refused token leaves the law, W is
 * what remains, and d is accepted where u W < p(d).  When no child is accepted the next
 * token is drawn from the law by the exponential race, argmax_t law(t) / noise(t), the lowest
 * t of equals (where the law is zero everywhere, p takes its place).
 *   target       [R][N][V] logits (strides in desc), aligned to an element
 *   draft        [R][N or N-1][V] logits or NULL (the rows of nodes without children are not
 *                read, so the last row may be absent)
 *   token        [R][N] int32: the drafts' tokens (node 0's is not read); a token outside
 *                [0, V) is refused and leaves the law as it is
 *   parent       [R][N] int32 with 0 <= parent[r][n] < n for n >= 1 (other values: the node
 *                is nobody's child), or NULL for chains (parent n - 1)
 *   count        [R] int32 nodes of each request, or NULL for N
 *   temperature  [R] fp32, or NULL for 1; T <= 0 (or NaN) is greedy: p is all on the target's
 *                largest logit, the lowest index of equals, and the draft is not looked at
 *   u            [R][N] fp32 in [0, 1): u[r][n] decides on node n
 *   noise        [R][V] fp32 > 0, exponentially distributed (stride in desc)
 *   n_accept     [R] int32: accepted drafts, the `accept` of bdgdn_accept_states for a chain
 *                recorded with block N and n_record N - 1
 *   n_path       [R] int32: n_accept + 1, the nodes of the path (bdgdn_cache_append's count),
 *                or NULL
 *   path         [R][N] int32: the path's nodes, node 0 first, then -1
 *   next_token   [R] int32
 * A row with a NaN, a +inf or nothing finite has no law: no child of its node is accepted,
 * and if it is a target's, the next token is -1; so it is for count[r] < 1, with n_accept 0,
 * n_path 0.
 * Logits of -inf are tokens of probability zero.  Deterministic.
 */
int bdgdn_verify(const bdgdn_verify_desc_t *desc, const void *target, const void *draft,
                 const int32_t *token, const int32_t *parent, const int32_t *count,
                 const float *temperature, const float *u, const float *noise, int32_t *n_accept,
                 int32_t *n_path, int32_t *path, int32_t *next_token, void *workspace,
                 size_t workspace_bytes, void *stream);

/*
 * The tables of a cache (device memory).  refcount[p] is the number of table entries that
 * hold page p; bit p % 32 of free_bits[p / 32] is set where that is zero.  An empty cache has
 * seq_len and refcount zero and the bits of pages 0 .. n_pages - 1 set, those beyond clear.
 * Pages are taken lowest first, in the order of the requests, so the tables depend on
 * nothing but the calls.  The slots of a call must differ (calls with repeated slots race),
 * and calls on one cache must be ordered by their streams.
 */
typedef struct {
    int32_t *page_table;    /* [n_slots][max_pages]; entries past a sequence's pages are -1 */
    int32_t *seq_len;       /* [n_slots]                                                    */
    int32_t *refcount;      /* [n_pages]                                                    */
    uint32_t *free_bits;    /* [(n_pages + 31) / 32]                                        */
} bdgdn_cache_tables_t;

/* What a cache call did with a request (status[r]). */
#define BDGDN_CACHE_DONE     0
#define BDGDN_CACHE_NO_PAGES 1   /* too few free pages for it, after the requests before it  */
#define BDGDN_CACHE_NO_ROOM  2   /* more tokens than max_pages * page                        */
#define BDGDN_CACHE_BAD_SLOT 3   /* a slot outside [0, n_slots); a fork into a slot in use   */
#define BDGDN_CACHE_BAD_KEEP 4   /* positions to keep that do not rise or are not there      */

/* Bytes of device workspace bdgdn_cache_append (rows_max: the rows that a request may add)
 * and bdgdn_cache_compact (rows_max: the positions that it may keep) need for num_req
 * requests, 0 for a descriptor or sizes that they reject (at most 65535 requests, which
 * together may touch 2^30 pages). */
size_t bdgdn_cache_workspace(const bdgdn_cache_desc_t *cache, int32_t num_req, int32_t rows_max);

/*
 * Appends rows to the sequences in slot[0 .. R-1]: rows path[r][0 .. count[r]-1] of request r
 * (rows 0 .. count[r]-1 where path is NULL) go behind its last token, in every pool.  A last
 * page that is not full and is shared with another sequence when the call begins is replaced
 * by a page of its own with a copy of its tokens (copy on write); one that is not there (its table
 * entry was dropped), by a page with rows of zeros for them.
 *   pools        host array of n_pools device pointers (keys and values of every layer), each
 *                with the geometry of `cache`, 16-byte aligned
 *   rows         host array of n_pools device pointers: [R][N][h_kv][d] of the pools' dtype
 *                with row_stride elements between the rows of two nodes (0: contiguous), the
 *                k and v that bdgdn_tree_attn took; 16-byte aligned
 *   path         [R][N] int32 (the path of bdgdn_verify), or NULL; a node outside [0, N)
 *                gives a row of zeros
 *   count        [R] int32, 0 .. N (values outside are clamped)
 *   status       [R] int32, or NULL: what was done; a request that is not done leaves its
 *                sequence as it was
 *   workspace    at least bdgdn_cache_workspace(cache, R, N) bytes, 256-byte aligned
 */
int bdgdn_cache_append(const bdgdn_cache_desc_t *cache, const bdgdn_cache_tables_t *tables, void *const *pools,
                       const void *const *rows, int32_t n_pools, int32_t num_req, int32_t nodes,
                       int64_t row_stride, const int32_t *slot, const int32_t *path, const int32_t *count,
                       int32_t *status, void *workspace, size_t workspace_bytes, void *stream);

/* Gives slot dst[i] the sequence of src[i] by sharing its pages, i = 0 .. num_req - 1.  The
 * slots dst must be empty (seq_len 0, else BDGDN_CACHE_BAD_SLOT) and no slot may be both a
 * source and a destination; a source may be forked many times. */
int bdgdn_cache_fork(const bdgdn_cache_desc_t *cache, const bdgdn_cache_tables_t *tables, int32_t num_req,
                     const int32_t *src, const int32_t *dst, int32_t *status, void *stream);

/*
 * Keeps the positions keep[r][0 .. count[r]-1] (rising, each below the sequence's length) of
 * slot[r] and drops the others: token j of the sequence is now what token keep[r][j] was, in
 * every pool.  Leading pages whose tokens all stay where they are are kept (also shared ones);
 * the tokens behind them move to new pages (as rows of zeros where their page is not there), and
 * the old ones are given back.  keep is [R][M]
 * int32, count [R] int32 (values outside 0 .. M are clamped); pools, status and workspace
 * (bdgdn_cache_workspace(cache, R, M)) as for bdgdn_cache_append.
 */
int bdgdn_cache_compact(const bdgdn_cache_desc_t *cache, const bdgdn_cache_tables_t *tables, void *const *pools,
                        int32_t n_pools, int32_t num_req, int32_t keep_max, const int32_t *slot,
                        const int32_t *keep, const int32_t *count, int32_t *status, void *workspace,
                        size_t workspace_bytes, void *stream);

/* Shortens the sequences in slot[0 .. R-1] to min(seq_len, length[r]) tokens (length NULL or
 * negative: 0, which frees the slot) and gives back the pages that they no longer use. */
int bdgdn_cache_truncate(const bdgdn_cache_desc_t *cache, const bdgdn_cache_tables_t *tables, int32_t num_req,
                         const int32_t *slot, const int32_t *length, void *stream);

/*
 * ------------------------------------------------------------------------------------
 * Around the mixers.  What a hybrid layer does with its rows before and behind the Gated
 * DeltaNet and the attention, and with the logits before bdgdn_verify: rotary positions
 * (bdgdn_rope), the norms behind and in front of a mixer with gate, scale and residual
 * (bdgdn_norm_fwd, bdgdn_norm_bwd), projections in 8-bit integers (bdgdn_quant_rows,
 * bdgdn_quant_matmul), penalties, biases and grammar masks (bdgdn_logits, bdgdn_history_add).
 *
 * Tensors of these calls have contiguous innermost rows and otherwise the strides (elements,
 * not negative) of the descriptor, so they may be parts of the rows of one projection; they
 * are aligned to an element, and run fastest where addresses and strides are multiples of 16
 * bytes.  Rows of an output share no memory (BDGDN_ERR_INVALID_ARG).  Where a call may work in
 * place, the output is the input: the same address and the same strides.
 */
typedef enum {
    BDGDN_ROPE_HALF = 0,    /* element i of the rotated ones turns with element i + rot / 2 */
    BDGDN_ROPE_PAIRS = 1    /* element 2 i turns with element 2 i + 1                       */
} bdgdn_rope_layout_t;

typedef enum {
    BDGDN_ROPE_PLAIN = 0,   /* w_i = base^(-2 i / rot)                                      */
    BDGDN_ROPE_LINEAR = 1,  /* w_i / factor: positions pressed together                     */
    BDGDN_ROPE_NTK = 2,     /* base factor^(rot / (rot - 2)) for base                       */
    BDGDN_ROPE_PARTS = 3    /* pairs that turn more than `fast` times over `original` positions
                               keep w_i, those of fewer than `slow` turns take w_i / factor,
                               those between a mixture of both, linear in the turns         */
} bdgdn_rope_scaling_t;

typedef struct {
    int32_t rot;            /* rotated elements of a head, even                             */
    int32_t scaling;        /* bdgdn_rope_scaling_t                                         */
    double base, factor;    /* base >= 1, factor > 0                                        */
    double original, slow, fast;   /* BDGDN_ROPE_PARTS: original > 0, 0 <= slow < fast      */
} bdgdn_rope_freq_t;

/* Fills turns_host[0 .. rot/2 - 1] (host memory) with the pairs' turns a position,
 * w_i / (2 pi), as fractions in units of 2^-64 (whole turns left out).  A position's angle is
 * then an integer product modulo 2^64: exact for every position, near or far. */
int bdgdn_rope_freqs(const bdgdn_rope_freq_t *freq, uint64_t *turns_host);

typedef struct {
    int64_t req, row, head;          /* elements between requests, rows, heads              */
} bdgdn_heads_t;

typedef struct {
    int32_t num_req, nodes;          /* R requests (or sequences) of N rows                 */
    int32_t h_q, h_k;                /* heads of q and of k (0: q alone)                    */
    int32_t d, rot;                  /* head dimension (at most 4096), rotated elements     */
    int32_t layout;                  /* bdgdn_rope_layout_t                                 */
    int32_t dtype;                   /* bdgdn_dtype_t of q, k and the outputs               */
    int32_t inverse;                 /* turn back: the gradient of the rotation             */
    int32_t n_slots;                 /* entries of seq_len                                  */
    float scale;                     /* multiplies the rotated elements                     */
    bdgdn_heads_t q, k, q_out, k_out;
} bdgdn_rope_desc_t;

/*
 * Rotary positions.  The first rot elements of every head of row n of request r turn by the
 * position p = seq_len[slot[r]] + pos[r][n]: a pair (a, b) becomes
 *     scale (a cos t - b sin t),  scale (a sin t + b cos t),   t = 2 pi turns[i] p / 2^64
 * the other elements stay.  inverse turns by -t: for an upstream gradient of the rotated rows
 * it gives the gradient of the rows.
 *   q, k        [R][N][heads][d] (k NULL where h_k is 0)
 *   turns       [rot / 2] 64-bit words of bdgdn_rope_freqs, on the device
 *   pos         [R][N] int32, or NULL for n (a tree's depths: bdgdn_tree_mask's depth)
 *   seq_len     [n_slots] int32 cached tokens (negative: 0), or NULL for 0
 *   slot        [R] int32, or NULL for slot[r] = r (then R <= n_slots); a slot outside
 *               [0, n_slots) is an empty sequence
 *   count       [R] int32 rows of each request, or NULL for N; rows behind them are not read
 *               and their outputs left as they were
 *   q_out, k_out  as q, k; may be q, k
 * Angles are exact to 2^-33 of a turn, cos and sin to 2^-23; results are rounded once.
 */
int bdgdn_rope(const bdgdn_rope_desc_t *desc, const void *q, const void *k, const uint64_t *turns,
               const int32_t *pos, const int32_t *seq_len, const int32_t *slot, const int32_t *count,
               void *q_out, void *k_out, void *stream);

typedef struct {
    int64_t outer, inner;            /* elements between rows [a][b] in a and in b          */
} bdgdn_rows_t;

typedef struct {
    int32_t outer, inner;            /* rows [outer][inner] (tokens and heads; inner 1)     */
    int32_t d;                       /* elements of a row, 1 .. 16384                       */
    int32_t x_dtype, r_dtype, dtype; /* bdgdn_dtype_t of x; of r and r_out; of z and y      */
    int32_t post, pre;               /* 1: normalise behind the mixer, in front of the next */
    int32_t act;                     /* bdgdn_act_t of the gate                             */
    float scale, eps;
    bdgdn_rows_t x, z, r, r_out, y;
    bdgdn_rows_t dx, dz, dr, dr_out, dy;   /* the backward's                                */
} bdgdn_norm_desc_t;

/*
 * The norms around a mixer, its gate, scale and residual, a row at a time:
 *     n  = post ? x / rms(x) * w_post : x,          rms(x) = sqrt(mean x^2 + eps)
 *     u  = z ? n act(z) : n
 *     r' = r + scale layer_scale u
 *     y  = pre ? r' / rms(r') * w_pre : r'
 * With x alone and post it is an RMS norm, with z the gated norm of a Gated DeltaNet's heads.
 *   x           mixer's output; z its gate or NULL; r the residual or NULL for 0
 *   w_post, w_pre, layer_scale   [d] fp32, or NULL for 1
 *   r_out       r', of r's type, may be r; or NULL
 *   y           of dtype, or NULL (not both)
 * Sums and statistics are fp32; y comes from the unrounded r'; each result is rounded once.
 * Types: x, r, dtype bf16 or fp32, with dtype fp32 only if x and r are.  r_dtype counts also
 * where there is no r.
 */
int bdgdn_norm_fwd(const bdgdn_norm_desc_t *desc, const void *x, const void *z, const void *r,
                   const float *w_post, const float *w_pre, const float *layer_scale, void *r_out,
                   void *y, void *stream);

/* Bytes of device workspace bdgdn_norm_bwd needs, 0 for a descriptor that it rejects. */
size_t bdgdn_norm_bwd_workspace(const bdgdn_norm_desc_t *desc);

/*
 * Its backward, for upstream gradients dy of y and dr_out of r'.
 *   x, z, w_post, w_pre, layer_scale   what the forward took
 *   r_out       the forward's r' (as stored); NULL only where it took no r: then r' is computed
 *               again
 *   dy          of dtype, dr_out of r_dtype; either NULL for 0
 *   dx, dz, dr  of x's, z's and r's type, or NULL (dr may be dr_out)
 *   dw_post, dw_pre, dlayer_scale   [d] fp32 sums over the rows, or NULL.  They need post, pre
 *               and nothing; deterministic
 *   workspace   256-byte aligned, owned by the call until the stream passes it
 */
int bdgdn_norm_bwd(const bdgdn_norm_desc_t *desc, const void *x, const void *z, const void *r_out,
                   const float *w_post, const float *w_pre, const float *layer_scale, const void *dy,
                   const void *dr_out, void *dx, void *dz, void *dr, float *dw_post, float *dw_pre,
                   float *dlayer_scale, void *workspace, size_t workspace_bytes, void *stream);

typedef struct {
    int32_t num_req, nodes;          /* R requests of N nodes (the anchor and drafts), 1 .. 64 */
    int32_t vocab;
    int32_t dtype, out_dtype;        /* bdgdn_dtype_t of logits and out                     */
    int32_t n_slots;                 /* rows of history                                     */
    int32_t n_bias;                  /* entries of bias of each request                     */
    int64_t req_stride, row_stride;            /* of logits                                 */
    int64_t out_req_stride, out_row_stride;
    int64_t history_stride;                    /* words between the slots' rows             */
    int64_t allow_req_stride, allow_row_stride;   /* words; 0 for what all share            */
} bdgdn_logits_desc_t;

/*
 * Logits as the requests ask for them, in front of bdgdn_verify (and for plain sampling with
 * N = 1).  Row n of request r holds the logits after node n.  For token t, c is how often t has
 * been generated, in the history of slot[r] or by a node that n's mask word names, and t is
 * seen where c > 0 or the prompt holds it:
 *     x = seen ? (x > 0 ? x (1 / repetition) : x repetition) : x      (1 / repetition in fp32)
 *     x = x - (c > 0 ? presence : 0) - frequency c
 *     x = x + bias,   -inf where the grammar does not allow t
 *   logits       [R][N][V] of dtype (rows contiguous)
 *   history      [n_slots][V] int32: generated occurrences, + 2^30 where the prompt holds the
 *                token (bdgdn_history_add); NULL for none
 *   slot         [R] int32, or NULL for slot[r] = r (then R <= n_slots); a slot outside
 *                [0, n_slots) has no history
 *   token        [R][N] int32 the nodes' tokens, or NULL where they do not count; a token
 *                outside [0, V) counts for nothing (-1 for an anchor that is the prompt's last
 *                token: it was not generated, and the history has marked it)
 *   mask         [R][N] 64-bit words of bdgdn_tree_mask (bit j: node j is n or its ancestor),
 *                or NULL for chains
 *   count        [R] int32 nodes of each request, or NULL for N; rows behind them are not read,
 *                and left as they were
 *   repetition, presence, frequency   [R] fp32, or NULL for 1, 0, 0; a repetition that is not
 *                above zero counts as 1
 *   bias_token, bias   [R][n_bias] int32 and fp32; entries outside [0, V) count for nothing, of
 *                entries with one token the last one counts
 *   allow        bit t % 32 of word t / 32 of the row: t is allowed; NULL: all are
 *   out          [R][N][V] of out_dtype, may be logits where the types are the same
 * fp32 arithmetic, rounded once.  (dtype, out_dtype): (bf16, bf16), (bf16, fp32), (fp32, fp32).
 */
int bdgdn_logits(const bdgdn_logits_desc_t *desc, const void *logits, const int32_t *history,
                 const int32_t *slot, const int32_t *token, const uint64_t *mask, const int32_t *count,
                 const float *repetition, const float *presence, const float *frequency,
                 const int32_t *bias_token, const float *bias, const uint32_t *allow, void *out, void *stream);

/*
 * Adds tokens to histories: token[r][path[r][j]], j < count[r], of request r to the history of
 * slot[r], as generated ones (one more each) or, with prompt 1, as the prompt's (bit 30 set).
 *   history     [n_slots][vocab] int32 with history_stride between the slots
 *   token       [R][N] int32 (outside [0, vocab): left out); path [R][N] int32 (bdgdn_verify's
 *               path; a node outside [0, N) is left out) or NULL for rows in order
 *   count       [R] int32 (clamped to 0 .. N), or NULL for N;  slot as for bdgdn_logits
 * Slots may repeat.  A token may have been generated fewer than 2^30 times.
 */
int bdgdn_history_add(int32_t num_req, int32_t nodes, int32_t vocab, int32_t n_slots, int64_t history_stride,
                      int32_t *history, const int32_t *slot, const int32_t *token, const int32_t *path,
                      const int32_t *count, int32_t prompt, void *stream);

typedef struct {
    int32_t rows, cols;              /* of x                                                */
    int32_t width;                   /* of q: cols filled up to a multiple of 128           */
    int32_t dtype;                   /* bdgdn_dtype_t of x                                  */
    int64_t x_stride, q_stride;      /* elements between rows                               */
} bdgdn_quant_desc_t;

/*
 * 8-bit integers with a scale for each row (a token's activations, a channel's weights):
 *     scale = max |x| (1 / 127),  q = x / scale rounded to the nearest integer (of two the even one)
 * where 1 / 127, the product and the quotient are fp32 numbers.  Columns cols .. width - 1 of q are
 * zeros.  A row of zeros has scale 0; a row that holds a NaN or an infinity scale NaN; q is 0 in
 * both.  Fewer than 2^24 rows.
 *   x  [rows][cols];  q  [rows][width] int8, 16-byte aligned, q_stride a multiple of 16
 *   scale  [rows] fp32
 */
int bdgdn_quant_rows(const bdgdn_quant_desc_t *desc, const void *x, int8_t *q, float *scale, void *stream);

typedef struct {
    int32_t m, n, k;                 /* out [m][n]; k a multiple of 128, at most 130944     */
    int32_t out_dtype;
    int64_t a_stride, w_stride, out_stride;   /* elements between rows; a's and w's multiples of 16 */
} bdgdn_quant_matmul_desc_t;

/* Bytes of device workspace bdgdn_quant_matmul needs (0 also where it needs none). */
size_t bdgdn_quant_matmul_workspace(const bdgdn_quant_matmul_desc_t *desc);

/*
 * The product of rows of 8-bit integers with scales for each token and channel:
 *     out[i][j] = a_scale[i] w_scale[j] sum_k a[i][k] w[j][k] + bias[j]
 *   a  [m][k] int8, w  [n][k] int8, 16-byte aligned (bdgdn_quant_rows fills k up with zeros)
 *   a_scale [m], w_scale [n], bias [n] (or NULL) fp32;  out [m][n] of out_dtype
 *   workspace   256-byte aligned, owned by the call until the stream passes it
 * Sums are 32-bit integers and exact; the result is rounded to fp32 three times and to out's
 * type once.  Deterministic.
 */
int bdgdn_quant_matmul(const bdgdn_quant_matmul_desc_t *desc, const int8_t *a, const float *a_scale,
                       const int8_t *w, const float *w_scale, const float *bias, void *out, void *workspace,
                       size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* BDGDN_H */
