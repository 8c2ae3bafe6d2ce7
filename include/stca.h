/*
 * stca.h - C ABI of the MI355X (gfx950) STCA library.
 *
 * Stacked Target-to-History Cross Attention under Request Level Batching:
 * every target (candidate item) of a request attends, with a single query per
 * head, to that request's whole history, layer after layer (paper Sec. 3.1,
 * "Multi-head target-to-history cross attention" and Eq. layer-output).
 * The history of a request is projected to the per-layer K/V once and the
 * projection is shared by all of that request's targets (Sec. 3.2, App. A.3).
 * Ragged batches are packed without padding; per-request offset arrays mark
 * the segments (App. A.4, the index-based ragged target attention).
 *
 * Layer (the benchmark workloads' form of the stacked update, Sec. 3.1
 * "Stacking" replaced by a residual FFN; biases omitted as in the paper):
 *   s^(0)   = x_t
 *   q       = s^(i) W_Q^i                          head j: columns [j d_h, (j+1) d_h)
 *   a_j     = softmax(q_j (X W_K^i)_j^T / sqrt(d_h)) (X W_V^i)_j      over the request's history X
 *   u       = s^(i) + [a_1 | ... | a_h] W_O^i
 *   s^(i+1) = u + ReLU(u W_1^i) W_2^i
 *   out     = s^(n)
 *
 * Conventions shared by every entry point:
 *  - All tensor pointers are device pointers unless named *_host, and must be
 *    16-byte aligned.  Matrices are row-major; y = x W (W is [d_in][d_out]).
 *  - Weights are stacked per layer: wq, wk, wv, wo [n_layers][d][d],
 *    w1 [n_layers][d][ffn_hidden], w2 [n_layers][ffn_hidden][d].
 *  - Storage dtype (STCA_F32 or STCA_BF16) applies to hist, tgt, the weights,
 *    out and dout; accumulation is always fp32; gradients are fp32 (of the
 *    stand-alone attention: in the storage dtype, its bias table's fp32).
 *  - Range of the bf16 path.  bf16 storage keeps two bytes per value inside
 *    the kernels as well, but in fp16 (three more mantissa bits, which the
 *    attention's accuracy needs): the projected K and V, the queries, the
 *    softmax weights and the target update's activations are fp16 MFMA
 *    operands (fp32 accumulation), so each must stay below 65504 in
 *    magnitude (the fp32 state and the fp32 sums have no such limit).  The
 *    inputs themselves may use the whole bf16 range.  The forward's target
 *    update checks every value it rounds to fp16 (input targets, merged
 *    attention output, activations, next queries); an overflowed V, or a K
 *    whose overflow drives a score to plus infinity, reaches it as a
 *    non-finite attention output.  A violation is recorded in the workspace
 *    and stca_device_status() then returns STCA_ERR_RANGE; outputs of such a
 *    call are undefined.  A K entry whose overflow drives its score to minus
 *    infinity only removes that history row from the softmax and is not
 *    detected.  The backward of at most 32 targets per request recomputes the
 *    attention on fp16 operands of two terms (hi + lo), which have the same
 *    range and are not checked; with more targets, and in the generic form, K,
 *    V and the queries are fp32.  Non-finite inputs propagate.
 *  - Request r owns hist rows [hist_off[r], hist_off[r+1]) and tgt rows
 *    [tgt_off[r], tgt_off[r+1]).  offsets[0] = 0, non-decreasing,
 *    offsets[R] = n_hist / n_tgt.  A request with targets must have at least
 *    one history row (the stand-alone attention takes it without); a request
 *    with no targets is legal and produces nothing.
 *  - The caller owns every buffer.  The library never allocates, frees or
 *    synchronises: all work is enqueued on `stream`, and calls return before it
 *    runs.  Calls on different streams need distinct workspaces.
 *  - Errors found on the host are returned before anything is enqueued.
 *    Offsets are checked on the host when the *_host copies are given;
 *    otherwise the device scheduler checks them, produces no work for a bad
 *    request and records STCA_ERR_INVALID_ARG in the workspace, readable with
 *    stca_device_status().  No exception crosses the ABI.
 */
#ifndef STCA_H_
#define STCA_H_

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  STCA_OK = 0,
  STCA_ERR_INVALID_ARG = -1, /* bad pointer, size or offsets */
  STCA_ERR_UNSUPPORTED = -2, /* valid but not implemented shape/dtype/form */
  STCA_ERR_WORKSPACE = -3,   /* workspace or saved buffer too small */
  STCA_ERR_HIP = -4,         /* a HIP runtime call or launch failed */
  STCA_ERR_RANGE = -5        /* (device status only) an fp16 intermediate of the bf16 path
                                overflowed or a non-finite value appeared; see below */
} stca_status_t;

typedef enum { STCA_F32 = 0, STCA_BF16 = 1 } stca_dtype_t;

/* Execution forms of the bf16 MFMA path (0 = automatic everywhere).  The
 * generic fp32-arithmetic path has one form of each and ignores them.
 *
 * kv_form  STCA_KV_AUTO: each layer's K/V is projected inside the attention
 *          kernel and never stored, except when the host offsets show a
 *          request with more than 64 targets: then one GEMM writes every
 *          layer's K/V to the workspace once and the attention reads it once
 *          per 128 targets.  STCA_KV_FUSED: always the former.
 *          STCA_KV_MATERIALIZE: always the latter.
 * attn_form STCA_ATTN_AUTO: with d_h = 32 and host offsets, the requests
 *          with at most 32 / n_heads targets run in the reordered
 *          single-query form of App. A.2.2 (Eq. attn-optimized: scores
 *          u . x with u = q W_K^T, output (P X) W_V; no K/V) and the others
 *          in the standard form, in the same call; without host offsets the
 *          standard form.
 *          STCA_ATTN_STANDARD: always the standard form.
 *          STCA_ATTN_REORDERED: every request in the reordered form, for
 *          requests of up to 256 / n_heads targets (d_h = 32, host offsets
 *          given); STCA_ERR_UNSUPPORTED for other batches.
 * bwd_form STCA_BWD_AUTO: with d_h = 32, d_model in {64, 128, 256},
 *          ffn_hidden a multiple of d_model and host offsets showing at most
 *          32 targets per request, the backward on bf16 storage recomputes the
 *          forward with the history projected inside the attention kernel and
 *          then runs in the reordered form (the attention gradients through
 *          u = q W_K^T and h = da W_V^T per target and head, no K, V, dK or
 *          dV, in groups of 128 / n_heads targets; Sec. 3.1's reordering
 *          applied to the backward; d_model 128 or 256) or in the fused form
 *          (K/V formed inside the attention kernels, dK | dV written for the
 *          history-side products): reordered for histories balanced over the
 *          compute units with at most 128 / n_heads targets, else where an
 *          estimate of the two forms' kernels favours it.  Otherwise every
 *          layer's K | V are formed by a GEMM and the attention runs in exact
 *          fp32 both ways (generic).
 *          STCA_BWD_GENERIC: always the generic form.  STCA_BWD_FUSED: the
 *          fused form.  STCA_BWD_REORDERED: the reordered form with one
 *          target group per request (at most 128 / n_heads targets).  Each is
 *          STCA_ERR_UNSUPPORTED for a batch outside its conditions.
 * chunk_blocks: history chunk length, in 32-row blocks, of the attention's
 *          split over a request's history (at most 16 chunks per request, so
 *          long histories get longer chunks); 0 = chosen from the batch size
 *          and the number of compute units (then up to 64 chunks per request
 *          in a forward of few requests).
 * Out-of-range values are STCA_ERR_INVALID_ARG. */
typedef enum { STCA_KV_AUTO = 0, STCA_KV_FUSED = 1, STCA_KV_MATERIALIZE = 2 } stca_kv_form_t;
typedef enum { STCA_ATTN_AUTO = 0, STCA_ATTN_STANDARD = 1, STCA_ATTN_REORDERED = 2 } stca_attn_form_t;
typedef enum { STCA_BWD_AUTO = 0, STCA_BWD_FUSED = 1, STCA_BWD_GENERIC = 2, STCA_BWD_REORDERED = 3 } stca_bwd_form_t;

/* Model shape and execution forms.  d_model % n_heads == 0 and ffn_hidden a
 * multiple of 32.  STCA_BF16 with d_head = d_model / n_heads = 32, d_model in
 * {64, 128, 256} and ffn_hidden a multiple of 256 runs on the bf16 MFMA
 * kernels; every other shape with d_head in {8, 16, 32, 64} (either dtype)
 * runs on the generic fp32-arithmetic kernels (stca_path tells which).
 * Every size and launch decision depends only on this structure and the
 * batch, so a workspace sized for a (dims, batch) pair fits every call with
 * the same pair.  Zero-initialise the structure to get the automatic forms. */
typedef struct {
  int32_t d_model;
  int32_t n_heads;
  int32_t n_layers;
  int32_t ffn_hidden;
  int32_t dtype;        /* stca_dtype_t */
  int32_t kv_form;      /* stca_kv_form_t */
  int32_t attn_form;    /* stca_attn_form_t */
  int32_t bwd_form;     /* stca_bwd_form_t */
  int32_t chunk_blocks; /* >= 0 */
} stca_dims_t;

/* A packed ragged batch (App. A.4: flattened rows plus segment boundaries). */
typedef struct {
  int32_t n_requests;           /* R >= 1 */
  int64_t n_hist;               /* total history rows, < 2^31 */
  int64_t n_tgt;                /* total target rows, < 2^31 */
  const int32_t* hist_off;      /* device [R+1] */
  const int32_t* tgt_off;       /* device [R+1] */
  const int32_t* hist_off_host; /* optional host copy [R+1]: enables host checks and exact sizing */
  const int32_t* tgt_off_host;  /* optional host copy [R+1] */
} stca_batch_t;

/* Per-layer weights (paper Sec. 3.1: W_Q, W_K, W_V, W_O; the FFN W_1, W_2). */
typedef struct {
  const void* wq;
  const void* wk;
  const void* wv;
  const void* wo;
  const void* w1;
  const void* w2;
} stca_weights_t;

/* Weight gradients, fp32, same shapes as the weights; overwritten. */
typedef struct {
  float* dwq;
  float* dwk;
  float* dwv;
  float* dwo;
  float* dw1;
  float* dw2;
} stca_wgrads_t;

/* Byte offsets into the `saved` buffer (all fp32 unless stated), for reading
 * per-layer intermediates back.  Each per-layer tensor is stacked on a leading
 * layer axis: s [n][n_tgt][d] (layer input state), a [n][n_tgt][d] (head
 * concatenation before W_O), u [n][n_tgt][d] (state after the attention
 * residual), lse [n][n_tgt][h] (natural log-sum-exp of each head's scores). */
typedef struct {
  size_t s, a, u, lse;
  size_t total;
} stca_saved_layout_t;

/* Workspace bytes needed by stca_forward (with_backward = 0) or stca_backward
 * (with_backward = 1).  Returns 0 for invalid or unsupported arguments. */
size_t stca_workspace_size(const stca_dims_t* dims, const stca_batch_t* batch, int with_backward);

/* Bytes of the optional `saved` buffer that stca_forward fills. */
size_t stca_saved_size(const stca_dims_t* dims, const stca_batch_t* batch);

/* Offsets of the saved tensors; returns STCA_ERR_INVALID_ARG / UNSUPPORTED
 * like the other calls. */
stca_status_t stca_saved_layout(const stca_dims_t* dims, const stca_batch_t* batch,
                                stca_saved_layout_t* layout);

/* Forward pass: out[n_tgt][d] (storage dtype) = s^(n) for every target.
 *  hist  [n_hist][d], tgt [n_tgt][d]  storage dtype, device
 *  saved nullable; when given (stca_saved_size bytes) the per-layer
 *        intermediates (see stca_saved_layout_t) are written there
 *  ws    device workspace of ws_bytes >= stca_workspace_size(dims, batch, 0)
 * The bf16 MFMA path's forms of K/V and of the attention follow
 * dims->kv_form and dims->attn_form. */
stca_status_t stca_forward(const stca_dims_t* dims, const stca_batch_t* batch,
                           const void* hist, const void* tgt, const stca_weights_t* w,
                           void* out, void* saved, void* ws, size_t ws_bytes,
                           hipStream_t stream);

/* Backward pass: the gradients of f = sum_t <dout_t, out_t> with respect to
 * hist, tgt and every weight, for the same inputs as a forward call.  The
 * layer states are recomputed from the inputs in fp32 (activation
 * recomputation), so every ReLU gate and softmax weight of the backward
 * follows fp32 states.  Writes (overwrites) dhist [n_hist][d], dtgt [n_tgt][d]
 * and all weight gradients, fp32.  dout is [n_tgt][d] in the storage dtype.
 * ws_bytes >= stca_workspace_size(dims, batch, 1). */
stca_status_t stca_backward(const stca_dims_t* dims, const stca_batch_t* batch,
                            const void* hist, const void* tgt, const stca_weights_t* w,
                            const void* dout, float* dhist, float* dtgt,
                            const stca_wgrads_t* dw, void* ws, size_t ws_bytes,
                            hipStream_t stream);

/* Forward without a workspace argument, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid allocation).  The same computation and results as
 * stca_forward, with the workspace in a device array of the library of
 * STCA_NOALLOC_SCRATCH_BYTES bytes, one per GPU, set up on the first call on
 * that GPU (with it current) and held until the process ends; nothing is
 * allocated by any call.  Returns STCA_ERR_WORKSPACE, before anything is
 * launched, when stca_workspace_size(dims, batch, 0) exceeds that size; other
 * errors as stca_forward.  Every call on a GPU uses that GPU's one array:
 * calls that may overlap on the same GPU (other streams, other threads) race
 * and must be serialised by the caller.  Nothing in the array needs to start
 * at zero; the device-side status of such a call (stca_device_status) is not
 * readable, so give host offsets to have them checked. */
#define STCA_NOALLOC_SCRATCH_BYTES ((size_t)256 << 20)
stca_status_t stca_forward_noalloc(const stca_dims_t* dims, const stca_batch_t* batch, const void* hist,
                                   const void* tgt, const stca_weights_t* w, void* out, void* saved,
                                   hipStream_t stream);

/* Training step in two calls, for batches the fused backward takes (bf16,
 * d_h = 32, FFN width a multiple of d, host offsets showing at most 32
 * targets per request): the forward writes, besides out, a training record
 * of the per-layer tensors the backward needs, computed to fp32 accuracy (so
 * the ReLU gates follow fp32 states), and the backward reads it instead of
 * recomputing them.
 *
 * stca_train_record_size: bytes of the record; 0 when the batch does not
 * qualify or the arguments are invalid.
 * stca_forward_train: out as stca_forward (evaluated to fp32 accuracy before
 * the final rounding to the storage dtype); record (device, 16-byte aligned,
 * stca_train_record_size bytes) is overwritten; ws as for stca_backward
 * (ws_bytes >= stca_workspace_size(dims, batch, 1)).
 * stca_backward_record: the same gradients as stca_backward for the inputs
 * that produced `record` (which must not change in between), without the
 * recomputation.  Both return STCA_ERR_UNSUPPORTED for batches that do not
 * qualify; other errors as stca_forward / stca_backward. */
size_t stca_train_record_size(const stca_dims_t* dims, const stca_batch_t* batch);
stca_status_t stca_forward_train(const stca_dims_t* dims, const stca_batch_t* batch,
                                 const void* hist, const void* tgt, const stca_weights_t* w,
                                 void* out, void* record, void* ws, size_t ws_bytes, hipStream_t stream);
stca_status_t stca_backward_record(const stca_dims_t* dims, const stca_batch_t* batch,
                                   const void* hist, const void* tgt, const stca_weights_t* w,
                                   const void* record, const void* dout, float* dhist, float* dtgt,
                                   const stca_wgrads_t* dw, void* ws, size_t ws_bytes,
                                   hipStream_t stream);

/* Measurement variant of stca_forward: the same work, plus hipEventRecord on
 * `stream` around every kernel launch so a caller can time each kernel on the
 * stream it runs on.  events[0] is recorded before the first launch and
 * events[k+1] right after launch k; n_events must be at least
 * stca_forward_launch_count(dims, batch) + 1.  labels (nullable, n_events - 1
 * entries) receive static kernel names ("proj", "attn", "update", ...).  The
 * count has a place for every kernel that a batch may need; one whose work
 * runs inside another launch ("setup": schedules and weight repacking;
 * "attn_mixed": the attention of a batch of several widths or forms) has the
 * label "none" and no duration.
 * The events must have been created by the caller (hipEventCreate). */
int stca_forward_launch_count(const stca_dims_t* dims, const stca_batch_t* batch);
stca_status_t stca_forward_profiled(const stca_dims_t* dims, const stca_batch_t* batch,
                                    const void* hist, const void* tgt, const stca_weights_t* w,
                                    void* out, void* saved, void* ws, size_t ws_bytes,
                                    hipStream_t stream, hipEvent_t* events, int n_events,
                                    const char** labels);

/* Measurement variant of stca_backward: the same work, plus hipEventRecord on
 * `stream` at phase boundaries.  events[0] is recorded before the first
 * launch and events[k+1] at the end of phase k; labels (nullable) receive the
 * phase names ("sched", "prep", "kv_gemm", "attn_fwd", "target_gemm",
 * "attn_bwd", "dw_kv", "dx", "out").  n_events must be at least
 * stca_backward_launch_count(dims, batch) + 1; the events are the caller's. */
int stca_backward_launch_count(const stca_dims_t* dims, const stca_batch_t* batch);
stca_status_t stca_backward_profiled(const stca_dims_t* dims, const stca_batch_t* batch,
                                     const void* hist, const void* tgt, const stca_weights_t* w,
                                     const void* dout, float* dhist, float* dtgt,
                                     const stca_wgrads_t* dw, void* ws, size_t ws_bytes,
                                     hipStream_t stream, hipEvent_t* events, int n_events,
                                     const char** labels);

/* ---- Stochastic-length training batches (Sec. 3.3; App. "Extrapolation
 * details": Beta sampling, Eq. beta-scale and Eq. beta; batch-level load
 * balancing).  Host functions on host arrays; no GPU involved.
 *
 * stca_sl_beta: the Beta shape beta that makes E[L_raw] = l_avg (Eq. beta):
 * alpha (l_max - l_avg) / (l_avg - l_min).  NaN unless alpha > 0 and
 * 0 <= l_min < l_avg < l_max.
 *
 * stca_sl_sample: per request r, s ~ Beta(alpha, beta) from a counter-based
 * stream keyed by (seed, r), L_raw = l_min + s (l_max - l_min) (written to
 * l_raw[r] when l_raw is not NULL), and l_train[r] = L_raw rounded to the
 * nearest multiple of 8, clamped to [max(8, l_min rounded), l_max].
 *
 * stca_sl_allocate: global length allocation under a token budget (the paper
 * uses B * l_avg): l_keep[r] = min(l_full[r], l_train[r]); if their sum
 * exceeds `budget`, every l_keep is capped at the largest multiple of 8 that
 * brings the sum within it (at least 8).
 *
 * stca_sl_pack: sequence compaction with temporal-suffix selection.  full_off
 * [n+1] segments the full histories; request r keeps its last l_keep[r] rows.
 * Writes hist_off [n+1] of the packed layout and, when src_rows is not NULL,
 * src_rows [hist_off[n]]: the full-history row each packed row comes from.
 *
 * All return STCA_ERR_INVALID_ARG on inconsistent arguments. */
double stca_sl_beta(double alpha, int32_t l_min, int32_t l_avg, int32_t l_max);
stca_status_t stca_sl_sample(uint64_t seed, int32_t n, double alpha, int32_t l_min, int32_t l_avg,
                             int32_t l_max, double* l_raw, int32_t* l_train);
stca_status_t stca_sl_allocate(int32_t n, const int32_t* l_full, const int32_t* l_train, int64_t budget,
                               int32_t* l_keep);
stca_status_t stca_sl_pack(int32_t n, const int32_t* full_off, const int32_t* l_keep, int32_t* hist_off,
                           int32_t* src_rows);

/* ---- Paper-exact layer stack (Sec. 3.1, "Input encoding", "Multi-head
 * target-to-history cross attention", "Stacking and target-conditioned
 * fusion", "Prediction head and objective").  With M = n_layers, F =
 * ffn_hidden (= r d, the SwiGLU width) and SwiGLUFFN(x) = ((x W_u) *
 * (x W_v * sigmoid(x W_v))) W_o (Eq. swigluffn, no biases):
 *   X~^(i)    = LN(SwiGLUFFN^(i)(X))                          every history row, i = 1..M
 *   q^(1)     = LN(SwiGLUFFN^(1)(x_t))
 *   o^(i)     = [heads of the cross attention of q^(i) onto X~^(i)] W_O^(i)   (Eq. layer-output)
 *   q^(i+1)   = LN(SwiGLUFFN^(i+1)([o^(1) || ... || o^(i) || x_t] W_C^(i+1)))  (Eq. fuse)
 *   z         = SwiGLUFFN_z([o^(1) || ... || o^(M) || x_t] W_Z)
 * LN normalises each row over its d features (biased variance, eps 1e-5,
 * unit scale, zero shift).  SwiGLUFFN^(i) is one block per layer, used for
 * both the history and the query input of layer i.  The attention heads,
 * scale and per-request sharing are those of stca_forward.
 *
 * Weights (storage dtype, row-major, y = x W):
 *   ffn_u, ffn_v [M][d][F], ffn_o [M][F][d]   SwiGLUFFN^(1..M)
 *   wq, wk, wv, wo [M][d][d]
 *   wc   W_C^(2), ..., W_C^(M) one after the other, W_C^(k) being k d rows
 *        x d (rows in concatenation order, x_t's block last); NULL when M = 1
 *   wz   [(M+1) d][d]
 *   z_u, z_v [d][F], z_o [F][d]              the head's SwiGLU block
 * Shapes: as stca_forward (stca_path tells the kernel family); on the bf16
 * MFMA path the history transform runs as one fused SwiGLU + LayerNorm kernel
 * per layer (the hidden activations never leave the registers) and the
 * transformed history is stored in bf16 for the attention; the generic path
 * keeps everything in fp32.  The target-side blocks run on fp32 arithmetic. */
typedef struct {
  const void* ffn_u;
  const void* ffn_v;
  const void* ffn_o;
  const void* wq;
  const void* wk;
  const void* wv;
  const void* wo;
  const void* wc;
  const void* wz;
  const void* z_u;
  const void* z_v;
  const void* z_o;
} stca_paper_weights_t;

/* Byte offsets into the optional `saved` buffer of stca_forward_paper, fp32:
 * q [M][n_tgt][d] (the layer queries q^(i)), a [M][n_tgt][d] (head
 * concatenation before W_O), o [n_tgt][M d] (row t = o^(1) || ... || o^(M)),
 * lse [M][n_tgt][h] (natural log-sum-exp of each head's scores) and xt
 * [M][n_hist][d] (the transformed histories X~^(i)). */
typedef struct {
  size_t q, a, o, lse, xt;
  size_t total;
} stca_paper_saved_layout_t;

size_t stca_paper_workspace_size(const stca_dims_t* dims, const stca_batch_t* batch);
size_t stca_paper_saved_size(const stca_dims_t* dims, const stca_batch_t* batch);
stca_status_t stca_paper_saved_layout(const stca_dims_t* dims, const stca_batch_t* batch,
                                      stca_paper_saved_layout_t* layout);

/* Forward pass of the paper-exact stack: z [n_tgt][d] (storage dtype) for
 * every target.  hist, tgt, z, saved and ws as in stca_forward, with
 * ws_bytes >= stca_paper_workspace_size(dims, batch) and saved (nullable)
 * of stca_paper_saved_size bytes.  Errors as for stca_forward. */
stca_status_t stca_forward_paper(const stca_dims_t* dims, const stca_batch_t* batch,
                                 const void* hist, const void* tgt, const stca_paper_weights_t* w,
                                 void* z, void* saved, void* ws, size_t ws_bytes, hipStream_t stream);

/* Measurement variant of stca_forward_paper (events and labels as in
 * stca_forward_profiled; n_events >= stca_paper_launch_count + 1). */
int stca_paper_launch_count(const stca_dims_t* dims, const stca_batch_t* batch);
stca_status_t stca_forward_paper_profiled(const stca_dims_t* dims, const stca_batch_t* batch,
                                          const void* hist, const void* tgt, const stca_paper_weights_t* w,
                                          void* z, void* saved, void* ws, size_t ws_bytes, hipStream_t stream,
                                          hipEvent_t* events, int n_events, const char** labels);

/* ---- Stand-alone attention (the operator without the layer around it):
 * ragged target-to-history cross attention with capped scores, a learned bias
 * by buckets of distance and a mask to the part of the history that a target
 * may see, and its gradients.  For target t, query head h of kv head
 * g = h / (n_heads / n_kv_heads) and history row j of t's request:
 *   z = scale q_{t,h} . k_{j,g}
 *   y = softcap tanh(z / softcap)                  (softcap > 0; y = z for 0)
 *   x = y + bias[h][b(D)],  D = tgt_pos[t] - hist_pos[j]
 *   out_{t,h} = sum_j softmax_j(x) v_{j,g}          over the visible rows j
 * b(D) is the number of edges that are at most max(D, 0); a row is hidden when
 * `masked` and D < 0, or when its bucket's bias is minus infinity.  Hidden rows
 * contribute nothing, whatever their K and V hold; a target that sees no row
 * (its request may have none) has the output 0, and no part in any gradient.
 * D saturates at the ends of int32.  Sums, maxima and weights are fp32; with
 * bf16 storage the weights enter the matrix cores as two bf16 terms, the second
 * rounded (2^-16 of a weight), and as three, an fp32 whole, in a forward that
 * saves: its output may differ in the last bit from one that does not.  A call
 * repeats bitwise; how a request's sums are divided, and so their last bits,
 * depends on the whole batch.  Any finite V whose weighted mean is finite may
 * be given.
 *
 * Calls of one batch on different streams need distinct workspaces.  Targets
 * of a request without history are legal here.  Offsets are checked on the
 * device too: a request of more rows, or in the backward targets, than a call
 * planned on the host copies takes is STCA_ERR_INVALID_ARG there, its results are
 * undefined, and nothing is written outside the buffers. */
typedef struct {
  int32_t n_heads;           /* query heads, a multiple of n_kv_heads (at most 64 times as many) */
  int32_t n_kv_heads;        /* heads of K and V, each shared by n_heads / n_kv_heads query heads */
  int32_t d_head;            /* 32, 64 or 128; n_heads d_head at most 65536 */
  int32_t dtype;             /* stca_dtype_t of q, k, v, out, dout, dq, dk, dv */
  float scale;               /* finite, times log2 e as well */
  float softcap;             /* >= 0, 0 = none; likewise, and scale / softcap 0 or in fp32's normal range */
  int32_t masked;            /* nonzero: rows with hist_pos > tgt_pos are hidden */
  int32_t n_buckets;         /* 0 = no bias; at most 128 */
  const int32_t* edges_host; /* host [n_buckets - 1], strictly ascending in 1..2^31-2; read by the call */
} stca_attn_t;

/* Positions and tables of bias, and a cache's pos, need 4-byte alignment only.
 * Rows of q, k, v hold their heads one after the other; ld* are row strides in
 * elements (0 = dense; a multiple of 16 bytes, below 16 MB).  tgt_pos is needed with a mask
 * or a bias; hist_pos NULL: a row's position is its index in its request. */
typedef struct {
  const void* q;            /* [n_tgt][n_heads][d_head] */
  const void* k;            /* [n_hist][n_kv_heads][d_head] */
  const void* v;            /* [n_hist][n_kv_heads][d_head] */
  int64_t ldq, ldk, ldv;
  const int32_t* tgt_pos;   /* device [n_tgt] */
  const int32_t* hist_pos;  /* device [n_hist], any order */
  const float* bias;        /* device [n_heads][n_buckets], fp32 */
} stca_attn_in_t;

typedef struct {
  void* dq;      /* shapes and strides as q, k, v, storage dtype; overwritten */
  void* dk;
  void* dv;
  int64_t lddq, lddk, lddv;
  float* dbias;  /* [n_heads][n_buckets], fp32, overwritten; NULL without a bias */
} stca_attn_grads_t;

/* Byte offsets into the buffer that a forward saves for its backward, fp32:
 * a [n_tgt][n_heads][d_head] (the output before rounding), and per target and
 * head a score max near the largest (8 below to 40 above), in units of log2 e, and the sum of
 * 2^(x log2 e - max) [n_tgt][n_heads]. */
typedef struct {
  size_t a, max, sum;
  size_t total;
} stca_attn_saved_layout_t;

/* Sizes; 0 for invalid or unsupported arguments. */
size_t stca_attn_workspace_size(const stca_attn_t* attn, const stca_batch_t* batch, int with_backward);
size_t stca_attn_saved_size(const stca_attn_t* attn, const stca_batch_t* batch);
stca_status_t stca_attn_saved_layout(const stca_attn_t* attn, const stca_batch_t* batch,
                                     stca_attn_saved_layout_t* layout);

/* out [n_tgt][n_heads][d_head] (dense, storage dtype); saved nullable. */
stca_status_t stca_attn_forward(const stca_attn_t* attn, const stca_batch_t* batch, const stca_attn_in_t* in,
                                void* out, void* saved, void* ws, size_t ws_bytes, hipStream_t stream);

/* Gradients of f = sum <dout, out>, from the inputs of a forward and what it
 * saved.  dout as out.  Gradients of shared heads are summed over the sharing
 * heads; nothing is added in order of arrival, so results repeat bitwise.
 * ws_bytes >= stca_attn_workspace_size(attn, batch, 1). */
stca_status_t stca_attn_backward(const stca_attn_t* attn, const stca_batch_t* batch, const stca_attn_in_t* in,
                                 const void* saved, const void* dout, const stca_attn_grads_t* grads, void* ws,
                                 size_t ws_bytes, hipStream_t stream);

/* Bucket edges as distances grow: 1, 2, ..., n_exact, then a geometric series
 * to max_distance (each at least one more than the last), n_buckets - 1 in all.
 * Host function.  1 <= n_exact < n_buckets <= 128,
 * n_buckets <= max_distance < 2^31 - 1. */
stca_status_t stca_bias_edges(int32_t n_buckets, int32_t n_exact, int32_t max_distance, int32_t* edges);

/* ---- Paged history cache.  K and V of a history row do not depend on the
 * targets, so they can be kept from one request of a user to the next.  Rows
 * live in pages of page_size slots; a request's table lists its pages, and its
 * row i is slot i % page_size of page table[i / page_size].
 *   k [n_pages][n_kv_heads][page_size][d_head]
 *   v [n_pages][n_kv_heads][d_head][page_size]
 * in bf16 (STCA_CACHE_BF16), or as int8 with a power-of-two step per row and kv
 * head (STCA_CACHE_INT8): step = 2^max(floor(log2 max|x|) - 6, -126),
 * n = x / step rounded to nearest even, at most 127 in magnitude, and
 * k_exp, v_exp [n_pages][n_kv_heads][page_size] hold log2(step) + 127.  A row
 * with a value that is not finite is stored as 255 and reads as NaN.
 * pos (optional) [n_pages][page_size]: the rows' positions. */
typedef enum { STCA_CACHE_BF16 = 0, STCA_CACHE_INT8 = 1 } stca_cache_format_t;
typedef struct {
  int32_t n_pages;
  int32_t page_size;   /* 16, 32, 64, 128 or 256 */
  int32_t n_kv_heads;
  int32_t d_head;      /* 32, 64 or 128 */
  int32_t format;      /* stca_cache_format_t */
  void* k;
  void* v;
  uint8_t* k_exp;      /* STCA_CACHE_INT8 only */
  uint8_t* v_exp;
  int32_t* pos;        /* nullable */
} stca_cache_t;

/* Packed rows of several requests and where they lie in the cache: request r's
 * rows [row_off[r], row_off[r+1]) are its cache rows start[r], start[r] + 1, ... */
typedef struct {
  int32_t n_requests;
  int64_t n_rows;          /* row_off[n_requests] */
  const int32_t* row_off;  /* device [n_requests + 1] */
  const int32_t* start;    /* device [n_requests] */
  const int32_t* table;    /* device [n_requests][table_ld] */
  int32_t table_ld;
} stca_cache_rows_t;

/* Writes rows k, v [n_rows][n_kv_heads][d_head] (dtype; row strides ldk, ldv,
 * 0 = dense) into their slots, and pos [n_rows] where both it and the cache's
 * are given.  Other slots keep what they hold.  A slot may be written once per
 * call.  The read is the reverse, rounded to dtype.  Rows without a page (an
 * entry of the table outside the pages) are left out.  ws (nullable): 256 device
 * bytes whose status stca_device_status reads: STCA_ERR_INVALID_ARG for bad
 * offsets, starts or pages. */
#define STCA_CACHE_WS_BYTES ((size_t)256)
stca_status_t stca_cache_write(const stca_cache_t* cache, const stca_cache_rows_t* rows, int32_t dtype,
                               const void* k, const void* v, int64_t ldk, int64_t ldv, const int32_t* pos,
                               void* ws, hipStream_t stream);
stca_status_t stca_cache_read(const stca_cache_t* cache, const stca_cache_rows_t* rows, int32_t dtype, void* k,
                              void* v, int64_t ldk, int64_t ldv, int32_t* pos, void* ws, hipStream_t stream);

/* Attention of the requests' new targets over their first lens[r] cached rows,
 * otherwise as stca_attn_forward (positions from the cache's pos, or row
 * indices; attn->dtype must be STCA_BF16).  lens may change between calls up to
 * max_len, on which sizes and launches depend.  Rows without a page are hidden.
 * Offsets, lengths and pages are checked on the device (stca_device_status). */
typedef struct {
  int32_t n_requests;
  int64_t n_tgt;
  const int32_t* tgt_off;       /* device [n_requests + 1] */
  const int32_t* tgt_off_host;  /* optional host copy: host checks and exact sizing */
  const int32_t* lens;          /* device [n_requests], 0..max_len */
  int32_t max_len;
  const int32_t* table;         /* device [n_requests][table_ld], table_ld page_size >= max_len */
  int32_t table_ld;
} stca_cache_batch_t;
size_t stca_cache_attn_workspace_size(const stca_attn_t* attn, const stca_cache_t* cache,
                                      const stca_cache_batch_t* batch);
stca_status_t stca_cache_attn(const stca_attn_t* attn, const stca_cache_t* cache, const stca_cache_batch_t* batch,
                              const void* q, int64_t ldq, const int32_t* tgt_pos, const float* bias, void* out,
                              void* ws, size_t ws_bytes, hipStream_t stream);

/* ---- Rows from ids, and the gradient of their tables.  What stands before the
 * layers (Sec. 3.1, "Input encoding": a history row is fused from several looked-up
 * embeddings) and behind their backward (dhist, dtgt):
 *   out_i = scale sum_f table_f[ids_f[i]]       sums in fp32, fields in order, one rounding
 * A negative id is no row and adds nothing.  An id behind its table is taken for
 * none as well, and sets the status in ws (nullable; 256 device bytes, cleared by
 * the caller: a lookup only sets it, so that several may share it). */
typedef struct {
  int32_t d;            /* features of a row: a multiple of 8, at most 8192 */
  int32_t table_dtype;  /* stca_dtype_t of the tables */
  int32_t out_dtype;    /* ... of out */
  float scale;          /* finite */
} stca_embed_t;
typedef struct {
  const void* table;    /* [n_rows][d] */
  int64_t n_rows;       /* at least 1, below 2^31 - 2^16 */
  int64_t ld;           /* row strides in elements as in stca_attn_in_t (0 = dense) */
  const int32_t* ids;   /* device [n] */
} stca_embed_field_t;
#define STCA_EMBED_FIELDS 8 /* most fields of a call */
stca_status_t stca_embed_forward(const stca_embed_t* embed, const stca_embed_field_t* fields, int32_t n_fields,
                                 int64_t n, void* out, int64_t ldo, void* ws, hipStream_t stream);

/* The gradient of one table, fp32, from up to four parts that look it up (a
 * request's history and targets share the item table):
 *   dT[v] = scale sum over the parts' rows i with ids[i] = v of dout_i
 * The rows of an id are added in the order of the parts and of their rows,
 * grouped by their place among all sorted ids; nothing is added in order of
 * arrival, so a call repeats bitwise.  n below is the rows of all parts together.
 *   dense   dtable [n_rows][d] (row stride ld), overwritten, or added to where
 *           accumulate is nonzero (rows without an id keep what they hold)
 *   sparse  rows [min(n, n_rows)]: the distinct ids in ascending order, grads
 *           [min(n, n_rows)][d]: their gradients, count [1]: their number; what
 *           lies behind it is left as it was
 * ws_bytes >= stca_embed_grad_workspace_size(grad, n) (0 for invalid or unsupported
 * arguments); an id behind the table sets stca_device_status. */
typedef struct {
  int32_t d;            /* a multiple of 8, at most 8192 */
  int32_t dtype;        /* of dout */
  int64_t n_rows;
  float scale;
} stca_embed_grad_t;
typedef struct {
  const int32_t* ids;   /* device [n] */
  const void* dout;     /* [n][d] */
  int64_t ld;
  int64_t n;
} stca_embed_part_t;
#define STCA_EMBED_PARTS 4
size_t stca_embed_grad_workspace_size(const stca_embed_grad_t* grad, int64_t n);
stca_status_t stca_embed_grad_dense(const stca_embed_grad_t* grad, const stca_embed_part_t* parts, int32_t n_parts,
                                    float* dtable, int64_t ld, int accumulate, void* ws, size_t ws_bytes,
                                    hipStream_t stream);
stca_status_t stca_embed_grad_sparse(const stca_embed_grad_t* grad, const stca_embed_part_t* parts, int32_t n_parts,
                                     int32_t* rows, float* grads, int32_t* count, void* ws, size_t ws_bytes,
                                     hipStream_t stream);

/* ---- Norms before and after a block, its gate and its residual scale, for
 * models that put their own blocks around the stand-alone attention.  For row i
 * of x (the residual stream), block (what the block gave) and gate:
 *   t = post(block) act(gate)      post: a norm with weight and bias, or nothing; act: sigmoid, silu or 1
 *   h = x + scale layer_scale t    layer_scale [d], or 1
 *   y = pre(h)                     the norm in front of the next block, or nothing
 * norm(v) = weight (v - mean) / sqrt(var + eps) + bias (STCA_NORM_LAYER, biased
 * variance), or weight v / sqrt(mean(v^2) + eps) + bias (STCA_NORM_RMS).  Weights
 * and biases are fp32 [d], 4-byte aligned; NULL for ones and zeros.  Without a block
 * h is x and y its norm.  Everything between the inputs and the outputs is fp32 and
 * unrounded (y is the norm of h before its rounding).  Rows may have any finite
 * values: squares that leave fp32 are taken smaller.  h and y may lie on x, block
 * or gate, dx, dblock and dgate on those or on dh and dy, with the same stride. */
typedef enum { STCA_NORM_RMS = 0, STCA_NORM_LAYER = 1 } stca_norm_kind_t;
typedef enum { STCA_GATE_NONE = 0, STCA_GATE_SIGMOID = 1, STCA_GATE_SILU = 2 } stca_gate_t;
typedef struct {
  int32_t d;            /* a multiple of 8, at most 4096 */
  int32_t dtype;        /* of rows and their gradients */
  int32_t kind;         /* stca_norm_kind_t */
  int32_t gate;         /* stca_gate_t; needs a block */
  int32_t post;         /* nonzero: the block's rows are normed; needs a block */
  int32_t pre;          /* nonzero: y is wanted; 0 needs a block */
  float scale;          /* finite */
  float eps;            /* finite, at least 1e-20 */
} stca_norm_t;
typedef struct {
  const void* x;        /* [n][d] */
  const void* block;    /* [n][d], nullable */
  const void* gate;     /* [n][d], with a gate */
  int64_t ldx, ldblock, ldgate;
  const float* pre_w;
  const float* pre_b;
  const float* post_w;
  const float* post_b;
  const float* layer_scale;
} stca_norm_in_t;
/* Of f = sum <dh, h> + sum <dy, y>.  A NULL gradient is not computed.  The five of
 * [d] are fp32 sums over the rows, joined in a fixed order. */
typedef struct {
  void* dx;
  void* dblock;
  void* dgate;
  int64_t lddx, lddblock, lddgate;
  float* dpre_w;
  float* dpre_b;
  float* dpost_w;
  float* dpost_b;
  float* dlayer_scale;
} stca_norm_grads_t;
/* h [n][d] (NULL without a block), y [n][d] (NULL without pre). */
stca_status_t stca_norm_forward(const stca_norm_t* norm, const stca_norm_in_t* in, int64_t n, void* h, int64_t ldh,
                                void* y, int64_t ldy, hipStream_t stream);
/* dh nullable with pre (h is not used but for y); dy with pre.  Nothing is saved
 * by a forward: the inputs are enough. */
size_t stca_norm_workspace_size(const stca_norm_t* norm, int64_t n);
stca_status_t stca_norm_backward(const stca_norm_t* norm, const stca_norm_in_t* in, int64_t n, const void* dh,
                                 int64_t lddh, const void* dy, int64_t lddy, const stca_norm_grads_t* grads, void* ws,
                                 size_t ws_bytes, hipStream_t stream);

/* ---- The norm of many gradients together, and clipping:
 *   norm = sqrt(sum over all elements g^2);  out = g min(1, max_norm / norm)
 * Squares are added, and the factor is applied, in fp64: any finite gradient has
 * its norm (written as fp32).  A norm that is not finite scales nothing: out = g,
 * and the caller sees it.  A sparse gradient counts as far as *count rows of `row`
 * elements; what lies behind is neither read nor written.  A result may lie on its
 * own gradient (same type), and on nothing else of the list; the same result twice
 * is refused. */
typedef struct {
  const void* g;          /* n elements, dense, aligned to an element */
  void* out;              /* NULL: the gradient only counts */
  int64_t n;              /* at most 2^40 */
  int32_t dtype;
  int32_t out_dtype;
  const int32_t* count;   /* device [1], nullable: rows in use (0..n / row) */
  int32_t row;            /* elements of a row, which divide n; with a count */
} stca_grad_t;
size_t stca_clip_workspace_size(int32_t n_grads);
/* max_norm > 0; infinity only measures and copies.  norm: device [1], nullable. */
stca_status_t stca_clip(const stca_grad_t* grads, int32_t n_grads, double max_norm, float* norm, void* ws,
                        size_t ws_bytes, hipStream_t stream);

/* Reads (synchronising on `stream`) the status the kernels recorded in `ws`
 * during the last call that used it: STCA_ERR_INVALID_ARG when the device
 * scheduler found bad offsets, else STCA_ERR_RANGE when the forward's target
 * update found an fp16 intermediate out of range or a non-finite attention
 * output (bf16 path, see "Range of the bf16 path"), else STCA_OK. */
stca_status_t stca_device_status(const void* ws, hipStream_t stream);

/* Static description of a status code. */
const char* stca_status_string(stca_status_t status);

/* Which kernel family a shape runs on: 1 = bf16 MFMA path, 0 = generic fp32
 * path, negative = a status code for invalid or unsupported dims. */
int stca_path(const stca_dims_t* dims);

#ifdef __cplusplus
}
#endif

#endif /* STCA_H_ */
