/*
 * sdp_ops.h -- C ABI of libsdp, the training operators beside the update.
 *
 * The update of sdp.h takes the BF16 gradients of R data-parallel ranks; the
 * operators here are where a training step of the paper's models makes such
 * gradients (the paper trains dense Qwen3 and mixture-of-experts models under
 * one data-parallel runtime: Evaluation, setup; MoE and correctness):
 *   sdp_qk_norm_rope       RMS norm of each query and key head, then the
 *                          position rotation; and its backward
 *   sdp_grouped_matmul     rows sorted by expert times that expert's weight;
 *                          and its backward
 *   sdp_distill_loss       loss of each row of logits against a teacher's top
 *                          logits and a label; and its backward
 * A weight gradient may be written as BF16 straight into a rank's gradient
 * buffer of an sdp_segment.
 *
 * Conventions (those of sdp.h, and):
 *  - All buffers are device memory of the context's GPU, owned by the caller.
 *    A pointer is aligned to its element; it need not be 16-byte aligned, but
 *    tensors whose rows are 16-byte aligned are read faster.
 *  - Strides count elements.  The last dimension is contiguous.  An input may
 *    have strides of 0 (a broadcast); an output may not overlap itself.
 *  - An output may overlap an input or another output only where a call says
 *    so; other overlaps are refused.
 *  - Every call is asynchronous on `stream`.  Calls that use the context's
 *    workspace (sdp_qk_norm_rope_backward with weight gradients,
 *    sdp_distill_loss except where rows stay in registers, gradients of few
 *    experts' weights, large grouped products of sizes or strides without whole
 *    16-byte pieces) order themselves after the context's last such call, whatever
 *    its stream; a workspace that has to grow waits for the device.  It stays as
 *    large as its largest call needed until the context is destroyed.
 *  - A call that uses no workspace may be captured into a HIP graph: the norm and
 *    rotation, their backward without weight gradients, sdp_distill_loss_backward,
 *    sdp_distill_loss with dlogits where rows stay in registers (192 or more, of at
 *    most 311,311 bytes each), grouped products of whole 16-byte pieces other than
 *    gradients of few weights.  One that uses it is refused on a capturing stream:
 *    the graph would keep the workspace's address past the context's next larger
 *    call.
 *  - Sums, norms, softmax statistics and products are held in FP32 and an
 *    output is rounded once, to nearest even.  No atomics: the same inputs
 *    give the same bits.
 *  - Sizes of zero are valid: an output that has elements is still written.
 *  - Values in device memory that are out of range (a position past the
 *    table, a teacher's index or a label past the vocabulary) are never used
 *    as an address; the results that depend on them are NaN.
 */
#ifndef SDP_OPS_H
#define SDP_OPS_H

#include "sdp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- element types ------------------------------------------------------- */
#define SDP_TYPE_F32 0
#define SDP_TYPE_BF16 1
#define SDP_TYPE_I32 2
#define SDP_TYPE_I64 3

/* ---- limits -------------------------------------------------------------- */
#define SDP_QK_MAX_HEAD_DIM 1024
#define SDP_QK_MAX_HEADS 16384
#define SDP_DISTILL_MAX_K 1024
#define SDP_DISTILL_MAX_ROWS 4000000
#define SDP_GROUPED_MAX_GROUPS 2048

/* ---- norms of queries and keys with the position rotation ----------------- */

/* A [batch, tokens, heads, head_dim] tensor: element (b, s, h, i) is
 * data[b * batch_stride + s * token_stride + h * head_stride + i]. */
typedef struct {
    void *data;
    int64_t batch_stride, token_stride, head_stride;
} sdp_heads;

/* type: SDP_TYPE_BF16 or SDP_TYPE_F32, of q, k, their outputs and gradients.
 * weight_type: of q_weight, k_weight ([head_dim]; NULL: ones) and, backward,
 * of their gradients.  rotary_dim: even, at most head_dim; the dimensions
 * past it are normed and not rotated; 0: no rotation.  interleaved: the
 * rotated pairs are (2i, 2i + 1); else (i, i + rotary_dim / 2).
 * cos, sin: FP32 [table_rows, rotary_dim / 2], contiguous.
 * positions: [batch, tokens] contiguous, SDP_TYPE_I32 or SDP_TYPE_I64, each
 * in 0..table_rows - 1; NULL: the token's index in its sequence.
 * q_heads or k_heads may be 0. */
typedef struct {
    int32_t type, weight_type;
    int32_t batch, tokens;
    int32_t q_heads, k_heads, head_dim, rotary_dim;
    int32_t interleaved;
    int32_t position_type;
    double eps;
    int64_t table_rows;
    const float *cos, *sin;
    const void *positions;
    const void *q_weight, *k_weight;
} sdp_qk_norm_rope_desc;

/* For every token and head of q (and k, with k_weight), over the head's
 * elements x:
 *   n = x * w / sqrt(mean(x^2) + eps)
 *   (a, b) = a rotated pair of n at the token's angle:
 *   a' = a cos - b sin,  b' = b cos + a sin
 * q_out may be q itself, and k_out k (same data and strides); q and k may be
 * heads of one fused tensor, and so may q_out and k_out. */
SDP_API int sdp_qk_norm_rope(sdp_ctx *ctx, const sdp_qk_norm_rope_desc *desc, const sdp_heads *q, const sdp_heads *k,
                             const sdp_heads *q_out, const sdp_heads *k_out, void *stream);

/* Its backward: from q, k and the gradients dq_out, dk_out of the outputs,
 * the gradients dq, dk of the inputs and, where not NULL, dq_weight and
 * dk_weight ([head_dim], weight_type; overwritten):
 *   dn = the rotation's transpose of dy;  dw = sum over tokens and heads of
 *   dn x r,  r = 1 / sqrt(mean(x^2) + eps);  u = dn w;
 *   dx = r (u - x r mean(u x r))
 * dq may be dq_out or q itself, and dk likewise. */
SDP_API int sdp_qk_norm_rope_backward(sdp_ctx *ctx, const sdp_qk_norm_rope_desc *desc, const sdp_heads *q,
                                      const sdp_heads *k, const sdp_heads *dq_out, const sdp_heads *dk_out,
                                      const sdp_heads *dq, const sdp_heads *dk, void *dq_weight, void *dk_weight,
                                      void *stream);

/* ---- matrix products grouped by expert ------------------------------------ */

/* rows of x are sorted by group: group e has rows ends[e - 1] .. ends[e] - 1
 * (ends[-1] = 0), so ends is the running sum of the groups' counts,
 * [groups], SDP_TYPE_I32 or SDP_TYPE_I64, in device memory.  A value below
 * the one before it, or past rows, is taken as that one.  Rows past the last
 * end belong to no group.  x, w, dy are BF16; out_type (SDP_TYPE_BF16 or
 * SDP_TYPE_F32) is y's and dw's.  groups * out_features * in_features is at
 * most 2^60. */
typedef struct {
    int64_t rows;
    int32_t groups;
    int32_t in_features, out_features;
    int32_t out_type;
    int32_t ends_type;
    const void *ends;
    int64_t x_stride;  /* row strides of x [rows, in], y [rows, out], dy, dx */
    int64_t y_stride;
    int64_t dx_stride;
} sdp_grouped_desc;

/* y[t] = x[t] w[e]^T for every row t of group e; w is [groups, out, in],
 * contiguous.  Rows of no group are set to 0.  Large products of tensors without
 * whole 16-byte pieces take copies of them in the context's workspace (up to
 * 2 GiB, from about 110 operations for each byte copied on). */
SDP_API int sdp_grouped_matmul(sdp_ctx *ctx, const sdp_grouped_desc *desc, const uint16_t *x, const uint16_t *w,
                               void *y, void *stream);

/* Its backward, from dy (BF16, y_stride): dx[t] = dy[t] w[e] (BF16,
 * dx_stride; rows of no group are set to 0) and dw[e] = the sum over the
 * group's rows of dy[t]^T x[t] (contiguous like w; 0 for an empty group).
 * dx or dw may be NULL; w may be NULL without dx, x without dw. */
SDP_API int sdp_grouped_matmul_backward(sdp_ctx *ctx, const sdp_grouped_desc *desc, const uint16_t *x,
                                        const uint16_t *w, const uint16_t *dy, uint16_t *dx, void *dw, void *stream);

/* ---- distillation from a teacher's top logits ------------------------------ */

/* logits z: [rows, vocab], logit_type SDP_TYPE_BF16 or SDP_TYPE_F32, rows
 * logit_stride apart.  Teacher: teacher_k (0..SDP_DISTILL_MAX_K) entries a
 * row: teacher_logits (teacher_type SDP_TYPE_BF16 or SDP_TYPE_F32) and
 * teacher_index (index_type SDP_TYPE_I32 or SDP_TYPE_I64), both [rows,
 * teacher_k], contiguous; a negative index marks an entry that is not there.
 * labels: [rows], index_type, or NULL; a negative label marks a row without
 * one.  temperature: 1e-6..1e6. */
typedef struct {
    int64_t rows;
    int32_t vocab;
    int32_t logit_type;
    const void *logits;
    int64_t logit_stride;
    int32_t teacher_k, teacher_type, index_type;
    const void *teacher_logits, *teacher_index;
    const void *labels;
    double temperature, distill_weight, label_weight;
} sdp_distill_desc;

/* For each row, with tau = temperature, over the entries j that are there:
 *   q = softmax_j(t / tau),  L_tau = log sum_v exp(z_v / tau),
 *   L_1 = log sum_v exp(z_v)
 *   loss = distill_weight tau^2 sum_j q_j (log q_j - z_j / tau + L_tau)
 *        + label_weight (L_1 - z_label)
 * Terms with q_j = 0 are 0.  A row without entries (or whose entries are all
 * minus infinity) has no first term, a row without label no second; a row
 * with neither has loss 0 and a zero gradient, whatever its logits hold; a
 * weight of 0 leaves its term out, and a row_grad of 0 makes a zero gradient.
 * loss: FP32 [rows].  lse: FP32 [rows, 2], L_tau and L_1 of every row, or
 * NULL.  Where dlogits is not NULL (dlogits_stride apart, logit_type), the
 * gradient is made in the same pass: dlogits = row_grad[row] * d loss / d z,
 * row_grad FP32 [rows] the weight of each row's loss in what is minimised.
 * dlogits may be logits itself (same stride).  An index that is named twice
 * counts with the sum of its q. */
SDP_API int sdp_distill_loss(sdp_ctx *ctx, const sdp_distill_desc *desc, float *loss, float *lse,
                             const float *row_grad, void *dlogits, int64_t dlogits_stride, void *stream);

/* The gradient alone, from lse as sdp_distill_loss wrote it:
 *   d loss / d z_v = distill_weight tau (exp(z_v / tau - L_tau) - q_v)
 *                  + label_weight (exp(z_v - L_1) - [v = label])
 * L's rounding to FP32, up to 2^-24 |L|, is a relative error of the
 * exponentials: small for logits around zero, but a row of the type's lowest
 * value has no L that this can be made from.  The loss and the gradient of
 * sdp_distill_loss come from the logits' differences and have no such limit. */
SDP_API int sdp_distill_loss_backward(sdp_ctx *ctx, const sdp_distill_desc *desc, const float *lse,
                                      const float *row_grad, void *dlogits, int64_t dlogits_stride, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SDP_OPS_H */
