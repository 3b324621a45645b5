/*
 * sdp_layer.h -- C ABI of libsdp, the training operators around the experts'
 * products.
 *
 * The operators of sdp_ops.h are a layer's products of experts, its norm and
 * rotation of heads, and the loss; the ones here are what a training step of
 * a mixture-of-experts model does between them (the paper trains such models
 * under the same data-parallel runtime: Evaluation, MoE and correctness):
 *   sdp_embed            scaled rows of a table at the tokens' ids; and the
 *                        table's gradient
 *   sdp_block_norm       the norm of a block's output, its gate, the residual
 *                        scale and addition, and the norm before the next
 *                        block, in one pass; and its backward
 *   sdp_route            each token's experts and their weights; and its backward
 *   sdp_expert_order     where each chosen row stands among the rows sorted by
 *                        expert, and the ends that sdp_grouped_matmul takes
 *   sdp_expert_gather    tokens to those rows; and its backward
 *   sdp_expert_combine   the weighted sum of each token's rows; and its backward
 * A weight gradient may be written as BF16 straight into a rank's gradient
 * buffer of an sdp_segment.
 *
 * Conventions are those of sdp_ops.h: device memory of the caller's, aligned
 * to its elements; strides in elements, the last dimension contiguous, inputs
 * may be broadcast (a stride of 0); asynchronous on `stream`; statistics and
 * sums in FP32 and each output rounded once; the same inputs give the same
 * bits (the only atomics count integers in LDS); sizes of zero are valid;
 * values in device memory that are out of range are never used as an address.
 * hidden is at most 2^30; scale, eps and weight_offset are finite in FP32.
 *
 * sdp_embed_backward and sdp_block_norm_backward with gradients that are sums
 * over tokens (weights, a gate that tokens share) use the context's workspace:
 * they run after the context's last call that used it and are refused on a
 * capturing stream.  All other calls may be captured into a HIP graph.
 */
#ifndef SDP_LAYER_H
#define SDP_LAYER_H

#include "sdp_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- limits -------------------------------------------------------------- */
#define SDP_ROUTE_MAX_EXPERTS 2048
#define SDP_ROUTE_MAX_TOP 64
#define SDP_ROUTE_MAX_GROUPS 64

/* A [rows, columns] tensor: element (r, c) is data[r * stride + c]. */
typedef struct {
    void *data;
    int64_t stride;
} sdp_rows;

/* ---- token embeddings ------------------------------------------------------ */

/* table_type: SDP_TYPE_BF16 or SDP_TYPE_F32, of the table and its gradient
 * ([vocab, hidden]); row_type likewise, of out and dout ([tokens, hidden]).
 * ids: [tokens], id_type SDP_TYPE_I32 or SDP_TYPE_I64.  tokens is at most
 * 2^31 - 1. */
typedef struct {
    int64_t tokens;
    int32_t vocab, hidden;
    int32_t table_type, row_type, id_type;
    const void *ids;
    double scale;
} sdp_embed_desc;

/* out[t] = scale table[ids[t]].  A negative id names nothing (padding): a row
 * of zeros; an id past the vocabulary gives NaN. */
SDP_API int sdp_embed(sdp_ctx *ctx, const sdp_embed_desc *desc, const sdp_rows *table, const sdp_rows *out,
                      void *stream);

/* Its backward: dtable[v] = scale * the sum of dout[t] over the tokens with
 * ids[t] = v, in the tokens' order, 16 at a time.
 * accumulate 0: every row of dtable is written, those that no token names
 * with zeros; else the sum is added to what dtable holds (a table that is the
 * head's weight too), and rows that no token names are left as they are.
 * Tokens whose id is negative or past the vocabulary have no part in it. */
SDP_API int sdp_embed_backward(sdp_ctx *ctx, const sdp_embed_desc *desc, const sdp_rows *dout,
                               const sdp_rows *dtable, int32_t accumulate, void *stream);

/* ---- norms around a block --------------------------------------------------- */

#define SDP_GATE_NONE 0
#define SDP_GATE_CHANNEL 1  /* gate [hidden], for every token */
#define SDP_GATE_TOKEN 2    /* gate [tokens], gate_stride apart, for every channel */
#define SDP_GATE_ELEMENT 3  /* gate [tokens, hidden], rows gate_stride apart */

/* stream_type: SDP_TYPE_BF16 or SDP_TYPE_F32, of the residual stream h, h_out
 * and their gradients; type likewise, of the block's output y, n_out, the gate
 * and their gradients; weight_type likewise, of post_weight and pre_weight
 * ([hidden]; NULL: a factor of one) and their gradients.  A weight w counts as
 * weight_offset + w.  tokens is at most 2^31 - 1. */
typedef struct {
    int64_t tokens;
    int32_t hidden;
    int32_t stream_type, type, weight_type;
    int32_t post_norm;     /* not 0: y is normed */
    int32_t gate_form;     /* SDP_GATE_... */
    int32_t gate_sigmoid;  /* not 0: the gate goes through a sigmoid */
    double scale, eps, weight_offset;
    const void *gate;
    int64_t gate_stride;
    const void *post_weight, *pre_weight;
} sdp_block_norm_desc;

/* For each token, with rms(x) = sqrt(mean(x^2) + eps) over its channels:
 *   u = post_norm ? y (weight_offset + post_weight) / rms(y) : y
 *   h_out = h + scale a u,  a = gate, sigmoid(gate) or 1
 *   n_out = h_out (weight_offset + pre_weight) / rms(h_out)
 * n_out comes from h_out before its rounding.  y may be NULL (nothing is
 * added; h_out is then NULL too, and n_out is the norm of h); either output
 * may be NULL.  h_out may be h itself, and n_out y (same data and stride). */
SDP_API int sdp_block_norm(sdp_ctx *ctx, const sdp_block_norm_desc *desc, const sdp_rows *h, const sdp_rows *y,
                           const sdp_rows *h_out, const sdp_rows *n_out, void *stream);

/* The gradients that sdp_block_norm_backward writes; each may be NULL.  dgate:
 * like the gate ([hidden]; [tokens], dgate_stride apart; [tokens, hidden], rows
 * dgate_stride apart), type.  dpost_weight, dpre_weight: [hidden], weight_type. */
typedef struct {
    const sdp_rows *dh, *dy;
    void *dgate;
    int64_t dgate_stride;
    void *dpost_weight, *dpre_weight;
} sdp_block_norm_grads;

/* Its backward, from the stream after the addition (h_out), y, and the
 * gradients dh_out and dn of the outputs (either may be NULL: zero):
 *   g = dh_out + the norm's gradient of dn;  dh = g;  du = scale a g
 *   dgate = the sum of scale u g (times the sigmoid's slope) over what shares it
 *   dy = post_norm ? the norm's gradient of du : du
 *   dpre_weight = sum over tokens of dn h_out / rms(h_out)
 *   dpost_weight = sum over tokens of du y / rms(y)
 * where the norm's gradient of v is (v w - x mean(v w x) / rms(x)^2) / rms(x).
 * h_out may be NULL without dn; y where neither post_norm (with dy) nor
 * dgate nor dpost_weight needs it.  dpre_weight needs dn, dpost_weight
 * post_norm, dgate a gate.  dh may be dh_out itself, and dy may be dn
 * or y. */
SDP_API int sdp_block_norm_backward(sdp_ctx *ctx, const sdp_block_norm_desc *desc, const sdp_rows *h_out,
                                    const sdp_rows *y, const sdp_rows *dh_out, const sdp_rows *dn,
                                    const sdp_block_norm_grads *grads, void *stream);

/* ---- routing to experts -------------------------------------------------------- */

/* logits z: [tokens, experts], logit_type SDP_TYPE_BF16 or SDP_TYPE_F32, rows
 * logit_stride apart.  index and the weights are [tokens, top], contiguous:
 * index_type SDP_TYPE_I32 or SDP_TYPE_I64, weight_type SDP_TYPE_F32 or
 * SDP_TYPE_BF16.  top: 1..min(experts, SDP_ROUTE_MAX_TOP).  groups: 1 (none) or
 * a divisor of experts, at most SDP_ROUTE_MAX_GROUPS; top_groups: 1..groups;
 * group_best: 1 or 2. */
typedef struct {
    int64_t tokens;
    int32_t experts, top;
    int32_t logit_type, index_type, weight_type;
    int32_t sigmoid;      /* not 0: scores are sigmoid(z), else softmax(z) */
    int32_t renormalize;  /* not 0: a token's weights are divided by their sum */
    int32_t groups, top_groups, group_best;
    double scale;
    int64_t logit_stride;
} sdp_route_desc;

/* Each token's experts, the best first: those of largest score + bias (bias:
 * FP32 [experts], or NULL) and, among equals, of lowest index.  The
 * comparison is of 64-bit scores; without bias and groups, which change no
 * order, it is of the logits.  With groups (runs of experts / groups experts)
 * only experts of the top_groups best groups are taken, a group's worth being
 * the sum of its group_best largest score + bias.
 *   weight = scale score, or with renormalize scale score / (sum of the scores
 *   of the token's experts)
 * The bias has no part in a weight.  An expert whose logit or bias is minus
 * infinity is not there: it is never chosen, and a group of such experts
 * neither; places that are left over have index -1 and weight 0 (all of them,
 * in a row of nothing but minus infinity).  A NaN counts as larger than
 * everything, and makes the weights that depend on it NaN. */
SDP_API int sdp_route(sdp_ctx *ctx, const sdp_route_desc *desc, const void *logits, const float *bias, void *index,
                      void *weights, void *stream);

/* Its backward: dlogits (logit_type, dlogits_stride apart) from the weights'
 * gradient and the index that sdp_route wrote; groups, top_groups and
 * group_best are not looked at, nor with renormalize logits that the index
 * does not name.  The choice itself has no gradient.  Negative indexes are
 * places left over; a row with an index past the experts gives NaN.  An index
 * that is named twice counts twice.  dlogits may be logits itself (same
 * stride). */
SDP_API int sdp_route_backward(sdp_ctx *ctx, const sdp_route_desc *desc, const void *logits, const void *index,
                               const void *dweights, void *dlogits, int64_t dlogits_stride, void *stream);

/* ---- rows to the experts and back --------------------------------------------- */

/* index: [entries], index_type SDP_TYPE_I32 or SDP_TYPE_I64: the expert of each
 * entry (a token's `top` entries follow each other, as in sdp_route's index).
 * ends: [experts], ends_type SDP_TYPE_I32 or SDP_TYPE_I64.  entries is at most
 * 2^31 - 1, experts SDP_GROUPED_MAX_GROUPS. */
typedef struct {
    int64_t entries;
    int32_t experts;
    int32_t index_type, ends_type;
} sdp_order_desc;

/* Sorts the entries by expert, those of one expert in their own order:
 *   place[e] (I32 [entries]) = the row of entry e
 *   ends[x] = the number of entries of experts 0..x
 *   order (I32 [entries], or NULL): order[place[e]] = e
 * An entry with a negative index, or one past the experts, has no expert: it
 * is matched with a row p past the last end (in the entries' order too), its
 * place is -1 - p, and order[p] is -1. */
SDP_API int sdp_expert_order(sdp_ctx *ctx, const sdp_order_desc *desc, const void *index, void *ends, int32_t *place,
                             int32_t *order, void *stream);

/* tokens of `top` entries each, and rows: [tokens * top, hidden] of them sorted
 * by expert, at most 2^31 - 1; place: [tokens, top] as sdp_expert_order wrote
 * it.  row_type: SDP_TYPE_BF16 or SDP_TYPE_F32, of the rows and of what is
 * gathered; stream_type likewise, of residual, out and dout; weight_type
 * likewise, of weights and dweights ([tokens, top], contiguous). */
typedef struct {
    int64_t tokens;
    int32_t top, hidden;
    int32_t row_type, stream_type, weight_type;
    const int32_t *place;
} sdp_expert_desc;

/* rows[place[t, j]] = x[t]; rows that no entry of an expert has are set to 0.
 * A place that names no row writes nothing. */
SDP_API int sdp_expert_gather(sdp_ctx *ctx, const sdp_expert_desc *desc, const sdp_rows *x, const sdp_rows *rows,
                              void *stream);

/* dx[t] = the sum over j of drows[place[t, j]] (row_type), without the entries
 * that have no expert.  A place that names no row gives NaN. */
SDP_API int sdp_expert_gather_backward(sdp_ctx *ctx, const sdp_expert_desc *desc, const sdp_rows *drows,
                                       const sdp_rows *dx, void *stream);

/* out[t] = residual[t] (NULL: 0) + the sum over j of weights[t, j]
 * rows[place[t, j]], without the entries that have no expert.  A place that
 * names no row gives NaN.  out may be residual itself. */
SDP_API int sdp_expert_combine(sdp_ctx *ctx, const sdp_expert_desc *desc, const sdp_rows *rows, const void *weights,
                               const sdp_rows *residual, const sdp_rows *out, void *stream);

/* Its backward: drows[place[t, j]] = weights[t, j] dout[t] (row_type; rows of no
 * expert are set to 0) and dweights[t, j] = the inner product of dout[t] and
 * rows[place[t, j]] (0 for an entry without an expert, NaN where the place
 * names no row).  drows or dweights may be NULL; weights may be NULL without
 * drows, rows without dweights.  drows may be rows itself.  The residual's
 * gradient is dout. */
SDP_API int sdp_expert_combine_backward(sdp_ctx *ctx, const sdp_expert_desc *desc, const sdp_rows *rows,
                                        const void *weights, const sdp_rows *dout, const sdp_rows *drows,
                                        void *dweights, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SDP_LAYER_H */
