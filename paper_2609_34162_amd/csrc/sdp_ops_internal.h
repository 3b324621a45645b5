// Internals of the training operators (include/sdp_ops.h): what their entry
// points (sdp_ops.hip) pass to the kernels' launch functions (sdp_qk.hip,
// sdp_grouped.hip, sdp_distill.hip).  Not installed; not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "sdp_ops.h"

namespace sdpops {

// ---- norms of queries and keys with the rotation --------------------------

// A [batch, tokens, heads, dim] tensor as the kernels address it (elements).
struct Heads {
    const void *data;
    int64_t b, s, h;
};

// The query or the key heads of a call: x in, y in (backward: the outputs'
// gradient), out written.
struct QkSide {
    Heads x, y, out;
    int32_t heads;
    const void *weight;   // NULL: ones
    float *partials;      // backward: [blocks, dim] sums of dn x r, one row a block; NULL: not wanted
    void *dweight;
};

struct QkArgs {
    QkSide side[2];
    int64_t rows_total[2];  // batch * tokens * heads
    int32_t blocks[2];      // of each side; backward each leaves a row of partial sums
    int32_t batch, tokens, dim, rotary, interleaved;
    int32_t weight_bf16, positions64;
    float eps;
    int64_t table_rows;
    const float *cos, *sin;
    const void *positions;
    // how the call is split (qk_split): runs of heads that a wave takes, how many
    // of them a token has on each side, and the heads that it reads at once (log 2)
    int32_t chunk_heads, chunks[2], heads_log[2];
    bool stream;  // non-temporal loads and stores
};

// Fills in how the call is split over blocks.
void qk_split(QkArgs &a, bool bf16, bool backward);
hipError_t launch_qk(const QkArgs &a, bool bf16, bool backward, hipStream_t s);

// ---- grouped products ------------------------------------------------------

struct GroupedArgs {
    const uint16_t *x, *w, *dy;
    uint16_t *dx;
    void *y, *dw;
    const void *ends;
    int64_t rows, x_stride, y_stride, dx_stride;
    int32_t groups, n_in, n_out;
    int32_t ends64, out_f32;
    float *partials;   // FP32 sums of parts of the rows, where dw is split
    int32_t splits;
};

// Whether each product's tiles fit one launch.
bool grouped_fits(const GroupedArgs &a, bool forward, bool dx, bool dw);
// Bytes of workspace that the call needs (0: none): partial sums, or copies of tensors
// in whole pieces.
size_t grouped_workspace(const GroupedArgs &a, bool forward, bool dx, bool dw);
hipError_t launch_grouped(const GroupedArgs &a, bool forward, bool dx, bool dw, void *space, hipStream_t s);

// ---- distillation ----------------------------------------------------------

struct DistillArgs {
    const void *logits;
    int64_t logit_stride, rows;
    int32_t vocab, k;
    const void *teacher_logits, *teacher_index, *labels;
    int32_t teacher_bf16, index64;
    float inv_tau, tau;
    float distill_weight, label_weight;
    float *loss, *lse;             // forward: written (lse may be NULL)
    const float *lse_in;           // backward: read
    const float *row_grad;
    void *dlogits;                 // NULL: loss only
    int64_t dlogits_stride;
    float *partials;               // [rows, splits, kDistillPartials]: what each part of a row found
    int32_t splits;                // parts of a row for its sums; 0: rows stay in registers
    int32_t parts;                 // and for its gradient
};

constexpr int kDistillPartials = 8;

// The parts of a row for its sums, or 0 where the call takes no partials.
int distill_splits(const DistillArgs &a, bool bf16);
hipError_t launch_distill(const DistillArgs &a, bool bf16, hipStream_t s);
hipError_t launch_distill_backward(const DistillArgs &a, bool bf16, hipStream_t s);

}  // namespace sdpops
