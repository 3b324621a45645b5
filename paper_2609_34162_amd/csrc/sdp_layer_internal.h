// Internals of the training operators around the experts' products
// (include/sdp_layer.h): what their entry points (sdp_layer.hip) pass to the
// kernels' launch functions (sdp_embed.hip, sdp_norm.hip, sdp_route.hip,
// sdp_order.hip, sdp_experts.hip).  Not installed; not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "sdp_layer.h"

namespace sdpops {

// A [rows, columns] tensor as the kernels address it (elements).
struct Rows {
    void *data;
    int64_t stride;
};

// ---- sorting by a small key --------------------------------------------------

// One pass of a stable counting sort: n entries by digits in [0, digits).  The
// counts of each block of entries lie in a row of `digits` of their own.
struct SortArgs {
    const void *keys;         // [n] expert indexes or token ids, in the order before the pass
    int32_t keys64;
    int32_t limit;            // keys outside 0..limit - 1 count as limit
    int64_t n;
    const int32_t *order_in;  // entry at each place before the pass; NULL: the entries' own order
    int32_t *order_out;       // and after it (may be NULL)
    int32_t shift, digits;    // digit = key >> shift & (2^bits - 1)
    int32_t bits;
    // of experts (limit + 1 digits, the last one of entries without an expert)
    int32_t *place;           // place of each entry, or -1 - place; NULL: not wanted
    void *ends;
    int32_t ends64;
    int32_t *keys_out;        // key at each place after the pass (may be NULL)
    int32_t *counts;          // [blocks] rows, counts_stride apart
    bool apart;               // they are not place itself
    int64_t counts_stride;
    int64_t chunk;            // entries of a block
    int32_t blocks;
};

// How the entries are split over blocks; counts may be place itself, rows a chunk apart.
void sort_split(SortArgs &a);
bool sort_needs_counts(const SortArgs &a);
hipError_t launch_sort(const SortArgs &a, hipStream_t s);

// ---- embeddings ----------------------------------------------------------------

struct EmbedArgs {
    const void *ids;
    int32_t ids64;
    int64_t tokens;
    int32_t vocab, hidden;
    float scale;
    Rows table;  // or its gradient
    Rows rows;   // out, or dout
    int32_t accumulate;
    // workspace of the gradient
    int32_t *order, *order_spare, *key, *key_spare, *counts;
    // [pieces, 2, hidden] sums of what a piece of the places has of ids that go on
    // before it (or all through it) and of ids that go on behind it
    float *sums;
};

size_t embed_workspace(EmbedArgs &a, char *space);
hipError_t launch_embed(const EmbedArgs &a, bool table_bf16, bool rows_bf16, hipStream_t s);
hipError_t launch_embed_backward(const EmbedArgs &a, bool table_bf16, bool rows_bf16, hipStream_t s);

// ---- norms around a block ---------------------------------------------------------

struct NormArgs {
    int64_t tokens;
    int32_t hidden;
    int32_t weight_bf16, post_norm, gate_form, sigmoid;
    float scale, eps, offset;
    const void *gate;
    int64_t gate_stride;
    const void *post_weight, *pre_weight;
    Rows h, y, h_out, n_out;   // forward: in, in, out, out; data NULL: not there
    Rows dn, dh_out, dh, dy;   // backward: in, in, out, out (h is the stream after the addition)
    void *dgate;
    int64_t dgate_stride;
    void *dpost, *dpre;
    // partial sums over tokens, [blocks, hidden] each, of dn h r (for dpre) and of y ry g, times
    // the gate where it is a token's own (for dpost and the channels' dgate); NULL: not wanted
    float *sums[2];
    int32_t blocks;
    int32_t team;  // lanes to a row (set by the launch)
};

// Blocks of the backward call, each of which leaves a row of partial sums.
int norm_blocks(const NormArgs &a, bool stream_bf16, bool bf16);
hipError_t launch_norm(const NormArgs &a, bool stream_bf16, bool bf16, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs &a, bool stream_bf16, bool bf16, hipStream_t s);
// What the backward call writes where hidden is 0.
hipError_t launch_norm_no_channels(const NormArgs &a, bool bf16, hipStream_t s);

// ---- routing -------------------------------------------------------------------------

struct RouteArgs {
    const void *logits;
    int64_t logit_stride, tokens;
    int32_t experts, top;
    int32_t index64, weight_bf16;
    int32_t sigmoid, renormalize;
    int32_t groups, top_groups, group_best;
    float scale;
    const float *bias;
    void *index, *weights;         // forward: written
    const void *index_in, *dweights;
    void *dlogits;
    int64_t dlogits_stride;
    // set by the launch: lanes of a token, and the launch's first wave's worth of tokens
    int32_t lanes;
    int64_t first;
};

hipError_t launch_route(const RouteArgs &a, bool bf16, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs &a, bool bf16, hipStream_t s);

// ---- rows to the experts and back -------------------------------------------------------

struct ExpertArgs {
    int64_t tokens;
    int32_t top, hidden;
    int32_t weight_bf16;
    const int32_t *place;
    Rows rows, drows;       // sorted by expert
    Rows side, out;         // of the tokens: x, residual or dout; and what is written
    const void *weights;
    void *dweights;
};

hipError_t launch_gather(const ExpertArgs &a, bool row_bf16, hipStream_t s);
// weights NULL: ones
hipError_t launch_combine(const ExpertArgs &a, bool row_bf16, bool stream_bf16, hipStream_t s);
hipError_t launch_combine_backward(const ExpertArgs &a, bool row_bf16, bool stream_bf16, hipStream_t s);

}  // namespace sdpops
