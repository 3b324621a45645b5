// C ABI of libsdp, the training operators around the experts' products
// (include/sdp_layer.h): checks of the arguments and the launches.  The kernels
// are in sdp_embed.hip, sdp_norm.hip, sdp_route.hip, sdp_order.hip and
// sdp_experts.hip.
#include "sdp_layer_internal.h"
#include "sdp_ops_host.h"

using namespace sdprt;
using namespace sdpops;

namespace {

int need(const char *call, const sdp_ctx *ctx, const void *desc) {
    if (!ctx) return fail(SDP_ERR_INVALID_ARGUMENT, "context is NULL");
    if (!desc) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: the description is NULL", call);
    return SDP_OK;
}

// Kernels count in 32 bits within a row.
constexpr int32_t kMostHidden = 1 << 30;

// Finite as what the kernels take.
bool is_finite(double v) { return std::isfinite((float)v); }

Rows kernel_rows(const sdp_rows *r) { return r ? Rows{r->data, r->stride} : Rows{nullptr, 0}; }

// Adds a [rows, cols] tensor to a call's; absent ones have no elements.
int add(std::vector<Tensor> &ts, const char *what, const sdp_rows *r, int64_t rows, int64_t cols, int type,
        bool written) {
    ts.push_back(rows_of(what, r ? r->data : nullptr, r ? rows : 0, r ? r->stride : 0, cols, type_size(type), written));
    return (int)ts.size() - 1;
}

// ---- embeddings ----------------------------------------------------------------

int embed_call(sdp_ctx *ctx, const char *call, const sdp_embed_desc *d, const sdp_rows *table, const sdp_rows *rows,
               bool backward, int32_t accumulate, void *stream) {
    SDP_TRY(need(call, ctx, d));
    if (!table || !rows) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a tensor is NULL", call);
    if (d->tokens < 0 || d->tokens > INT32_MAX || d->vocab < 0 || d->hidden < 0 || d->hidden > kMostHidden)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: tokens, vocab or hidden out of range", call);
    if (!is_float_type(d->table_type) || !is_float_type(d->row_type) || !is_int_type(d->id_type))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a type is none of those allowed", call);
    if (!is_finite(d->scale)) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: scale must be finite", call);
    std::vector<Tensor> ts;
    add(ts, backward ? "dtable" : "table", table, d->vocab, d->hidden, d->table_type, backward);
    add(ts, backward ? "dout" : "out", rows, d->tokens, d->hidden, d->row_type, !backward);
    ts.push_back(dense("ids", d->ids, d->hidden ? d->tokens : 0, type_size(d->id_type), false));
    DeviceGuard guard(ctx->device);
    SDP_TRY(check_tensors(ctx, call, ts, {}));

    EmbedArgs a{};
    a.ids = d->ids;
    a.ids64 = d->id_type == SDP_TYPE_I64;
    a.tokens = d->tokens;
    a.vocab = d->vocab;
    a.hidden = d->hidden;
    a.scale = (float)d->scale;
    a.table = kernel_rows(table);
    a.rows = kernel_rows(rows);
    a.accumulate = accumulate != 0;
    hipStream_t s = (hipStream_t)stream;
    const bool table_bf16 = d->table_type == SDP_TYPE_BF16, rows_bf16 = d->row_type == SDP_TYPE_BF16;
    if (!backward) {
        HIP_TRY(launch_embed(a, table_bf16, rows_bf16, s));
        return SDP_OK;
    }
    if (d->vocab == 0 || d->hidden == 0) return SDP_OK;
    const size_t bytes = embed_workspace(a, nullptr);
    SDP_TRY(take_ops_space(ctx, call, bytes, s));
    embed_workspace(a, ctx->ops_space);
    HIP_TRY(launch_embed_backward(a, table_bf16, rows_bf16, s));
    return ops_mark(ctx, s);
}

// ---- norms around a block ---------------------------------------------------------

int check_norm(const char *call, sdp_ctx *ctx, const sdp_block_norm_desc *d) {
    SDP_TRY(need(call, ctx, d));
    if (d->tokens < 0 || d->tokens > INT32_MAX || d->hidden < 0 || d->hidden > kMostHidden)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: tokens or hidden out of range", call);
    if (!is_float_type(d->stream_type) || !is_float_type(d->type) || !is_float_type(d->weight_type))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a type is none of those allowed", call);
    if (d->gate_form < SDP_GATE_NONE || d->gate_form > SDP_GATE_ELEMENT)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: gate_form is none of those allowed", call);
    if (!is_finite(d->eps) || d->eps < 0.0)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: eps must be finite and >= 0", call);
    if (!is_finite(d->scale) || !is_finite(d->weight_offset))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: scale and weight_offset must be finite", call);
    return SDP_OK;
}

// The gate, or its gradient: each form as the rows and columns that it has.
Tensor gate_tensor(const char *what, const sdp_block_norm_desc *d, const void *p, int64_t stride, bool written) {
    const int64_t size = type_size(d->type);
    switch (d->gate_form) {
        case SDP_GATE_CHANNEL: return dense(what, p, d->hidden, size, written);
        case SDP_GATE_TOKEN: return rows_of(what, p, d->hidden || written ? d->tokens : 0, stride, 1, size, written);
        default: return rows_of(what, p, d->tokens, stride, d->hidden, size, written);
    }
}

NormArgs norm_args(const sdp_block_norm_desc *d, const sdp_rows *h, const sdp_rows *y) {
    NormArgs a{};
    a.tokens = d->tokens;
    a.hidden = d->hidden;
    a.weight_bf16 = d->weight_type == SDP_TYPE_BF16;
    a.post_norm = d->post_norm != 0;
    a.gate_form = d->gate_form;
    a.sigmoid = d->gate_sigmoid != 0;
    a.scale = (float)d->scale;
    a.eps = (float)d->eps;
    a.offset = (float)d->weight_offset;
    a.gate = d->gate;
    a.gate_stride = d->gate_stride;
    a.post_weight = d->post_weight;
    a.pre_weight = d->pre_weight;
    a.h = kernel_rows(h);
    a.y = kernel_rows(y);
    return a;
}

// ---- routing -------------------------------------------------------------------------

int check_route(const char *call, sdp_ctx *ctx, const sdp_route_desc *d, bool groups) {
    SDP_TRY(need(call, ctx, d));
    if (d->tokens < 0 || d->tokens > ((int64_t)1 << 40) || d->experts < 1 || d->experts > SDP_ROUTE_MAX_EXPERTS)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: tokens out of range, or experts not in 1..%d", call,
                    SDP_ROUTE_MAX_EXPERTS);
    if (d->top < 1 || d->top > d->experts || d->top > SDP_ROUTE_MAX_TOP)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: top must be in 1..min(experts, %d) (got %d)", call,
                    SDP_ROUTE_MAX_TOP, d->top);
    if (!is_float_type(d->logit_type) || !is_int_type(d->index_type) || !is_float_type(d->weight_type))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a type is none of those allowed", call);
    if (!is_finite(d->scale)) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: scale must be finite", call);
    if (!groups) return SDP_OK;
    if (d->groups < 1 || d->groups > SDP_ROUTE_MAX_GROUPS || d->experts % d->groups != 0)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: groups must divide experts and be in 1..%d (got %d)", call,
                    SDP_ROUTE_MAX_GROUPS, d->groups);
    if (d->top_groups < 1 || d->top_groups > d->groups || d->group_best < 1 || d->group_best > 2)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: top_groups must be in 1..groups and group_best 1 or 2", call);
    return SDP_OK;
}

RouteArgs route_args(const sdp_route_desc *d, const void *logits) {
    RouteArgs a{};
    a.logits = logits;
    a.logit_stride = d->logit_stride;
    a.tokens = d->tokens;
    a.experts = d->experts;
    a.top = d->top;
    a.index64 = d->index_type == SDP_TYPE_I64;
    a.weight_bf16 = d->weight_type == SDP_TYPE_BF16;
    a.sigmoid = d->sigmoid != 0;
    a.renormalize = d->renormalize != 0;
    a.groups = d->groups;
    a.top_groups = d->top_groups;
    a.group_best = d->group_best;
    a.scale = (float)d->scale;
    return a;
}

// ---- rows to the experts and back -------------------------------------------------------

int check_experts(const char *call, sdp_ctx *ctx, const sdp_expert_desc *d, int64_t *entries) {
    SDP_TRY(need(call, ctx, d));
    if (d->tokens < 0 || d->top < 0 || d->hidden < 0 || d->hidden > kMostHidden || d->tokens > INT32_MAX ||
        (*entries = d->tokens * d->top) > INT32_MAX)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: tokens, top or hidden out of range", call);
    if (!is_float_type(d->row_type) || !is_float_type(d->stream_type) || !is_float_type(d->weight_type))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a type is none of those allowed", call);
    return SDP_OK;
}

ExpertArgs expert_args(const sdp_expert_desc *d) {
    ExpertArgs a{};
    a.tokens = d->tokens;
    a.top = d->top;
    a.hidden = d->hidden;
    a.weight_bf16 = d->weight_type == SDP_TYPE_BF16;
    a.place = d->place;
    return a;
}

}  // namespace

extern "C" {

int sdp_embed(sdp_ctx *ctx, const sdp_embed_desc *desc, const sdp_rows *table, const sdp_rows *out, void *stream) {
    return guarded([&] { return embed_call(ctx, "sdp_embed", desc, table, out, false, 0, stream); });
}

int sdp_embed_backward(sdp_ctx *ctx, const sdp_embed_desc *desc, const sdp_rows *dout, const sdp_rows *dtable,
                       int32_t accumulate, void *stream) {
    return guarded([&] { return embed_call(ctx, "sdp_embed_backward", desc, dtable, dout, true, accumulate, stream); });
}

int sdp_block_norm(sdp_ctx *ctx, const sdp_block_norm_desc *desc, const sdp_rows *h, const sdp_rows *y,
                   const sdp_rows *h_out, const sdp_rows *n_out, void *stream) {
    return guarded([&] {
        const char *call = "sdp_block_norm";
        SDP_TRY(check_norm(call, ctx, desc));
        if (!h) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: h is NULL", call);
        if (!h_out && !n_out) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: both outputs are NULL", call);
        if (h_out && !y) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: h_out without y", call);
        const int64_t t = desc->tokens, n = desc->hidden, wsize = type_size(desc->weight_type);
        std::vector<Tensor> ts;
        const int hi = add(ts, "h", h, t, n, desc->stream_type, false);
        const int yi = add(ts, "y", y, t, n, desc->type, false);
        const int ho = add(ts, "h_out", h_out, t, n, desc->stream_type, true);
        const int no = add(ts, "n_out", n_out, t, n, desc->type, true);
        const bool gated = y && desc->gate_form != SDP_GATE_NONE;
        const bool post = y && desc->post_norm && desc->post_weight, pre = n_out && desc->pre_weight;
        if (gated) ts.push_back(gate_tensor("gate", desc, desc->gate, desc->gate_stride, false));
        if (post) ts.push_back(dense("post_weight", desc->post_weight, t ? n : 0, wsize, false));
        if (pre) ts.push_back(dense("pre_weight", desc->pre_weight, t ? n : 0, wsize, false));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call, ts, {{ho, hi}, {no, yi}}));
        if (t == 0 || n == 0) return SDP_OK;
        NormArgs a = norm_args(desc, h, y);
        a.h_out = kernel_rows(h_out);
        a.n_out = kernel_rows(n_out);
        if (!gated) a.gate_form = SDP_GATE_NONE;
        if (!post) a.post_weight = nullptr;
        if (!pre) a.pre_weight = nullptr;
        HIP_TRY(launch_norm(a, desc->stream_type == SDP_TYPE_BF16, desc->type == SDP_TYPE_BF16, (hipStream_t)stream));
        return SDP_OK;
    });
}

int sdp_block_norm_backward(sdp_ctx *ctx, const sdp_block_norm_desc *desc, const sdp_rows *h_out, const sdp_rows *y,
                            const sdp_rows *dh_out, const sdp_rows *dn, const sdp_block_norm_grads *grads,
                            void *stream) {
    return guarded([&] {
        const char *call = "sdp_block_norm_backward";
        SDP_TRY(check_norm(call, ctx, desc));
        if (!grads) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: the gradients are NULL", call);
        const sdp_block_norm_grads &g = *grads;
        if (!dh_out && !dn) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: dh_out and dn are NULL", call);
        if (dn && !h_out) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: h_out is NULL with dn", call);
        if (g.dgate && desc->gate_form == SDP_GATE_NONE)
            return fail(SDP_ERR_INVALID_ARGUMENT, "%s: dgate without a gate", call);
        if (g.dpost_weight && !desc->post_norm)
            return fail(SDP_ERR_INVALID_ARGUMENT, "%s: dpost_weight without post_norm", call);
        if (g.dpre_weight && !dn) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: dpre_weight without dn", call);
        const bool uses_y = (desc->post_norm && g.dy) || g.dgate || g.dpost_weight;
        if (uses_y && !y) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: y is NULL", call);
        const int64_t t = desc->tokens, n = desc->hidden, wsize = type_size(desc->weight_type);
        std::vector<Tensor> ts;
        add(ts, "h_out", dn ? h_out : nullptr, t, n, desc->stream_type, false);
        const int yi = add(ts, "y", uses_y ? y : nullptr, t, n, desc->type, false);
        const int di = add(ts, "dh_out", dh_out, t, n, desc->stream_type, false);
        const int ni = add(ts, "dn", dn, t, n, desc->type, false);
        const int ho = add(ts, "dh", g.dh, t, n, desc->stream_type, true);
        const int yo = add(ts, "dy", g.dy, t, n, desc->type, true);
        const bool gated = desc->gate_form != SDP_GATE_NONE && (g.dy || g.dgate || g.dpost_weight);
        const bool post = desc->post_norm && (g.dy || g.dgate) && desc->post_weight, pre = dn && desc->pre_weight;
        if (gated) ts.push_back(gate_tensor("gate", desc, desc->gate, desc->gate_stride, false));
        if (post) ts.push_back(dense("post_weight", desc->post_weight, t ? n : 0, wsize, false));
        if (pre) ts.push_back(dense("pre_weight", desc->pre_weight, t ? n : 0, wsize, false));
        if (g.dgate) ts.push_back(gate_tensor("dgate", desc, g.dgate, g.dgate_stride, true));
        if (g.dpost_weight) ts.push_back(dense("dpost_weight", g.dpost_weight, n, wsize, true));
        if (g.dpre_weight) ts.push_back(dense("dpre_weight", g.dpre_weight, n, wsize, true));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call, ts, {{ho, di}, {yo, ni}, {yo, yi}}));
        NormArgs a = norm_args(desc, dn ? h_out : nullptr, uses_y ? y : nullptr);
        if (!gated) a.gate_form = SDP_GATE_NONE;
        if (!post) a.post_weight = nullptr;
        if (!pre) a.pre_weight = nullptr;
        a.dn = kernel_rows(dn);
        a.dh_out = kernel_rows(dh_out);
        a.dh = kernel_rows(g.dh);
        a.dy = kernel_rows(g.dy);
        a.dgate = g.dgate;
        a.dgate_stride = g.dgate_stride;
        a.dpost = g.dpost_weight;
        a.dpre = g.dpre_weight;
        const bool wanted[2] = {g.dpre_weight != nullptr,
                                g.dpost_weight || (g.dgate && desc->gate_form == SDP_GATE_CHANNEL)};
        hipStream_t s = (hipStream_t)stream;
        const bool stream_bf16 = desc->stream_type == SDP_TYPE_BF16, bf16 = desc->type == SDP_TYPE_BF16;
        if (n == 0) {
            HIP_TRY(launch_norm_no_channels(a, bf16, s));
            return SDP_OK;
        }
        a.blocks = norm_blocks(a, stream_bf16, bf16);
        const int sums = wanted[0] + wanted[1];
        if (sums) {
            const size_t row = ((size_t)n + 3) / 4 * 4;
            SDP_TRY(take_ops_space(ctx, call, row * std::max(1, a.blocks) * sums * sizeof(float), s));
            float *at = (float *)ctx->ops_space;
            for (int k = 0; k < 2; ++k)
                if (wanted[k]) a.sums[k] = at, at += row * std::max(1, a.blocks);
        }
        HIP_TRY(launch_norm_backward(a, stream_bf16, bf16, s));
        return sums ? ops_mark(ctx, s) : SDP_OK;
    });
}

int sdp_route(sdp_ctx *ctx, const sdp_route_desc *desc, const void *logits, const float *bias, void *index,
              void *weights, void *stream) {
    return guarded([&] {
        const char *call = "sdp_route";
        SDP_TRY(check_route(call, ctx, desc, true));
        const int64_t t = desc->tokens, n = t * desc->top;
        std::vector<Tensor> ts = {
            rows_of("logits", logits, t, desc->logit_stride, desc->experts, type_size(desc->logit_type), false),
            dense("index", index, n, type_size(desc->index_type), true),
            dense("weights", weights, n, type_size(desc->weight_type), true)};
        if (bias) ts.push_back(dense("bias", bias, t ? desc->experts : 0, 4, false));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call, ts, {}));
        RouteArgs a = route_args(desc, logits);
        a.bias = bias;
        a.index = index;
        a.weights = weights;
        HIP_TRY(launch_route(a, desc->logit_type == SDP_TYPE_BF16, (hipStream_t)stream));
        return SDP_OK;
    });
}

int sdp_route_backward(sdp_ctx *ctx, const sdp_route_desc *desc, const void *logits, const void *index,
                       const void *dweights, void *dlogits, int64_t dlogits_stride, void *stream) {
    return guarded([&] {
        const char *call = "sdp_route_backward";
        SDP_TRY(check_route(call, ctx, desc, false));
        const int64_t t = desc->tokens, n = t * desc->top, zsize = type_size(desc->logit_type);
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call,
                              {rows_of("logits", logits, t, desc->logit_stride, desc->experts, zsize, false),
                               rows_of("dlogits", dlogits, t, dlogits_stride, desc->experts, zsize, true),
                               dense("index", index, n, type_size(desc->index_type), false),
                               dense("dweights", dweights, n, type_size(desc->weight_type), false)},
                              {{1, 0}}));
        RouteArgs a = route_args(desc, logits);
        a.index_in = index;
        a.dweights = dweights;
        a.dlogits = dlogits;
        a.dlogits_stride = dlogits_stride;
        HIP_TRY(launch_route_backward(a, desc->logit_type == SDP_TYPE_BF16, (hipStream_t)stream));
        return SDP_OK;
    });
}

int sdp_expert_order(sdp_ctx *ctx, const sdp_order_desc *desc, const void *index, void *ends, int32_t *place,
                     int32_t *order, void *stream) {
    return guarded([&] {
        const char *call = "sdp_expert_order";
        SDP_TRY(need(call, ctx, desc));
        if (desc->entries < 0 || desc->entries > INT32_MAX)
            return fail(SDP_ERR_INVALID_ARGUMENT, "%s: entries out of range", call);
        if (desc->experts < 0 || desc->experts > SDP_GROUPED_MAX_GROUPS)
            return fail(SDP_ERR_INVALID_ARGUMENT, "%s: experts must be in 0..%d (got %d)", call,
                        SDP_GROUPED_MAX_GROUPS, desc->experts);
        if (!is_int_type(desc->index_type) || !is_int_type(desc->ends_type))
            return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a type is none of those allowed", call);
        const int64_t n = desc->entries;
        std::vector<Tensor> ts = {dense("index", index, n, type_size(desc->index_type), false),
                                  dense("ends", ends, desc->experts, type_size(desc->ends_type), true),
                                  dense("place", place, n, 4, true)};
        if (order) ts.push_back(dense("order", order, n, 4, true));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call, ts, {}));
        SortArgs a{};
        a.keys = index;
        a.keys64 = desc->index_type == SDP_TYPE_I64;
        a.limit = desc->experts;
        a.n = n;
        a.order_out = order;
        a.digits = desc->experts + 1;
        a.bits = 12;
        a.place = place;
        a.ends = ends;
        a.ends64 = desc->ends_type == SDP_TYPE_I64;
        sort_split(a);
        // a block's counts lie where its own places will: no workspace
        a.counts = place;
        a.counts_stride = a.chunk;
        HIP_TRY(launch_sort(a, (hipStream_t)stream));
        return SDP_OK;
    });
}

int sdp_expert_gather(sdp_ctx *ctx, const sdp_expert_desc *desc, const sdp_rows *x, const sdp_rows *rows,
                      void *stream) {
    return guarded([&] {
        const char *call = "sdp_expert_gather";
        int64_t n = 0;
        SDP_TRY(check_experts(call, ctx, desc, &n));
        if (!x || !rows) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a tensor is NULL", call);
        std::vector<Tensor> ts;
        add(ts, "x", x, desc->top ? desc->tokens : 0, desc->hidden, desc->row_type, false);
        add(ts, "rows", rows, n, desc->hidden, desc->row_type, true);
        ts.push_back(dense("place", desc->place, desc->hidden ? n : 0, 4, false));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call, ts, {}));
        ExpertArgs a = expert_args(desc);
        a.side = kernel_rows(x);
        a.rows = kernel_rows(rows);
        HIP_TRY(launch_gather(a, desc->row_type == SDP_TYPE_BF16, (hipStream_t)stream));
        return SDP_OK;
    });
}

int sdp_expert_gather_backward(sdp_ctx *ctx, const sdp_expert_desc *desc, const sdp_rows *drows, const sdp_rows *dx,
                               void *stream) {
    return guarded([&] {
        const char *call = "sdp_expert_gather_backward";
        int64_t n = 0;
        SDP_TRY(check_experts(call, ctx, desc, &n));
        if (!drows || !dx) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a tensor is NULL", call);
        std::vector<Tensor> ts;
        add(ts, "drows", drows, n, desc->hidden, desc->row_type, false);
        add(ts, "dx", dx, desc->tokens, desc->hidden, desc->row_type, true);
        ts.push_back(dense("place", desc->place, desc->hidden ? n : 0, 4, false));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call, ts, {}));
        ExpertArgs a = expert_args(desc);
        a.rows = kernel_rows(drows);
        a.out = kernel_rows(dx);
        const bool bf16 = desc->row_type == SDP_TYPE_BF16;
        HIP_TRY(launch_combine(a, bf16, bf16, (hipStream_t)stream));
        return SDP_OK;
    });
}

int sdp_expert_combine(sdp_ctx *ctx, const sdp_expert_desc *desc, const sdp_rows *rows, const void *weights,
                       const sdp_rows *residual, const sdp_rows *out, void *stream) {
    return guarded([&] {
        const char *call = "sdp_expert_combine";
        int64_t n = 0;
        SDP_TRY(check_experts(call, ctx, desc, &n));
        if (!rows || !out) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a tensor is NULL", call);
        if (!weights && n > 0) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: weights is NULL", call);
        std::vector<Tensor> ts;
        add(ts, "rows", rows, n, desc->hidden, desc->row_type, false);
        const int ri = add(ts, "residual", residual, desc->tokens, desc->hidden, desc->stream_type, false);
        const int oi = add(ts, "out", out, desc->tokens, desc->hidden, desc->stream_type, true);
        ts.push_back(dense("place", desc->place, desc->hidden ? n : 0, 4, false));
        ts.push_back(dense("weights", weights, desc->hidden ? n : 0, type_size(desc->weight_type), false));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call, ts, {{oi, ri}}));
        ExpertArgs a = expert_args(desc);
        a.rows = kernel_rows(rows);
        a.side = kernel_rows(residual);
        a.out = kernel_rows(out);
        a.weights = weights;
        HIP_TRY(launch_combine(a, desc->row_type == SDP_TYPE_BF16, desc->stream_type == SDP_TYPE_BF16,
                               (hipStream_t)stream));
        return SDP_OK;
    });
}

int sdp_expert_combine_backward(sdp_ctx *ctx, const sdp_expert_desc *desc, const sdp_rows *rows, const void *weights,
                                const sdp_rows *dout, const sdp_rows *drows, void *dweights, void *stream) {
    return guarded([&] {
        const char *call = "sdp_expert_combine_backward";
        int64_t n = 0;
        SDP_TRY(check_experts(call, ctx, desc, &n));
        if (!dout || (dweights && !rows)) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a tensor is NULL", call);
        if (drows && !weights && n > 0) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: weights is NULL", call);
        const int64_t wsize = type_size(desc->weight_type);
        std::vector<Tensor> ts;
        const int ri = add(ts, "rows", dweights ? rows : nullptr, n, desc->hidden, desc->row_type, false);
        const int di = add(ts, "drows", drows, n, desc->hidden, desc->row_type, true);
        add(ts, "dout", dout, desc->top ? desc->tokens : 0, desc->hidden, desc->stream_type, false);
        ts.push_back(dense("place", desc->place, n, 4, false));
        if (drows) ts.push_back(dense("weights", weights, n, wsize, false));
        if (dweights) ts.push_back(dense("dweights", dweights, n, wsize, true));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call, ts, {{di, ri}}));
        ExpertArgs a = expert_args(desc);
        a.rows = dweights ? kernel_rows(rows) : Rows{nullptr, 0};
        a.drows = kernel_rows(drows);
        a.side = kernel_rows(dout);
        a.weights = weights;
        a.dweights = dweights;
        if (drows || dweights)
            HIP_TRY(launch_combine_backward(a, desc->row_type == SDP_TYPE_BF16, desc->stream_type == SDP_TYPE_BF16,
                                            (hipStream_t)stream));
        return SDP_OK;
    });
}

}  // extern "C"
