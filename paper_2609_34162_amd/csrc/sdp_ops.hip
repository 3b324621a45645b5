// C ABI of libsdp, the training operators (include/sdp_ops.h): checks of the
// arguments, the context's workspace for them, and the launches.  The kernels
// are in sdp_qk.hip, sdp_grouped.hip and sdp_distill.hip.
#include "sdp_ops_host.h"
#include "sdp_ops_internal.h"

using namespace sdprt;

namespace sdpops {

// ---- checks -----------------------------------------------------------------

// An allocation that a call's earlier buffers were found to lie in.
struct Allocation {
    const char *base;
    size_t size;
};

static int check_memory(const sdp_ctx *ctx, const char *call, const Tensor &t, int64_t bytes, Allocation &found) {
    hipPointerAttribute_t at;
    if (hipPointerGetAttributes(&at, t.p) != hipSuccess) {
        (void)hipGetLastError();
        return fail(SDP_ERR_NOT_DEVICE_MEMORY, "%s: %s (%p) is not device memory", call, t.what, t.p);
    }
    if (at.type != hipMemoryTypeDevice || at.device != ctx->device)
        return fail(SDP_ERR_NOT_DEVICE_MEMORY, "%s: %s (%p) is not device memory of GPU %d", call, t.what, t.p,
                    ctx->device);
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)t.p) != hipSuccess) {
        (void)hipGetLastError();
        return fail(SDP_ERR_NOT_DEVICE_MEMORY, "%s: %s (%p): allocation range unknown", call, t.what, t.p);
    }
    if ((size_t)bytes > size - (size_t)((const char *)t.p - (const char *)base))
        return fail(SDP_ERR_NOT_DEVICE_MEMORY, "%s: %s: %lld bytes at %p overrun its allocation", call, t.what,
                    (long long)bytes, t.p);
    found = {(const char *)base, size};
    return SDP_OK;
}

int check_tensors(const sdp_ctx *ctx, const char *call, const std::vector<Tensor> &ts,
                  const std::vector<std::pair<int, int>> &in_place) {
    constexpr size_t kMost = 32;  // more tensors than any call has
    int64_t bytes[kMost];         // from a tensor's first element to its last
    if (ts.size() > kMost) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: too many tensors", call);
    for (size_t i = 0; i < ts.size(); ++i) {
        const Tensor &t = ts[i];
        const int64_t elems = sdpops::span(t.layout);
        if (elems < 0) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: %s: a stride is negative or too large", call, t.what);
        bytes[i] = elems * t.size;
        if (elems == 0) continue;
        if (!t.p) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: %s is NULL", call, t.what);
        if ((uintptr_t)t.p % (uintptr_t)t.size != 0)
            return fail(SDP_ERR_ALIGNMENT, "%s: %s (%p) is not aligned to its %lld-byte elements", call, t.what, t.p,
                        (long long)t.size);
        if (t.written && !sdpops::injective(t.layout))
            return fail(SDP_ERR_INVALID_ARGUMENT, "%s: %s overlaps itself", call, t.what);
    }
    // a program's small buffers often share an allocation, which is then looked up once
    Allocation found[4];
    int founds = 0;
    for (size_t i = 0; i < ts.size(); ++i) {
        if (bytes[i] == 0) continue;
        const char *p = (const char *)ts[i].p;
        bool known = false;
        for (int k = 0; k < founds; ++k)
            known = known || (p >= found[k].base && (size_t)bytes[i] <= found[k].size &&
                              (size_t)(p - found[k].base) <= found[k].size - (size_t)bytes[i]);
        if (known) continue;
        Allocation a;
        SDP_TRY(check_memory(ctx, call, ts[i], bytes[i], a));
        if (founds < 4) found[founds++] = a;
    }
    for (size_t i = 0; i < ts.size(); ++i) {
        if (!ts[i].written || bytes[i] == 0) continue;
        for (size_t j = 0; j < ts.size(); ++j) {
            if (i == j || bytes[j] == 0 || (ts[j].written && j < i)) continue;
            const Tensor &a = ts[i], &b = ts[j];
            const char *pa = (const char *)a.p, *pb = (const char *)b.p;
            if (pa + bytes[i] <= pb || pb + bytes[j] <= pa) continue;
            bool may = false;
            for (const auto &pr : in_place)
                may = may || (pr.first == (int)i && pr.second == (int)j) || (pr.first == (int)j && pr.second == (int)i);
            if (may && a.size == b.size && sdpops::same_tensor(pa, a.layout, pb, b.layout)) continue;
            if (!(a.size == b.size && sdpops::disjoint(pa, a.layout, pb, b.layout, a.size)))
                return fail(SDP_ERR_INVALID_ARGUMENT, "%s: %s overlaps %s", call, a.what, b.what);
        }
    }
    return SDP_OK;
}

// ---- workspace ----------------------------------------------------------------

static int ensure_ops_space(sdp_ctx *ctx, size_t bytes) {
    if (bytes <= ctx->ops_space_cap) return SDP_OK;
    HIP_TRY(hipDeviceSynchronize());
    if (ctx->ops_space) HIP_TRY(hipFree(ctx->ops_space));
    ctx->ops_space = nullptr;
    ctx->ops_space_cap = 0;
    if (!ctx->ops_done) HIP_TRY(hipEventCreateWithFlags(&ctx->ops_done, hipEventDisableTiming));
    if (hipMalloc(&ctx->ops_space, bytes) != hipSuccess) {
        (void)hipGetLastError();
        ctx->ops_space = nullptr;
        return fail(SDP_ERR_OUT_OF_MEMORY, "cannot allocate %zu bytes of operator workspace", bytes);
    }
    ctx->ops_space_cap = bytes;
    return SDP_OK;
}

int take_ops_space(sdp_ctx *ctx, const char *call, size_t bytes, hipStream_t s) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (s) HIP_TRY(hipStreamIsCapturing(s, &capture));
    if (capture != hipStreamCaptureStatusNone)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a call that uses the context's workspace cannot be captured", call);
    SDP_TRY(ensure_ops_space(ctx, bytes));
    if (ctx->ops_done_valid) HIP_TRY(hipStreamWaitEvent(s, ctx->ops_done, 0));
    return SDP_OK;
}
int ops_mark(sdp_ctx *ctx, hipStream_t s) {
    HIP_TRY(hipEventRecord(ctx->ops_done, s));
    ctx->ops_done_valid = true;
    return SDP_OK;
}

}  // namespace sdpops

using namespace sdpops;

namespace {

// ---- norms of queries and keys -------------------------------------------------

Tensor heads_tensor(const char *what, const sdp_heads *h, const sdp_qk_norm_rope_desc *d, int heads, bool written) {
    Layout l{{d->batch, d->tokens, heads}, {h->batch_stride, h->token_stride, h->head_stride}, d->head_dim};
    for (int k = 0; k < 3; ++k)
        if (l.ext[k] <= 1) l.stride[k] = 0;
    return {what, h->data, l, type_size(d->type), written};
}

sdpops::Heads kernel_heads(const Tensor &t) {
    return {t.p, t.layout.stride[0], t.layout.stride[1], t.layout.stride[2]};
}

int qk_call(sdp_ctx *ctx, const char *call, const sdp_qk_norm_rope_desc *d, const sdp_heads *const x[2],
            const sdp_heads *const y[2], const sdp_heads *const out[2], void *const dweight[2], bool backward,
            void *stream) {
    if (!ctx) return fail(SDP_ERR_INVALID_ARGUMENT, "context is NULL");
    if (!d) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: the description is NULL", call);
    for (int k = 0; k < 2; ++k)
        if (!x[k] || !out[k] || (backward && !y[k]))
            return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a tensor is NULL", call);
    if (!is_float_type(d->type) || !is_float_type(d->weight_type))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: type and weight_type must be SDP_TYPE_F32 or SDP_TYPE_BF16", call);
    if (d->batch < 0 || d->tokens < 0 || d->q_heads < 0 || d->k_heads < 0 || d->q_heads > SDP_QK_MAX_HEADS ||
        d->k_heads > SDP_QK_MAX_HEADS)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: batch, tokens or heads out of range", call);
    if (d->head_dim < 1 || d->head_dim > SDP_QK_MAX_HEAD_DIM)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: head_dim must be in 1..%d (got %d)", call, SDP_QK_MAX_HEAD_DIM,
                    d->head_dim);
    if (d->rotary_dim < 0 || d->rotary_dim > d->head_dim || d->rotary_dim % 2 != 0)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: rotary_dim must be even and at most head_dim (got %d)", call,
                    d->rotary_dim);
    if (d->table_rows < 0 || d->table_rows > ((int64_t)1 << 40))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: table_rows out of range", call);
    if (d->positions && !is_int_type(d->position_type))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: positions must be SDP_TYPE_I32 or SDP_TYPE_I64", call);
    if (!std::isfinite(d->eps) || d->eps < 0.0)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: eps must be finite and >= 0", call);

    const int64_t tokens = (int64_t)d->batch * d->tokens, table = d->table_rows * (d->rotary_dim / 2);
    const int64_t wsize = type_size(d->weight_type);
    const int heads[2] = {d->q_heads, d->k_heads};
    static const char *const x_name[2] = {"q", "k"}, *const y_name[2] = {"dq_out", "dk_out"},
                             *const out_name[2][2] = {{"q_out", "k_out"}, {"dq", "dk"}};
    const void *const weight[2] = {d->q_weight, d->k_weight};
    std::vector<Tensor> ts;
    for (int k = 0; k < 2; ++k) {
        ts.push_back(heads_tensor(x_name[k], x[k], d, heads[k], false));
        ts.push_back(heads_tensor(y_name[k], backward ? y[k] : x[k], d, heads[k], false));
        ts.push_back(heads_tensor(out_name[backward][k], out[k], d, heads[k], true));
    }
    const std::vector<std::pair<int, int>> in_place = {{2, 0}, {2, 1}, {5, 3}, {5, 4}};
    ts.push_back(dense("cos", d->cos, tokens ? table : 0, 4, false));
    ts.push_back(dense("sin", d->sin, tokens ? table : 0, 4, false));
    for (int k = 0; k < 2; ++k) {
        if (weight[k]) ts.push_back(dense(k ? "k_weight" : "q_weight", weight[k], d->head_dim, wsize, false));
        if (dweight[k]) ts.push_back(dense(k ? "dk_weight" : "dq_weight", dweight[k], d->head_dim, wsize, true));
    }
    if (d->positions)
        ts.push_back(dense("positions", d->positions, tokens, type_size(d->position_type), false));
    DeviceGuard guard(ctx->device);
    SDP_TRY(check_tensors(ctx, call, ts, in_place));

    sdpops::QkArgs a{};
    for (int k = 0; k < 2; ++k) {
        a.side[k].x = kernel_heads(ts[3 * k]);
        a.side[k].y = kernel_heads(ts[3 * k + 1]);
        a.side[k].out = kernel_heads(ts[3 * k + 2]);
        a.side[k].heads = heads[k];
        a.side[k].weight = weight[k];
        a.side[k].dweight = dweight[k];
        a.rows_total[k] = tokens * heads[k];
    }
    a.batch = d->batch;
    a.tokens = d->tokens;
    a.dim = d->head_dim;
    a.rotary = d->rotary_dim;
    a.interleaved = d->interleaved != 0;
    a.weight_bf16 = d->weight_type == SDP_TYPE_BF16;
    a.positions64 = d->position_type == SDP_TYPE_I64;
    a.eps = (float)d->eps;
    a.table_rows = d->table_rows;
    a.cos = d->cos;
    a.sin = d->sin;
    a.positions = d->positions;
    hipStream_t s = (hipStream_t)stream;
    const bool sums = dweight[0] || dweight[1], bf16 = d->type == SDP_TYPE_BF16;
    sdpops::qk_split(a, bf16, backward);
    if (sums) {
        const int64_t per[2] = {(int64_t)a.blocks[0] * a.dim, (int64_t)a.blocks[1] * a.dim};
        SDP_TRY(take_ops_space(ctx, call, (size_t)(per[0] + per[1] + 4) * 4, s));
        a.side[0].partials = dweight[0] ? (float *)ctx->ops_space : nullptr;
        a.side[1].partials = dweight[1] ? (float *)ctx->ops_space + per[0] : nullptr;
    }
    HIP_TRY(sdpops::launch_qk(a, bf16, backward, s));
    if (sums) SDP_TRY(ops_mark(ctx, s));
    return SDP_OK;
}

// ---- grouped products -----------------------------------------------------------

int check_grouped(const char *call, sdp_ctx *ctx, const sdp_grouped_desc *d) {
    if (!ctx) return fail(SDP_ERR_INVALID_ARGUMENT, "context is NULL");
    if (!d) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: the description is NULL", call);
    if (d->rows < 0 || d->rows > INT32_MAX || d->in_features < 0 || d->out_features < 0)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: rows, in_features or out_features out of range", call);
    if (d->groups < 0 || d->groups > SDP_GROUPED_MAX_GROUPS)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: groups must be in 0..%d (got %d)", call, SDP_GROUPED_MAX_GROUPS,
                    d->groups);
    if (sdpops::product(d->groups, d->out_features, d->in_features) < 0)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: groups, out_features and in_features multiply to more than 2^60", call);
    if (!is_float_type(d->out_type) || !is_int_type(d->ends_type))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: out_type or ends_type is none of those allowed", call);
    return SDP_OK;
}

sdpops::GroupedArgs grouped_args(const sdp_grouped_desc *d) {
    sdpops::GroupedArgs a{};
    a.ends = d->ends;
    a.rows = d->rows;
    a.x_stride = d->x_stride;
    a.y_stride = d->y_stride;
    a.dx_stride = d->dx_stride;
    a.groups = d->groups;
    a.n_in = d->in_features;
    a.n_out = d->out_features;
    a.ends64 = d->ends_type == SDP_TYPE_I64;
    a.out_f32 = d->out_type == SDP_TYPE_F32;
    return a;
}

int check_grids(const char *call, const sdpops::GroupedArgs &a, bool forward, bool dx, bool dw) {
    if (!sdpops::grouped_fits(a, forward, dx, dw))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: more tiles than one launch takes", call);
    return SDP_OK;
}

// The products of a call, with the workspace that they need.
int run_grouped(sdp_ctx *ctx, const char *call, const sdpops::GroupedArgs &a, bool forward, bool dx, bool dw,
                hipStream_t s) {
    const size_t bytes = sdpops::grouped_workspace(a, forward, dx, dw);
    if (bytes > 0) SDP_TRY(take_ops_space(ctx, call, bytes, s));
    HIP_TRY(sdpops::launch_grouped(a, forward, dx, dw, ctx->ops_space, s));
    if (bytes > 0) SDP_TRY(ops_mark(ctx, s));
    return SDP_OK;
}

// ---- distillation ----------------------------------------------------------------

int distill_call(sdp_ctx *ctx, const char *call, const sdp_distill_desc *d, float *loss, float *lse,
                 const float *lse_in, const float *row_grad, void *dlogits, int64_t dlogits_stride, bool backward,
                 void *stream) {
    if (!ctx) return fail(SDP_ERR_INVALID_ARGUMENT, "context is NULL");
    if (!d) return fail(SDP_ERR_INVALID_ARGUMENT, "%s: the description is NULL", call);
    if (d->rows < 0 || d->rows > SDP_DISTILL_MAX_ROWS || d->vocab < 1)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: rows must be in 0..%d and vocab at least 1", call,
                    SDP_DISTILL_MAX_ROWS);
    if (d->teacher_k < 0 || d->teacher_k > SDP_DISTILL_MAX_K)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: teacher_k must be in 0..%d (got %d)", call, SDP_DISTILL_MAX_K,
                    d->teacher_k);
    if (!is_float_type(d->logit_type) || (d->teacher_k > 0 && !is_float_type(d->teacher_type)) ||
        ((d->teacher_k > 0 || d->labels) && !is_int_type(d->index_type)))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a type is none of those allowed", call);
    if (!std::isfinite(d->distill_weight) || !std::isfinite(d->label_weight))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: weights must be finite", call);
    if (!(d->temperature >= 1e-6 && d->temperature <= 1e6))
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: temperature must be in 1e-6..1e6", call);
    if (dlogits && !row_grad && d->rows > 0)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: a gradient needs row_grad", call);
    if (backward && !dlogits && d->rows > 0)
        return fail(SDP_ERR_INVALID_ARGUMENT, "%s: dlogits is NULL", call);
    const int64_t rows = d->rows, zsize = type_size(d->logit_type), isize = type_size(d->index_type);
    std::vector<Tensor> ts = {rows_of("logits", d->logits, rows, d->logit_stride, d->vocab, zsize, false)};
    std::vector<std::pair<int, int>> in_place;
    if (d->teacher_k > 0) {
        ts.push_back(dense("teacher_logits", d->teacher_logits, rows * d->teacher_k, type_size(d->teacher_type), false));
        ts.push_back(dense("teacher_index", d->teacher_index, rows * d->teacher_k, isize, false));
    }
    if (d->labels) ts.push_back(dense("labels", d->labels, rows, isize, false));
    if (backward) {
        ts.push_back(dense("lse", lse_in, 2 * rows, 4, false));
    } else {
        ts.push_back(dense("loss", loss, rows, 4, true));
        if (lse) ts.push_back(dense("lse", lse, 2 * rows, 4, true));
    }
    if (dlogits) {
        ts.push_back(dense("row_grad", row_grad, rows, 4, false));
        in_place.push_back({(int)ts.size(), 0});
        ts.push_back(rows_of("dlogits", dlogits, rows, dlogits_stride, d->vocab, zsize, true));
    }
    DeviceGuard guard(ctx->device);
    SDP_TRY(check_tensors(ctx, call, ts, in_place));

    sdpops::DistillArgs a{};
    a.logits = d->logits;
    a.logit_stride = d->logit_stride;
    a.rows = rows;
    a.vocab = d->vocab;
    a.k = d->teacher_k;
    a.teacher_logits = d->teacher_logits;
    a.teacher_index = d->teacher_index;
    a.labels = d->labels;
    a.teacher_bf16 = d->teacher_type == SDP_TYPE_BF16;
    a.index64 = d->index_type == SDP_TYPE_I64;
    a.tau = (float)d->temperature;
    a.inv_tau = (float)(1.0 / d->temperature);
    a.distill_weight = (float)d->distill_weight;
    a.label_weight = (float)d->label_weight;
    a.loss = loss;
    a.lse = lse;
    a.lse_in = lse_in;
    a.row_grad = row_grad;
    a.dlogits = dlogits;
    a.dlogits_stride = dlogits_stride;
    hipStream_t s = (hipStream_t)stream;
    const bool bf16 = d->logit_type == SDP_TYPE_BF16;
    if (backward) {
        HIP_TRY(sdpops::launch_distill_backward(a, bf16, s));
        return SDP_OK;
    }
    a.splits = sdpops::distill_splits(a, bf16);
    const bool parts = a.splits > 0 && rows > 0;
    if (parts) {
        SDP_TRY(take_ops_space(ctx, call, (size_t)rows * a.splits * sdpops::kDistillPartials * sizeof(float), s));
        a.partials = (float *)ctx->ops_space;
    }
    HIP_TRY(sdpops::launch_distill(a, bf16, s));
    if (parts) SDP_TRY(ops_mark(ctx, s));
    return SDP_OK;
}

}  // namespace

extern "C" {

int sdp_qk_norm_rope(sdp_ctx *ctx, const sdp_qk_norm_rope_desc *desc, const sdp_heads *q, const sdp_heads *k,
                     const sdp_heads *q_out, const sdp_heads *k_out, void *stream) {
    return guarded([&] {
        const sdp_heads *const x[2] = {q, k}, *const y[2] = {nullptr, nullptr}, *const out[2] = {q_out, k_out};
        void *const none[2] = {nullptr, nullptr};
        return qk_call(ctx, "sdp_qk_norm_rope", desc, x, y, out, none, false, stream);
    });
}

int sdp_qk_norm_rope_backward(sdp_ctx *ctx, const sdp_qk_norm_rope_desc *desc, const sdp_heads *q, const sdp_heads *k,
                              const sdp_heads *dq_out, const sdp_heads *dk_out, const sdp_heads *dq,
                              const sdp_heads *dk, void *dq_weight, void *dk_weight, void *stream) {
    return guarded([&] {
        const sdp_heads *const x[2] = {q, k}, *const y[2] = {dq_out, dk_out}, *const out[2] = {dq, dk};
        void *const dw[2] = {dq_weight, dk_weight};
        return qk_call(ctx, "sdp_qk_norm_rope_backward", desc, x, y, out, dw, true, stream);
    });
}

int sdp_grouped_matmul(sdp_ctx *ctx, const sdp_grouped_desc *desc, const uint16_t *x, const uint16_t *w, void *y,
                       void *stream) {
    return guarded([&] {
        const char *call = "sdp_grouped_matmul";
        SDP_TRY(check_grouped(call, ctx, desc));
        const int64_t in = desc->in_features, out = desc->out_features;
        sdpops::GroupedArgs a = grouped_args(desc);
        a.x = x;
        a.w = w;
        a.y = y;
        SDP_TRY(check_grids(call, a, true, false, false));
        DeviceGuard guard(ctx->device);
        SDP_TRY(check_tensors(ctx, call,
                              {rows_of("x", x, desc->rows, desc->x_stride, in, 2, false),
                               dense("w", w, desc->groups * out * in, 2, false),
                               dense("ends", desc->ends, desc->groups, type_size(desc->ends_type), false),
                               rows_of("y", y, desc->rows, desc->y_stride, out, type_size(desc->out_type), true)},
                              {}));
        return run_grouped(ctx, call, a, true, false, false, (hipStream_t)stream);
    });
}

int sdp_grouped_matmul_backward(sdp_ctx *ctx, const sdp_grouped_desc *desc, const uint16_t *x, const uint16_t *w,
                                const uint16_t *dy, uint16_t *dx, void *dw, void *stream) {
    return guarded([&] {
        const char *call = "sdp_grouped_matmul_backward";
        SDP_TRY(check_grouped(call, ctx, desc));
        const int64_t in = desc->in_features, out = desc->out_features;
        sdpops::GroupedArgs a = grouped_args(desc);
        a.x = x;
        a.w = w;
        a.dy = dy;
        a.dx = dx;
        a.dw = dw;
        SDP_TRY(check_grids(call, a, false, dx != nullptr, dw != nullptr));
        DeviceGuard guard(ctx->device);
        std::vector<Tensor> ts = {rows_of("dy", dy, desc->rows, desc->y_stride, out, 2, false),
                                  dense("ends", desc->ends, desc->groups, type_size(desc->ends_type), false)};
        if (dx) {
            ts.push_back(dense("w", w, desc->groups * out * in, 2, false));
            ts.push_back(rows_of("dx", dx, desc->rows, desc->dx_stride, in, 2, true));
        }
        if (dw) {
            ts.push_back(rows_of("x", x, desc->rows, desc->x_stride, in, 2, false));
            ts.push_back(dense("dw", dw, desc->groups * out * in, type_size(desc->out_type), true));
        }
        SDP_TRY(check_tensors(ctx, call, ts, {}));
        return run_grouped(ctx, call, a, false, dx != nullptr, dw != nullptr, (hipStream_t)stream);
    });
}

int sdp_distill_loss(sdp_ctx *ctx, const sdp_distill_desc *desc, float *loss, float *lse, const float *row_grad,
                     void *dlogits, int64_t dlogits_stride, void *stream) {
    return guarded([&] {
        return distill_call(ctx, "sdp_distill_loss", desc, loss, lse, nullptr, row_grad, dlogits, dlogits_stride,
                            false, stream);
    });
}

int sdp_distill_loss_backward(sdp_ctx *ctx, const sdp_distill_desc *desc, const float *lse, const float *row_grad,
                              void *dlogits, int64_t dlogits_stride, void *stream) {
    return guarded([&] {
        return distill_call(ctx, "sdp_distill_loss_backward", desc, nullptr, nullptr, lse, row_grad, dlogits,
                            dlogits_stride, true, stream);
    });
}

}  // extern "C"
