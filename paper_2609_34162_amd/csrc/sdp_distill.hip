// gfx950 kernels of sdp_distill_loss and its backward.
//
// A row needs max z and the two sums S_tau = sum exp((z - max) / tau) and
// S_1 = sum exp(z - max) (one where tau = 1), then its loss from a few
// gathered logits, and its gradient
//   g (a tau (exp(z / tau - L_tau) - q) + b (exp(z - L_1) - [label]))
// HBM bounds it: each logit is read once and each gradient written once.
#include "sdp_ops_device.h"
#include "sdp_ops_internal.h"

namespace sdpops {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// max of z and the sums of exp((z - max) / tau) and exp(z - max) over what
// was seen; max = -inf (nothing but -inf) goes with sums of 0.
struct Stats {
    float top, s_tau, s_one;
};

__device__ __forceinline__ Stats nothing() { return {kNegInf, 0.0f, 0.0f}; }

// Sums of a shifted to another maximum; a part that saw nothing adds nothing.
__device__ __forceinline__ Stats join(Stats a, Stats b, float inv_tau) {
    const float top = fmaxf(a.top, b.top);
    const float ref = top == kNegInf ? 0.0f : top;
    const float da = a.top - ref, db = b.top - ref;
    return {top, a.s_tau * exp_of(da * inv_tau) + b.s_tau * exp_of(db * inv_tau),
            a.s_one * exp_of(da) + b.s_one * exp_of(db)};
}

__device__ __forceinline__ void add(Stats &st, float z, float inv_tau) {
    if (!(z <= st.top)) st = join(st, {z, 0.0f, 0.0f}, inv_tau);
    const float d = z - (st.top == kNegInf ? 0.0f : st.top);
    st.s_tau += exp_of(d * inv_tau);
    st.s_one += exp_of(d);
}

// The teacher's side of a row, in LDS: entries that are there, and their q.
template <int kMax>
struct Teacher {
    int32_t index[kMax];
    float q[kMax];     // t / tau, then q
    float log_q[kMax];
    float z[kMax];
};

constexpr int kThreads = 256;

template <bool SUM>
__device__ float block_reduce(float v, float *scratch) {
    v = SUM ? wave_sum(v) : wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = scratch[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) r = SUM ? r + scratch[w] : fmaxf(r, scratch[w]);
    return r;
}

// One block walks one row: statistics, loss, gradient.
template <typename T, bool BACK>
__global__ __launch_bounds__(kThreads) void k_distill_rows(DistillArgs a) {
    __shared__ Teacher<SDP_DISTILL_MAX_K> t;
    __shared__ float scratch[kThreads / 64];
    __shared__ Stats waves[kThreads / 64];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T *z = (const T *)a.logits + row * a.logit_stride;
    const int K = a.k;

    // the teacher's softmax over the entries that are there
    float top = kNegInf, bad = 0.0f;
    for (int j = tid; j < K; j += kThreads) {
        const int64_t idx = load_int(a.teacher_index, row * K + j, a.index64);
        const bool there = idx >= 0;
        if (there && idx >= a.vocab) bad = 1.0f;
        t.index[j] = there && idx < a.vocab ? (int)idx : -1;
        t.q[j] = there ? load_either(a.teacher_logits, row * K + j, a.teacher_bf16) * a.inv_tau : kNegInf;
        top = fmaxf(top, t.q[j]);
    }
    top = block_reduce<false>(top, scratch);
    bad = block_reduce<false>(bad, scratch);
    float sum = 0.0f;
    const float ref = top == kNegInf ? 0.0f : top;
    for (int j = tid; j < K; j += kThreads) sum += exp_of(t.q[j] - ref);
    sum = block_reduce<true>(sum, scratch);
    const float log_sum = logf(sum) + ref;
    const bool has_teacher = a.distill_weight != 0.0f && (top != kNegInf || sum != 0.0f);
    int64_t label = a.labels && a.label_weight != 0.0f ? load_int(a.labels, row, a.index64) : -1;
    if (label >= a.vocab) bad = 1.0f, label = -1;
    const bool has_label = label >= 0;
    for (int j = tid; j < K; j += kThreads) {
        t.log_q[j] = t.q[j] - log_sum;
        t.q[j] = t.q[j] == kNegInf ? 0.0f : exp_of(t.log_q[j]);
        t.z[j] = t.index[j] >= 0 ? load1(z + t.index[j]) : 0.0f;
    }
    const float z_label = has_label ? load1(z + label) : 0.0f;

    float l_tau, l_one;
    if (BACK) {
        l_tau = a.lse_in[2 * row];
        l_one = a.lse_in[2 * row + 1];
    } else {
        Stats st = nothing();
        for (int64_t v = tid; v < a.vocab; v += kThreads) add(st, load1(z + v), a.inv_tau);
        for (int d = 32; d > 0; d >>= 1)
            st = join(st, {__shfl_xor(st.top, d), __shfl_xor(st.s_tau, d), __shfl_xor(st.s_one, d)}, a.inv_tau);
        if ((tid & 63) == 0) waves[tid >> 6] = st;
        __syncthreads();
        st = waves[0];
        for (int w = 1; w < kThreads / 64; ++w) st = join(st, waves[w], a.inv_tau);
        l_tau = logf(st.s_tau) + st.top * a.inv_tau;
        l_one = logf(st.s_one) + st.top;
        float kl = 0.0f;
        for (int j = tid; j < K; j += kThreads)
            if (t.q[j] > 0.0f || t.q[j] != t.q[j])
                kl += t.q[j] * (t.log_q[j] - (t.z[j] * a.inv_tau - l_tau));
        kl = block_reduce<true>(kl, scratch);
        if (tid == 0) {
            float loss = 0.0f;
            if (has_teacher) loss = a.distill_weight * a.tau * a.tau * kl;
            if (has_label) loss += a.label_weight * (l_one - z_label);
            a.loss[row] = bad != 0.0f ? __builtin_nanf("") : loss;
            if (a.lse) {
                a.lse[2 * row] = l_tau;
                a.lse[2 * row + 1] = l_one;
            }
        }
    }
    if (!a.dlogits) return;

    // the gradient: every z_j is in LDS, so dlogits may be logits itself
    T *dz = (T *)a.dlogits + row * a.dlogits_stride;
    const float g = bad != 0.0f ? __builtin_nanf("") : a.row_grad[row];
    const float c_tau = has_teacher || bad != 0.0f ? g * a.distill_weight * a.tau : 0.0f;
    const float c_one = has_label || bad != 0.0f ? g * a.label_weight : 0.0f;
    auto plain = [&](float x) {
        float d = 0.0f;
        if (c_tau != 0.0f) d = c_tau * exp_of(x * a.inv_tau - l_tau);
        if (c_one != 0.0f) d += c_one * exp_of(x - l_one);
        return d;
    };
    __syncthreads();
    for (int64_t v = tid; v < a.vocab; v += kThreads) store1(dz + v, plain(load1(z + v)));
    __syncthreads();
    // the elements that the teacher or the label names, over what the walk wrote
    for (int j = tid; j < K + 1; j += kThreads) {
        const int64_t at = j < K ? t.index[j] : label;
        if (at < 0) continue;
        float d = plain(j < K ? t.z[j] : z_label);
        if (c_tau != 0.0f) {
            float q = 0.0f;
            for (int i = 0; i < K; ++i) q += t.index[i] == (int)at ? t.q[i] : 0.0f;
            d -= c_tau * q;
        }
        if (at == label) d -= c_one;
        store1(dz + at, d);
    }
}

}  // namespace

int distill_splits(const DistillArgs &, bool) { return 1; }

hipError_t launch_distill(const DistillArgs &a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    if (bf16)
        hipLaunchKernelGGL((k_distill_rows<uint16_t, false>), dim3((uint32_t)a.rows), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((k_distill_rows<float, false>), dim3((uint32_t)a.rows), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_distill_backward(const DistillArgs &a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    if (bf16)
        hipLaunchKernelGGL((k_distill_rows<uint16_t, true>), dim3((uint32_t)a.rows), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((k_distill_rows<float, true>), dim3((uint32_t)a.rows), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace sdpops
