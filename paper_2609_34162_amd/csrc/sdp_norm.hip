// gfx950 kernels of sdp_block_norm and its backward.
//
// For a token's rows, ry = 1 / rms(y), r = 1 / rms(h_out), w the weights with their
// offset and a the gate:
//   u = y ry w_post;  h_out = h + s a u;  n = h_out r w_pre
// and backward, with v = dn w_pre and mean over the channels:
//   g = dh_out + r (v - h_out r^2 mean(v h_out));  dh = g;  du = s a g
//   dy = ry (du w_post - y ry^2 mean(du w_post y));  dgate = s u g (times a (1 - a))
//   dw_pre = sum of dn h_out r;  dw_post = sum of du y ry
// Memory bounds both: each tensor is read once and written once.
#include <algorithm>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"

namespace sdpops {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float weight_at(const NormArgs &a, const void *w, int64_t i) {
    return w ? a.offset + load_either(w, i, a.weight_bf16) : 1.0f;
}

// The gate of an element, and its slope by the gate's input.
template <typename T>
__device__ __forceinline__ float gate_at(const NormArgs &a, int64_t t, int64_t i, float *slope) {
    *slope = 1.0f;
    if (a.gate_form == SDP_GATE_NONE) return 1.0f;
    const int64_t at = a.gate_form == SDP_GATE_CHANNEL ? i : t * a.gate_stride + (a.gate_form == SDP_GATE_ELEMENT ? i : 0);
    const float z = load1((const T *)a.gate + at);
    if (!a.sigmoid) return z;
    const float g = 1.0f / (1.0f + expf(-z));
    *slope = g * (1.0f / (1.0f + expf(z)));
    return g;
}

__device__ __forceinline__ float block_sum(float v, float *waves) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
    for (int w = 0; w < kThreads / 64; ++w) v += waves[w];
    return v;
}

// Any size: a block takes a row, a thread its columns a block apart, and the row is
// read again for each step.
template <typename S, typename T>
__global__ __launch_bounds__(kThreads) void k_norm_any(NormArgs a) {
    __shared__ float waves[kThreads / 64];
    const float inv = 1.0f / (float)a.hidden;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const S *h = (const S *)a.h.data + t * a.h.stride;
        const T *y = a.y.data ? (const T *)a.y.data + t * a.y.stride : nullptr;
        float ry = 1.0f;
        if (y && a.post_norm) {
            float sq = 0.0f;
            for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads) {
                const float v = load1(y + i);
                sq += v * v;
            }
            ry = rsqrtf(block_sum(sq, waves) * inv + a.eps);
        }
        auto sum_at = [&](int64_t i) {
            float v = load1(h + i), slope;
            if (y) {
                const float u = a.post_norm ? load1(y + i) * ry * weight_at(a, a.post_weight, i) : load1(y + i);
                v += a.scale * gate_at<T>(a, t, i, &slope) * u;
            }
            return v;
        };
        float r = 0.0f;
        if (a.n_out.data) {
            float sq = 0.0f;
            for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads) {
                const float v = sum_at(i);
                sq += v * v;
            }
            r = rsqrtf(block_sum(sq, waves) * inv + a.eps);
        }
        for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads) {
            const float v = sum_at(i);
            if (a.h_out.data) store1((S *)a.h_out.data + t * a.h_out.stride + i, v);
            if (a.n_out.data) store1((T *)a.n_out.data + t * a.n_out.stride + i, v * r * weight_at(a, a.pre_weight, i));
        }
        __syncthreads();
    }
}

__device__ __forceinline__ int64_t sums_stride(const NormArgs &a) { return ((int64_t)a.hidden + 3) / 4 * 4; }

template <typename S, typename T>
__global__ __launch_bounds__(kThreads) void k_norm_back_any(NormArgs a) {
    __shared__ float waves[kThreads / 64];
    const float inv = 1.0f / (float)a.hidden;
    float *sums[3];
    for (int k = 0; k < 3; ++k) {
        sums[k] = a.sums[k] ? a.sums[k] + blockIdx.x * sums_stride(a) : nullptr;
        if (sums[k])
            for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads) sums[k][i] = 0.0f;
    }
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const S *h = a.h.data ? (const S *)a.h.data + t * a.h.stride : nullptr;
        const T *y = a.y.data ? (const T *)a.y.data + t * a.y.stride : nullptr;
        const T *dn = a.dn.data ? (const T *)a.dn.data + t * a.dn.stride : nullptr;
        const S *dh_out = a.dh_out.data ? (const S *)a.dh_out.data + t * a.dh_out.stride : nullptr;
        float hh = 0.0f, vh = 0.0f, yy = 0.0f;
        for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads) {
            if (dn) {
                const float x = load1(h + i);
                hh += x * x;
                vh += load1(dn + i) * weight_at(a, a.pre_weight, i) * x;
            }
            if (y && a.post_norm) {
                const float x = load1(y + i);
                yy += x * x;
            }
        }
        float r = 0.0f, along = 0.0f, ry = 1.0f;
        if (dn) {
            r = rsqrtf(block_sum(hh, waves) * inv + a.eps);
            along = block_sum(vh, waves) * inv * r * r;
        }
        if (y && a.post_norm) ry = rsqrtf(block_sum(yy, waves) * inv + a.eps);
        auto g_at = [&](int64_t i) {
            float g = dh_out ? load1(dh_out + i) : 0.0f;
            if (dn) g += r * (load1(dn + i) * weight_at(a, a.pre_weight, i) - load1(h + i) * along);
            return g;
        };
        float dot = 0.0f;
        if (a.post_norm && a.dy.data) {
            for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads) {
                float slope;
                dot += a.scale * gate_at<T>(a, t, i, &slope) * g_at(i) * weight_at(a, a.post_weight, i) * load1(y + i);
            }
            dot = block_sum(dot, waves) * inv * ry * ry;
        }
        float gate_sum = 0.0f;
        for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads) {
            const float g = g_at(i);
            float slope;
            const float du = a.scale * gate_at<T>(a, t, i, &slope) * g;
            const float x = y ? load1(y + i) : 0.0f, w = a.post_norm ? weight_at(a, a.post_weight, i) : 1.0f;
            if (sums[0]) sums[0][i] += load1(dn + i) * load1(h + i) * r;
            if (sums[1]) sums[1][i] += du * x * ry;
            if (a.dgate) {
                const float d = a.scale * (x * ry * w) * g * slope;
                if (sums[2]) sums[2][i] += d;
                if (a.gate_form == SDP_GATE_ELEMENT) store1((T *)a.dgate + t * a.dgate_stride + i, d);
                gate_sum += d;
            }
            if (a.dh.data) store1((S *)a.dh.data + t * a.dh.stride + i, g);
            if (a.dy.data) {
                const float d = a.post_norm ? ry * (du * w - x * dot) : du;
                store1((T *)a.dy.data + t * a.dy.stride + i, d);
            }
        }
        if (a.dgate && a.gate_form == SDP_GATE_TOKEN) {
            gate_sum = block_sum(gate_sum, waves);
            if (threadIdx.x == 0) store1((T *)a.dgate + t * a.dgate_stride, gate_sum);
        }
        __syncthreads();
    }
}

// The blocks' partial sums, added in their order.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_sums(NormArgs a) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= a.hidden) return;
    for (int k = 0; k < 3; ++k) {
        if (!a.sums[k]) continue;
        float s = 0.0f;
        for (int b = 0; b < a.blocks; ++b) s += a.sums[k][b * sums_stride(a) + i];
        if (k == 2)
            store1((T *)a.dgate + i, s);
        else if (a.weight_bf16)
            store1((uint16_t *)(k ? a.dpost : a.dpre) + i, s);
        else
            ((float *)(k ? a.dpost : a.dpre))[i] = s;
    }
}

template <typename F>
void with_types(bool stream_bf16, bool bf16, F &&go) {
    if (stream_bf16)
        bf16 ? go((uint16_t *)nullptr, (uint16_t *)nullptr) : go((uint16_t *)nullptr, (float *)nullptr);
    else
        bf16 ? go((float *)nullptr, (uint16_t *)nullptr) : go((float *)nullptr, (float *)nullptr);
}

}  // namespace

int norm_blocks(const NormArgs &a) { return (int)std::min<int64_t>(a.tokens, 1024); }

hipError_t launch_norm(const NormArgs &a, bool stream_bf16, bool bf16, hipStream_t s) {
    const dim3 grid((uint32_t)std::min<int64_t>(a.tokens, 1 << 20));
    with_types(stream_bf16, bf16, [&](auto *st, auto *ty) {
        using S = std::remove_pointer_t<decltype(st)>;
        using T = std::remove_pointer_t<decltype(ty)>;
        hipLaunchKernelGGL((k_norm_any<S, T>), grid, dim3(kThreads), 0, s, a);
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormArgs &a, bool stream_bf16, bool bf16, hipStream_t s) {
    if (a.blocks > 0)
        with_types(stream_bf16, bf16, [&](auto *st, auto *ty) {
            using S = std::remove_pointer_t<decltype(st)>;
            using T = std::remove_pointer_t<decltype(ty)>;
            hipLaunchKernelGGL((k_norm_back_any<S, T>), dim3(a.blocks), dim3(kThreads), 0, s, a);
        });
    if (a.sums[0] || a.sums[1] || a.sums[2]) {
        const dim3 grid((a.hidden - 1) / kThreads + 1);
        if (bf16)
            hipLaunchKernelGGL((k_norm_sums<uint16_t>), grid, dim3(kThreads), 0, s, a);
        else
            hipLaunchKernelGGL((k_norm_sums<float>), grid, dim3(kThreads), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace sdpops
