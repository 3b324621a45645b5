// gfx950 kernels of sdp_expert_gather, sdp_expert_combine and their backward.
//
// Every one goes from the tokens' side, where place[t, j] says which row belongs to
// entry j of token t (-1 - p: entry without an expert, matched with row p past the
// last end):
//   gather:    rows[p] = x[t];        its backward: dx[t] = sum over j of drows[p]
//   combine:   out[t] = residual[t] + sum over j of w_j rows[p]
//   backward:  drows[p] = w_j dout[t],  dw_j = <dout[t], rows[p]>
// so that a token's row is read or written once and each sorted row once: memory
// bounds all of them.
#include <algorithm>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"

namespace sdpops {
namespace {

constexpr int kWaves = 4;
constexpr int kColumns = 512;  // of a wave: eight to a lane

__device__ __forceinline__ int64_t first_wave() { return (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); }
__device__ __forceinline__ int64_t all_waves() { return (int64_t)gridDim.x * kWaves; }

// A wave takes 512 columns of a token; T an integer of the rows' element size.
template <typename T>
__global__ __launch_bounds__(64 * kWaves) void k_gather(ExpertArgs a, int slices) {
    const int lane = threadIdx.x & 63;
    const int64_t n = a.tokens * a.top;
    for (int64_t w = first_wave(); w < a.tokens * slices; w += all_waves()) {
        const int64_t t = w / slices;
        const int c = (int)(w - t * slices) * kColumns + lane * 8, left = a.hidden - c;
        if (left <= 0) continue;
        const T *x = (const T *)a.side.data + t * a.side.stride + c;
        for (int j = 0; j < a.top; ++j) {
            const int32_t p = a.place[t * a.top + j];
            const int64_t row = p < 0 ? -1 - (int64_t)p : p;
            if (row >= n) continue;
            T *out = (T *)a.rows.data + row * a.rows.stride + c;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) out[k] = p < 0 ? T(0) : x[k];
        }
    }
}

template <typename T, typename S>
__global__ __launch_bounds__(64 * kWaves) void k_combine(ExpertArgs a, int slices) {
    const int lane = threadIdx.x & 63;
    const int64_t n = a.tokens * a.top;
    for (int64_t w = first_wave(); w < a.tokens * slices; w += all_waves()) {
        const int64_t t = w / slices;
        const int c = (int)(w - t * slices) * kColumns + lane * 8, left = a.hidden - c;
        if (left <= 0) continue;
        float sum[8] = {};
        for (int j = 0; j < a.top; ++j) {
            const int32_t p = a.place[t * a.top + j];
            if (p < 0) continue;
            const float weight = a.weights ? load_either(a.weights, t * a.top + j, a.weight_bf16) : 1.0f;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __builtin_nanf("");
            if (p < n) load_floats((const T *)a.rows.data + p * a.rows.stride + c, left, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += weight * v[k];
        }
        if (a.side.data) {
            float v[8];
            load_floats((const S *)a.side.data + t * a.side.stride + c, left, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += v[k];
        }
        store_floats((S *)a.out.data + t * a.out.stride + c, left, sum);
    }
}

// A wave takes an entry.
template <typename T, typename S>
__global__ __launch_bounds__(64 * kWaves) void k_combine_back(ExpertArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t n = a.tokens * a.top;
    for (int64_t e = first_wave(); e < n; e += all_waves()) {
        const int32_t p = a.place[e];
        const int64_t row = p < 0 ? -1 - (int64_t)p : p;
        const float weight = a.drows.data && p >= 0 ? load_either(a.weights, e, a.weight_bf16) : 0.0f;
        const S *d = (const S *)a.side.data + e / a.top * a.side.stride;
        float dot = 0.0f;
        if (row < n) {
            for (int c = lane * 8; c < a.hidden; c += kColumns) {
                const int left = a.hidden - c;
                float v[8], x[8];
                load_floats(d + c, left, v);
                if (a.dweights && p >= 0) {
                    load_floats((const T *)a.rows.data + row * a.rows.stride + c, left, x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) dot += v[k] * x[k];
                }
                if (a.drows.data) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = p < 0 ? 0.0f : weight * v[k];
                    store_floats((T *)a.drows.data + row * a.drows.stride + c, left, v);
                }
            }
        } else if (p >= 0) {
            dot = __builtin_nanf("");
        }
        if (a.dweights) {
            dot = wave_sum(dot);
            if (lane == 0) {
                if (a.weight_bf16)
                    store1((uint16_t *)a.dweights + e, dot);
                else
                    ((float *)a.dweights)[e] = dot;
            }
        }
    }
}

uint32_t grid_of(int64_t waves) { return (uint32_t)std::min<int64_t>((waves + kWaves - 1) / kWaves, 1 << 20); }

}  // namespace

hipError_t launch_gather(const ExpertArgs &a, bool row_bf16, hipStream_t s) {
    const int slices = a.hidden / kColumns + (a.hidden % kColumns != 0);
    const int64_t waves = a.tokens * slices;
    if (waves == 0 || a.top == 0) return hipSuccess;
    if (row_bf16)
        hipLaunchKernelGGL((k_gather<uint16_t>), dim3(grid_of(waves)), dim3(64 * kWaves), 0, s, a, slices);
    else
        hipLaunchKernelGGL((k_gather<uint32_t>), dim3(grid_of(waves)), dim3(64 * kWaves), 0, s, a, slices);
    return hipGetLastError();
}

hipError_t launch_combine(const ExpertArgs &a, bool row_bf16, bool stream_bf16, hipStream_t s) {
    const int slices = a.hidden / kColumns + (a.hidden % kColumns != 0);
    const int64_t waves = a.tokens * slices;
    if (waves == 0) return hipSuccess;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid_of(waves)), dim3(64 * kWaves), 0, s, a, slices); };
    if (row_bf16)
        stream_bf16 ? go(k_combine<uint16_t, uint16_t>) : go(k_combine<uint16_t, float>);
    else
        stream_bf16 ? go(k_combine<float, uint16_t>) : go(k_combine<float, float>);
    return hipGetLastError();
}

hipError_t launch_combine_backward(const ExpertArgs &a, bool row_bf16, bool stream_bf16, hipStream_t s) {
    const int64_t n = a.tokens * a.top;
    if (n == 0) return hipSuccess;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid_of(n)), dim3(64 * kWaves), 0, s, a); };
    if (row_bf16)
        stream_bf16 ? go(k_combine_back<uint16_t, uint16_t>) : go(k_combine_back<uint16_t, float>);
    else
        stream_bf16 ? go(k_combine_back<float, uint16_t>) : go(k_combine_back<float, float>);
    return hipGetLastError();
}

}  // namespace sdpops
