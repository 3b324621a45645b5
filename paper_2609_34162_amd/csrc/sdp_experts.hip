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
#include <type_traits>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"

namespace sdpops {
namespace {

constexpr int kWaves = 4;
constexpr int kColumns = 512;  // of a wave: eight to a lane

__device__ __forceinline__ int64_t all_waves() { return (int64_t)gridDim.x * kWaves; }

// The wave's items, one after the other.  (A division costs more than a piece of a row.)
__device__ __forceinline__ int64_t wave_index() {
    return (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

// A wave takes 1 KB of a token: copies of 16 bytes a lane, of any type.  size: of an element.
template <bool ONCE>
__global__ __launch_bounds__(64 * kWaves) void k_gather(ExpertArgs a, int slices, int size) {
    const int lane = threadIdx.x & 63;
    const int64_t n = a.tokens * a.top, bytes = (int64_t)a.hidden * size;
    for (int64_t w = wave_index(); w < a.tokens * slices; w += all_waves()) {
        const int64_t t = w / slices, c = (w - t * slices) * 1024 + lane * 16;
        const int left = (int)min(bytes - c, (int64_t)16);
        const char *x = (const char *)a.side.data + t * a.side.stride * size + c;
        u32x4 v = {0, 0, 0, 0};
        if (left == 16) v = load_any16<ONCE>(x);
        for (int j = 0; j < a.top; ++j) {
            const int32_t p = a.place[t * a.top + j];
            const int64_t row = p < 0 ? -1 - (int64_t)p : p;
            if (row >= n) continue;
            char *out = (char *)a.rows.data + row * a.rows.stride * size + c;
            if (left == 16) {
                store_any16<ONCE>(out, p < 0 ? u32x4{0, 0, 0, 0} : v);
            } else {
                for (int k = 0; k < left; k += 2) *(uint16_t *)(out + k) = p < 0 ? 0 : *(const uint16_t *)(x + k);
            }
        }
    }
}

// A wave takes 512 columns of a token; its lanes have the token's places and weights.
template <typename T, typename S, bool ONCE>
__global__ __launch_bounds__(64 * kWaves) void k_combine(ExpertArgs a, int slices) {
    constexpr int kAhead = 8;
    const int lane = threadIdx.x & 63;
    const int64_t n = a.tokens * a.top;
    for (int64_t w = wave_index(); w < a.tokens * slices; w += all_waves()) {
        const int64_t t = w / slices;
        const int c = (int)(w - t * slices) * kColumns + lane * 8, left = a.hidden - c;
        float sum[8] = {};
        bool lost = false;  // a place that names no row
        Eight<S> side = load_eight<ONCE>((const S *)a.side.data + t * a.side.stride + c, a.side.data ? left : 0);
        for (int j0 = 0; j0 < a.top; j0 += 64) {
            const int64_t mine = t * a.top + j0 + lane;
            const bool on = j0 + lane < a.top;
            const int32_t my_place = on ? a.place[mine] : -1;
            const float my_weight = on && a.weights ? load_either(a.weights, mine, a.weight_bf16) : 1.0f;
            const int count = min(64, a.top - j0);
            for (int j = 0; j < count; j += kAhead) {
                Eight<T> x[kAhead];
                bool there[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int32_t p = j + u < count ? __builtin_amdgcn_readlane(my_place, (j + u) & 63) : -1;
                    there[u] = p >= 0;
                    x[u] = load_eight<ONCE>((const T *)a.rows.data + p * a.rows.stride + c, p >= 0 && p < n ? left : 0);
                    lost = lost || p >= n;
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    if (!there[u]) continue;
                    const float weight =
                        __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_weight), (j + u) & 63));
                    float v[8];
                    x[u].floats(v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] += weight * v[k];
                }
            }
        }
        float v[8];
        side.floats(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] = lost ? __builtin_nanf("") : sum[k] + v[k];
        store_floats<ONCE>((S *)a.out.data + t * a.out.stride + c, left, sum);
    }
}

// A wave takes an entry.
template <typename T, typename S>
__global__ __launch_bounds__(64 * kWaves) void k_combine_back(ExpertArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t n = a.tokens * a.top;
    for (int64_t e = wave_index(); e < n; e += all_waves()) {
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

// Whether a call's data are past the last-level cache.
bool past_cache(int64_t bytes) { return bytes > (int64_t)256 << 20; }

uint32_t grid_of(int64_t waves) { return (uint32_t)std::min<int64_t>((waves + kWaves - 1) / kWaves, 1 << 20); }

}  // namespace

hipError_t launch_gather(const ExpertArgs &a, bool row_bf16, hipStream_t s) {
    const int size = row_bf16 ? 2 : 4, slices = (int)(((int64_t)a.hidden * size + 1023) / 1024);
    const int64_t waves = a.tokens * slices;
    if (waves == 0 || a.top == 0) return hipSuccess;
    const dim3 grid(grid_of(waves)), block(64 * kWaves);
    if (past_cache(a.tokens * (a.top + 1) * a.hidden * size))
        hipLaunchKernelGGL((k_gather<true>), grid, block, 0, s, a, slices, size);
    else
        hipLaunchKernelGGL((k_gather<false>), grid, block, 0, s, a, slices, size);
    return hipGetLastError();
}

hipError_t launch_combine(const ExpertArgs &a, bool row_bf16, bool stream_bf16, hipStream_t s) {
    const int slices = a.hidden / kColumns + (a.hidden % kColumns != 0);
    const int64_t waves = a.tokens * slices;
    if (waves == 0) return hipSuccess;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid_of(waves)), dim3(64 * kWaves), 0, s, a, slices);
    };
    const bool once = past_cache(a.tokens * a.hidden * ((int64_t)a.top * (row_bf16 ? 2 : 4) + (stream_bf16 ? 4 : 8)));
    auto pick = [&](auto is_once) {
        constexpr bool O = decltype(is_once)::value;
        if (row_bf16)
            stream_bf16 ? go(k_combine<uint16_t, uint16_t, O>) : go(k_combine<uint16_t, float, O>);
        else
            stream_bf16 ? go(k_combine<float, uint16_t, O>) : go(k_combine<float, float, O>);
    };
    once ? pick(std::true_type()) : pick(std::false_type());
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
