// gfx950 kernels of sdp_expert_gather, sdp_expert_combine and their backward.
//
// Every one goes from the tokens' side, where place[t, j] says which row belongs to
// entry j of token t (-1 - p: entry without an expert, matched with row p past the
// last end):
//   gather:    rows[p] = x[t];        its backward: dx[t] = sum over j of drows[p]
//   combine:   out[t] = residual[t] + sum over j of w_j rows[p]
//   backward:  drows[p] = w_j dout[t],  dw_j = <dout[t], rows[p]>
// so that a token's row is read or written once and each sorted row once: memory
// bounds all of them, at 4.9 to 5.2 TB/s for 8,192 tokens' 8 rows of 2,048 BF16 channels
// (gather 62 us, combine 60, its gradient 116).
#include <algorithm>
#include <type_traits>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"

namespace sdpops {
namespace {

constexpr int kWaves = 4;

__device__ __forceinline__ int64_t all_waves() { return (int64_t)gridDim.x * kWaves; }
__device__ __forceinline__ int64_t wave_index() {
    return (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

// Teams of LANES lanes take 16-byte pieces (or eight elements a lane) of a row: a slice of
// it each, one wave's teams the slices one after the other.  (A division by lanes costs
// more than a piece of a row.)
struct Item {
    int64_t row;
    int slice;
};
template <int LANES>
__device__ __forceinline__ Item item_of(int64_t wave, int slices) {
    constexpr int kTeams = 64 / LANES;
    Item o = {wave * kTeams / slices, 0};
    o.slice = (int)(wave * kTeams - o.row * slices);
    if (LANES == 64) return o;
    o.slice += (threadIdx.x & 63) / LANES;
#pragma unroll
    for (int k = 1; k < kTeams; ++k)
        if (o.slice >= slices) o.slice -= slices, ++o.row;
    return o;
}

// v of the team's i-th lane.
template <int LANES, typename V>
__device__ __forceinline__ V of_lane(V v, int i) {
    if (LANES < 64) return __shfl(v, i & (LANES - 1), LANES);
    const uint32_t bits = __builtin_amdgcn_readlane(__builtin_bit_cast(uint32_t, v), i & 63);
    return __builtin_bit_cast(V, bits);
}

// Copies of 16 bytes a lane, of any type; the last of a row begin early enough to be whole.
// size: of an element.
template <int LANES, bool ONCE>
__global__ __launch_bounds__(64 * kWaves) void k_gather(ExpertArgs a, int slices, int size) {
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t n = a.tokens * a.top, bytes = (int64_t)a.hidden * size;
    for (int64_t w = wave_index(); w * (64 / LANES) < a.tokens * slices; w += all_waves()) {
        const Item item = item_of<LANES>(w, slices);
        const int64_t t = item.row, at = ((int64_t)item.slice * LANES + lane) * 16;
        const bool on = LANES == 64 || t < a.tokens;
        const int left = on && at < bytes ? (int)min(bytes, (int64_t)16) : 0;
        const int64_t c = min(at, max(bytes - 16, (int64_t)0));
        const char *x = (const char *)a.side.data + t * a.side.stride * size + c;
        u32x4 v = {0, 0, 0, 0};
        if (left == 16) v = load_any16<ONCE>(x);
        for (int j0 = 0; j0 < a.top; j0 += LANES) {
            const int32_t my_place = on && j0 + lane < a.top ? a.place[t * a.top + j0 + lane] : 0;
            for (int j = 0; j < min(LANES, a.top - j0); ++j) {
                const int32_t p = of_lane<LANES>(my_place, j);
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
}

// A team takes a slice of a token; its lanes have the token's places and weights.
template <int LANES, typename T, typename S, bool ONCE>
__global__ __launch_bounds__(64 * kWaves) void k_combine(ExpertArgs a, int slices) {
    constexpr int kAhead = 8;
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t n = a.tokens * a.top;
    for (int64_t w = wave_index(); w * (64 / LANES) < a.tokens * slices; w += all_waves()) {
        const Item item = item_of<LANES>(w, slices);
        const int64_t t = item.row;
        const bool on = LANES == 64 || t < a.tokens;
        const int c = (item.slice * LANES + lane) * 8, left = on ? a.hidden - c : 0;
        float sum[8] = {};
        bool lost = false;  // a place that names no row
        Eight<S> side = load_eight<ONCE>((const S *)a.side.data + t * a.side.stride + c, a.side.data ? left : 0);
        for (int j0 = 0; j0 < a.top; j0 += LANES) {
            const int64_t mine = t * a.top + j0 + lane;
            const bool has = on && j0 + lane < a.top;
            const int32_t my_place = has ? a.place[mine] : -1;
            const float my_weight = has && a.weights ? load_either(a.weights, mine, a.weight_bf16) : 1.0f;
            const int count = min(LANES, a.top - j0);
            for (int j = 0; j < count; j += kAhead) {
                Eight<T> x[kAhead];
                bool there[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int32_t p = j + u < count ? of_lane<LANES>(my_place, j + u) : -1;
                    there[u] = p >= 0;
                    x[u] = load_eight<ONCE>((const T *)a.rows.data + p * a.rows.stride + c, p >= 0 && p < n ? left : 0);
                    lost = lost || p >= n;
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    if (LANES == 64 && !there[u]) continue;
                    const float weight = of_lane<LANES>(my_weight, j + u);
                    float v[8];
                    x[u].floats(v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] += LANES == 64 || there[u] ? weight * v[k] : 0.0f;
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

// A team takes an entry, and loads two pieces of a lane before either is worked on.
template <int LANES, typename T, typename S>
__global__ __launch_bounds__(64 * kWaves) void k_combine_back(ExpertArgs a) {
    constexpr int kStep = LANES * 8;
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t n = a.tokens * a.top;
    for (int64_t w = wave_index(); w * (64 / LANES) < n; w += all_waves()) {
        const Item item = item_of<LANES>(w, a.top);  // (an entry is a token's slice)
        const int64_t t = item.row, e = t * a.top + item.slice;
        if (LANES < 64 && e >= n) continue;
        const int32_t p = a.place[e];
        const int64_t row = p < 0 ? -1 - (int64_t)p : p;
        const float weight = a.drows.data && p >= 0 ? load_either(a.weights, e, a.weight_bf16) : 0.0f;
        const S *d = (const S *)a.side.data + t * a.side.stride;
        const bool dots = a.dweights && p >= 0;
        float dot = 0.0f;
        if (row < n) {
            for (int c0 = lane * 8; c0 < a.hidden; c0 += 2 * kStep) {
                Eight<S> side[2];
                Eight<T> of_row[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int c = c0 + u * kStep, left = a.hidden - c;
                    side[u] = load_eight<false>(d + c, left);
                    of_row[u] = load_eight<false>((const T *)a.rows.data + row * a.rows.stride + c, dots ? left : 0);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int c = c0 + u * kStep, left = a.hidden - c;
                    float v[8], x[8];
                    side[u].floats(v);
                    of_row[u].floats(x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) dot += dots ? v[k] * x[k] : 0.0f;
                    if (a.drows.data) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = p < 0 ? 0.0f : weight * v[k];
                        store_floats((T *)a.drows.data + row * a.drows.stride + c, left, v);
                    }
                }
            }
        } else if (p >= 0) {
            dot = __builtin_nanf("");
        }
        if (a.dweights) {
            dot = lanes_sum(dot, LANES);
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

// The most lanes of a team that leave at most an eighth of themselves idle over a row's
// pieces (14,235 tokens x 6 of 550 BF16 channels in teams of 16 and of 64: the gradient
// 61 us and 79, the gather with the entries' order 44 and 61).  Where the lanes add up
// rows (combine), that costs registers that only rows within one team are worth: 67 us, of
// 64 lanes 53, but 27,000 x 2 of 208 19 us and 24.
int lanes_of(int64_t pieces, bool sums_rows = false) {
    for (int lanes = 64; lanes > 16; lanes /= 2) {
        if (sums_rows ? pieces > lanes / 2 : (-pieces & (lanes - 1)) * 8 <= pieces + (-pieces & (lanes - 1)))
            return lanes;
    }
    return 16;
}

dim3 grid_of(int64_t teams, int lanes) {
    const int64_t per = 64 / lanes * kWaves;
    return dim3((uint32_t)std::min<int64_t>((teams + per - 1) / per, 1 << 20));
}

template <typename F>
void with_lanes(int lanes, F &&go) {
    switch (lanes) {
        case 64: go(std::integral_constant<int, 64>()); break;
        case 32: go(std::integral_constant<int, 32>()); break;
        default: go(std::integral_constant<int, 16>()); break;
    }
}

template <typename F>
void with_types(bool row_bf16, bool stream_bf16, F &&go) {
    if (row_bf16)
        stream_bf16 ? go(uint16_t(), uint16_t()) : go(uint16_t(), float());
    else
        stream_bf16 ? go(float(), uint16_t()) : go(float(), float());
}

}  // namespace

hipError_t launch_gather(const ExpertArgs &a, bool row_bf16, hipStream_t s) {
    const int size = row_bf16 ? 2 : 4;
    const int64_t pieces = ((int64_t)a.hidden * size + 15) / 16;
    const int lanes = lanes_of(pieces), slices = (int)((pieces + lanes - 1) / lanes);
    const int64_t teams = a.tokens * slices;
    if (teams == 0 || a.top == 0) return hipSuccess;
    const bool once = past_cache(a.tokens * (a.top + 1) * a.hidden * size);
    with_lanes(lanes, [&](auto n) {
        constexpr int L = decltype(n)::value;
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid_of(teams, L), dim3(64 * kWaves), 0, s, a, slices, size);
        };
        once ? go(k_gather<L, true>) : go(k_gather<L, false>);
    });
    return hipGetLastError();
}

hipError_t launch_combine(const ExpertArgs &a, bool row_bf16, bool stream_bf16, hipStream_t s) {
    const int64_t pieces = ((int64_t)a.hidden + 7) / 8;
    const int lanes = lanes_of(pieces, true), slices = (int)((pieces + lanes - 1) / lanes);
    const int64_t teams = a.tokens * slices;
    if (teams == 0) return hipSuccess;
    const bool once = past_cache(a.tokens * a.hidden * ((int64_t)a.top * (row_bf16 ? 2 : 4) + (stream_bf16 ? 4 : 8)));
    with_lanes(lanes, [&](auto n) {
        constexpr int L = decltype(n)::value;
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid_of(teams, L), dim3(64 * kWaves), 0, s, a, slices);
        };
        with_types(row_bf16, stream_bf16, [&](auto t, auto st) {
            using T = decltype(t);
            using S = decltype(st);
            once ? go(k_combine<L, T, S, true>) : go(k_combine<L, T, S, false>);
        });
    });
    return hipGetLastError();
}

hipError_t launch_combine_backward(const ExpertArgs &a, bool row_bf16, bool stream_bf16, hipStream_t s) {
    const int64_t n = a.tokens * a.top;
    if (n == 0) return hipSuccess;
    with_lanes(lanes_of(((int64_t)a.hidden + 7) / 8), [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        with_types(row_bf16, stream_bf16, [&](auto t, auto st) {
            const auto kernel = k_combine_back<L, decltype(t), decltype(st)>;
            hipLaunchKernelGGL(kernel, grid_of(n, L), dim3(64 * kWaves), 0, s, a);
        });
    });
    return hipGetLastError();
}

}  // namespace sdpops
