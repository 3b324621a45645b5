// gfx950 kernels of sdp_route and its backward.
//
// A token's experts are the `top` largest of score + bias, one after the other, among
// the experts of its best groups; its weights come from their scores:
//   softmax: p = exp(z - max) / sum;   sigmoid: p = 1 / (1 + exp(-z))
//   w_j = c p_j, or c p_j / sum over the chosen
// and backward, with g_j = c dw_j and q the chosen scores over their sum:
//   softmax  dz_i = p_i (g_i - sum of g p);    sigmoid  dz_j = g_j p_j (1 - p_j)
//   over their sum: dz_j = q_j (g_j - sum of g q), times 1 - p_j for a sigmoid
// Which of two close scores is larger has to come out the same for everyone who
// computes them well, so scores are compared in 64 bits.
#include <algorithm>

#include "sdp_layer_internal.h"
#include "sdp_ops_device.h"

namespace sdpops {
namespace {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr int64_t kNotThere = INT64_MIN;

// Larger keys for larger values, the largest for a NaN; -0 counts as 0.
__device__ __forceinline__ int64_t order_key(double x) {
    if (x != x) return INT64_MAX;
    const int64_t b = __double_as_longlong(x + 0.0);
    return b < 0 ? b ^ INT64_MAX : b;
}

__device__ __forceinline__ double wave_sum64(double v) {
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// The largest key of the wave, and the lowest place that has it.
__device__ __forceinline__ void wave_best(int64_t &key, int &at) {
    for (int d = 32; d > 0; d >>= 1) {
        const int64_t k = __shfl_xor(key, d);
        const int i = __shfl_xor(at, d);
        if (k > key || (k == key && i < at)) key = k, at = i;
    }
}

__device__ __forceinline__ void put_index(const RouteArgs &a, int64_t at, int index) {
    if (a.index64)
        ((int64_t *)a.index)[at] = index;
    else
        ((int32_t *)a.index)[at] = index;
}

// The largest and the sum of exp(z - max) of a row; max is 0 in a row of nothing but
// minus infinity.
template <typename T>
__device__ __forceinline__ void softmax_of(const T *z, int n, float &top, float &sum) {
    const int lane = threadIdx.x & 63;
    top = kNegInf;
    float nan = 0.0f;
    for (int i = lane; i < n; i += 64) {
        const float x = load1(z + i);
        top = fmaxf(top, x);
        nan += x != x ? 1.0f : 0.0f;
    }
    top = wave_max(top);
    top = top == kNegInf ? 0.0f : top;
    sum = 0.0f;
    for (int i = lane; i < n; i += 64) sum += expf(load1(z + i) - top);
    sum = wave_sum(sum);
    if (wave_sum(nan) != 0.0f) sum = __builtin_nanf("");
}

// A wave takes a token.
template <typename T>
__global__ __launch_bounds__(64) void k_route(RouteArgs a) {
    __shared__ double value[SDP_ROUTE_MAX_EXPERTS];
    __shared__ int64_t keys[SDP_ROUTE_MAX_EXPERTS];
    const int lane = threadIdx.x, E = a.experts;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const T *z = (const T *)a.logits + t * a.logit_stride;
        const bool scored = a.bias || a.groups > 1;
        float top = 0.0f, sum = 1.0f;
        if (!a.sigmoid) softmax_of(z, E, top, sum);
        double sum64 = 1.0;
        if (scored && !a.sigmoid) {
            sum64 = 0.0;
            for (int i = lane; i < E; i += 64) sum64 += exp((double)load1(z + i) - (double)top);
            sum64 = wave_sum64(sum64);
        }
        for (int i = lane; i < E; i += 64) {
            const float x = load1(z + i), b = a.bias ? a.bias[i] : 0.0f;
            double v = x;
            if (scored) {
                v = a.sigmoid ? 1.0 / (1.0 + exp(-(double)x)) : exp((double)x - (double)top) / sum64;
                v += (double)b;
            }
            value[i] = v;
            keys[i] = x == kNegInf || b == kNegInf ? kNotThere : order_key(v);
        }
        __syncthreads();
        if (a.groups > 1) {
            const int size = E / a.groups;
            int64_t worth = kNotThere;
            if (lane < a.groups) {
                int64_t best[2] = {kNotThere, kNotThere};
                double of[2] = {0.0, 0.0};
                for (int i = lane * size; i < (lane + 1) * size; ++i) {
                    if (keys[i] > best[0]) {
                        best[1] = best[0], of[1] = of[0];
                        best[0] = keys[i], of[0] = value[i];
                    } else if (keys[i] > best[1]) {
                        best[1] = keys[i], of[1] = value[i];
                    }
                }
                if (best[0] != kNotThere)
                    worth = order_key(a.group_best > 1 && best[1] != kNotThere ? of[0] + of[1] : of[0]);
            }
            bool keep = false;
            for (int k = 0; k < a.top_groups; ++k) {
                int64_t key = worth;
                int at = lane;
                wave_best(key, at);
                if (lane == at) keep = true, worth = kNotThere;
            }
            __syncthreads();
            if (lane < a.groups && !keep)
                for (int i = lane * size; i < (lane + 1) * size; ++i) keys[i] = kNotThere;
            __syncthreads();
        }
        // lane j keeps the j-th expert
        int mine = -1;
        for (int j = 0; j < a.top; ++j) {
            int64_t key = kNotThere;
            int at = E;
            for (int i = lane; i < E; i += 64)
                if (keys[i] > key) key = keys[i], at = i;
            wave_best(key, at);
            if (lane == j) mine = key == kNotThere ? -1 : at;
            if (key != kNotThere && (at & 63) == lane) keys[at] = kNotThere;
        }
        const bool on = lane < a.top, has = on && mine >= 0;
        const float x = has ? load1(z + mine) : kNegInf;
        float w;
        if (a.sigmoid)
            w = has ? 1.0f / (1.0f + expf(-x)) : 0.0f;
        else
            w = has ? expf(x - top) / sum : 0.0f;
        if (a.renormalize) {
            const float all = wave_sum(w);
            if (all < 1e-30f) {
                // too small for their ratios: a sigmoid that far down is exp(z) too
                const float best = wave_max(x);
                const float e = has ? expf(x - best) : 0.0f, es = wave_sum(e);
                w = has ? e / es : 0.0f;
            } else {
                w = has ? w / all : 0.0f;
            }
        }
        if (on) {
            put_index(a, t * a.top + lane, mine);
            const float out = a.scale * w;
            if (a.weight_bf16)
                store1((uint16_t *)a.weights + t * a.top + lane, out);
            else
                ((float *)a.weights)[t * a.top + lane] = out;
        }
        __syncthreads();
    }
}

template <typename T>
__global__ __launch_bounds__(64) void k_route_back(RouteArgs a) {
    const int lane = threadIdx.x, E = a.experts;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const T *z = (const T *)a.logits + t * a.logit_stride;
        T *dz = (T *)a.dlogits + t * a.dlogits_stride;
        float top = 0.0f, sum = 1.0f;
        if (!a.sigmoid) softmax_of(z, E, top, sum);
        int64_t index = -1;
        float g = 0.0f;
        if (lane < a.top) {
            index = load_int(a.index_in, t * a.top + lane, a.index64);
            if (index >= 0) g = a.scale * load_either(a.dweights, t * a.top + lane, a.weight_bf16);
        }
        const bool bad = __any(index >= E);
        const bool has = index >= 0 && index < E;
        const float x = has ? load1(z + index) : kNegInf;
        const float p = !has ? 0.0f : a.sigmoid ? 1.0f / (1.0f + expf(-x)) : expf(x - top) / sum;
        const float rest = !has || !a.sigmoid ? 1.0f : 1.0f / (1.0f + expf(x));  // 1 - p
        float term, all = 0.0f;
        if (a.renormalize) {
            float q = p;
            const float total = wave_sum(p);
            if (total < 1e-30f) {
                const float best = wave_max(x);
                const float e = has ? expf(x - best) : 0.0f;
                const float es = wave_sum(e);
                q = has ? e / es : 0.0f;
            } else {
                q = p / total;
            }
            const float mean = wave_sum(g * q);
            term = has ? q * (g - mean) * rest : 0.0f;
        } else if (a.sigmoid) {
            term = g * p * rest;
        } else {
            term = g * p;
            all = wave_sum(term);
        }
        for (int i0 = 0; i0 < E; i0 += 64) {
            const int i = i0 + lane;
            float d = 0.0f;
            for (int j = 0; j < a.top; ++j) {
                const int at = __shfl((int)index, j);
                const float add = __shfl(term, j);
                d += at == i ? add : 0.0f;
            }
            if (i < E) {
                // (a row of nothing but minus infinity has no scores, and no gradient)
                if (all != 0.0f) d -= expf(load1(z + i) - top) / sum * all;
                store1(dz + i, bad ? __builtin_nanf("") : d);
            }
        }
    }
}

}  // namespace

hipError_t launch_route(const RouteArgs &a, bool bf16, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    const dim3 grid((uint32_t)std::min<int64_t>(a.tokens, 1 << 20));
    if (bf16)
        hipLaunchKernelGGL((k_route<uint16_t>), grid, dim3(64), 0, s, a);
    else
        hipLaunchKernelGGL((k_route<float>), grid, dim3(64), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_route_backward(const RouteArgs &a, bool bf16, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    const dim3 grid((uint32_t)std::min<int64_t>(a.tokens, 1 << 20));
    if (bf16)
        hipLaunchKernelGGL((k_route_back<uint16_t>), grid, dim3(64), 0, s, a);
    else
        hipLaunchKernelGGL((k_route_back<float>), grid, dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace sdpops
