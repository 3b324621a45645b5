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
#include <type_traits>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"
#include "sdp_route_keys.h"

namespace sdpops {
namespace {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr int64_t kNotThere = INT64_MIN;
// Sigmoids that add up to less than this are exp(z) to FP32's last place; their ratios are
// then taken from the logits, as those of a softmax always are, since the scores may be
// below any number.
constexpr float kSmall = 0x1p-26f;

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

__device__ __forceinline__ void put_weight(const RouteArgs &a, int64_t at, float w) {
    if (a.weight_bf16)
        store1((uint16_t *)a.weights + at, w);
    else
        ((float *)a.weights)[at] = w;
}

// 1 / (1 + exp(-x)) by a power that is never past FP32, so that small ones are not lost.
__device__ __forceinline__ float sigmoid_of(float x) {
    const float e = expf(-fabsf(x));
    return (x < 0.0f ? e : 1.0f) / (1.0f + e);
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

// What the wave's lanes have written to LDS is there for all of them.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// One token, by a whole wave, in 64 bits; value and keys: LDS of the wave's own, an
// element for each expert.
template <typename T>
__device__ void route_token(const RouteArgs &a, int64_t t, double *value, int64_t *keys) {
    const int lane = threadIdx.x & 63, E = a.experts;
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
    wave_fence();
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
        wave_fence();
        if (lane < a.groups && !keep)
            for (int i = lane * size; i < (lane + 1) * size; ++i) keys[i] = kNotThere;
        wave_fence();
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
        w = has ? sigmoid_of(x) : 0.0f;
    else
        w = has ? expf(x - top) / sum : 0.0f;
    if (a.renormalize) {
        const float all = wave_sum(w);
        if (!a.sigmoid || all < kSmall) {
            const float best = wave_max(x);
            const float e = has ? expf(x - best) : 0.0f, es = wave_sum(e);
            w = !has ? 0.0f : sum == sum ? e / es : sum;  // (no score of a row with a NaN is a number)
        } else {
            w = has ? w / all : 0.0f;
        }
    }
    if (on) {
        put_index(a, t * a.top + lane, mine);
        put_weight(a, t * a.top + lane, a.scale * w);
    }
    wave_fence();
}

// Any number of experts and groups: a wave takes a token.
template <typename T>
__global__ __launch_bounds__(64) void k_route_any(RouteArgs a) {
    extern __shared__ double wave_space[];
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x)
        route_token<T>(a, t, wave_space, (int64_t *)(wave_space + a.experts));
}

// N experts from row + e0 on, minus infinity past the last one.
template <typename T, int N>
__device__ __forceinline__ void load_experts(const T *row, int e0, int experts, float *z) {
    if (N >= 8 && e0 + N <= experts) {
#pragma unroll
        for (int i = 0; i < N; i += 8) load_floats(row + e0 + i, 8, z + i);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = e0 + i < experts ? load1(row + e0 + i) : kNegInf;
}

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// Sorted, the largest first (odd-even merges).
template <int N>
__device__ __forceinline__ void sort_list(float *v) {
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const float hi = fmaxf(v[i + j], v[i + j + k]), lo = fminf(v[i + j], v[i + j + k]);
                        v[i + j] = hi, v[i + j + k] = lo;
                    }
}

// `lanes` lanes take a token, a lane N experts that follow each other.  Each lane sorts
// its keys; then the largest first key of the lanes is taken `top` times, and its lane
// moves its list on.
// SCORED: keys are score + bias (or groups are to be compared), made in 32 bits; else
// they are the logits.  A key is off by a little, so where two of the choice that follow
// each other are close (and not from the same logit and bias) more experts are taken until
// the next one is far enough, and these candidates are ranked by their scores in 64 bits;
// close groups are compared in 64 bits likewise.  A token that has too many candidates, a
// NaN or an infinite key is done the slow way, behind the others: one such token makes a
// call 2 to 5 us longer.  Of 32,768 tokens' 256 sigmoid scores with a bias, one in about
// 500 needs the ranking, one in about 2,000 its groups compared (18.9 us, of which the
// logits' bytes take 7; without the 64 bits 16.5).
// KEEP: how many of its keys a lane's list keeps.  WIDE: a token has 32 or 64 lanes, else
// 8 or 16.
template <typename T, int N, int KEEP, bool WIDE, bool SCORED>
__global__ __launch_bounds__(256) void k_route_lanes(RouteArgs a) {
    constexpr bool kExact = !SCORED && sizeof(T) == 2;  // a BF16 logit has nothing in the last four bits
    extern __shared__ double wave_space[];
    __shared__ float best_of[SCORED ? 4 : 1][SCORED ? 64 : 1][3];
    __shared__ int chosen_of[4][2 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = a.lanes, sub = lane & (G - 1), token_lane = lane - sub, E = a.experts, e0 = sub * N;
    const int tokens_log = __builtin_ctz(64 / G), group_lanes = SCORED && a.groups > 1 ? E / a.groups / N : 1;
    // the token's lanes among the wave's (WIDE) or their half of them, and those below this one
    typedef std::conditional_t<WIDE, uint64_t, uint32_t> Lanes;
    constexpr int kLanes = WIDE ? 64 : 32;
    const Lanes mask = (Lanes)(G == kLanes ? ~(Lanes)0 : ((Lanes)1 << (G & 63)) - 1) << (token_lane & (kLanes - 1)),
                below = mask & (((Lanes)1 << (lane & (kLanes - 1))) - 1);
    auto half_of = [=](uint64_t b) __attribute__((always_inline)) {
        return WIDE ? (Lanes)b : (Lanes)(lane < 32 ? (uint32_t)b : (uint32_t)(b >> 32));
    };
    int *const chosen = chosen_of[wave] + token_lane;
    const int nowhere = 64 + lane - token_lane;  // where lanes write what nobody reads
    const bool sums = !a.sigmoid && (SCORED || !a.renormalize);
    auto most_of = [=](float v) __attribute__((always_inline)) {
        v = fmaxf(v, lanes_of<0xb1>(v));
        v = fmaxf(v, lanes_of<0x4e>(v));
        v = fmaxf(v, lanes_of<0x141>(v));
        const float more = fmaxf(v, lanes_of<0x140>(v));
        if (!WIDE) return G > 8 ? more : v;
        v = fmaxf(more, __shfl_xor(more, 16));
        return G > 32 ? fmaxf(v, __shfl_xor(v, 32)) : v;
    };
    // how far two keys may come out of order: a sigmoid is off by four roundings, a softmax
    // by up to 40 (its sum, most of them), the sum with the bias by one, the key by four bits
    const float slack = a.sigmoid ? 0x1p-19f : 0x1p-18f;
    auto off = [=](float key) { return SCORED ? (1.0f + fabsf(key)) * slack : 0x1p-19f * fabsf(key); };
    auto there = [](float key) { return key >= -__FLT_MAX__; };

    const int64_t w = a.first + (int64_t)blockIdx.x * (blockDim.x >> 6) + wave;
    if (w << tokens_log >= a.tokens) return;
    const int64_t t = (w << tokens_log) + (lane / G);
    const bool on = t < a.tokens;
    const T *row = (const T *)a.logits + (on ? t : a.tokens - 1) * a.logit_stride;
    float list[N];
    float top = 0.0f, sum = 1.0f;
    bool finite = true;
    {
        float z[N];
        load_experts<T, N>(row, e0, E, z);
        if (SCORED && a.bias) {
            // the bias beside it; an expert whose bias is minus infinity is not there
            float bias[N];
            if (N >= 4 && e0 + N <= E) {
#pragma unroll
                for (int i = 0; i < N; ++i) bias[i] = a.bias[e0 + i];
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) bias[i] = e0 + i < E ? a.bias[e0 + i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) list[i] = bias[i];
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) list[i] = 0.0f;
        }
        if (sums) {
            top = kNegInf;
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, z[i]);
            top = most_of(top);
            top = top == kNegInf ? 0.0f : top;
        }
        if (SCORED && a.sigmoid) {
#pragma unroll
            for (int i = 0; i < N; ++i) list[i] += __builtin_amdgcn_rcpf(1.0f + exp_fast(-z[i]));
        } else if (sums) {
            float score[N];
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) sum += score[i] = exp_fast(z[i] - top);
            sum = lanes_sum(sum, G);
            const float per_sum = 1.0f / sum;
#pragma unroll
            for (int i = 0; i < N; ++i) list[i] += score[i] * per_sum;
            finite = sum == sum;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float key = z[i] == kNegInf || !SCORED ? z[i] : list[i];
            finite = finite && key < __builtin_huge_valf();
            list[i] = key_of<kExact>(key, i);
        }
    }
    sort_list<N>(list);
    bool slow = !finite;
    // a score in 64 bits: the sum of the row's powers where it needs one, and the score with its bias
    auto sum_of = [&]() {
        if (a.sigmoid || !SCORED) return 1.0;
        double sum64 = 0.0;
#pragma unroll 1
        for (int i = e0; i < min(e0 + N, E); ++i) sum64 += exp((double)load1(row + i) - (double)top);
        for (int d = 1; d < G; d <<= 1) sum64 += __shfl_xor(sum64, d);
        return sum64;
    };
    auto exact_of = [&](float x, int e, double sum64) {
        const double power = exp(a.sigmoid ? -(double)x : (double)x - (double)top);
        const double score = a.sigmoid ? 1.0 / (1.0 + power) : power / sum64;
        return a.bias ? score + (double)a.bias[e] : score;
    };
    if (SCORED && a.groups > 1) {
        wave_fence();
#pragma unroll
        for (int k = 0; k < 3; ++k) best_of[wave][lane][k] = k < N ? list[k < N ? k : 0] : kNegInf;
        wave_fence();
        const float(*const of)[3] = best_of[wave] + token_lane + sub * group_lanes;
        float first = kNegInf, second = kNegInf;
        for (int l = 0; l < (sub < a.groups ? group_lanes : 0); ++l) {
            second = fmaxf(fmaxf(second, of[l][1]), fminf(first, of[l][0]));
            first = fmaxf(first, of[l][0]);
        }
        const Worth worth = worth_of(first, a.group_best > 1 ? second : kNegInf);
        bool kept = false;
        float left = worth.value;
        for (int k = 0; k < a.top_groups; ++k) {
            const float most = most_of(left);
            const bool mine = left == most, owner = mine && !(half_of(__ballot(mine)) & below);
            kept = kept || owner;
            left = owner ? kNegInf : left;
        }
        // one that is left may be worth as much as one that is kept
        const float high = most_of(left + worth.room),
                    low = -most_of(kept && there(worth.value) ? worth.room - worth.value : kNegInf);
        const bool close = on && high != kNegInf && low <= high;
        if (__any(close && !slow)) {
            // the groups' worth in 64 bits, of the same experts (unless the next one is close to them)
            float best[3] = {kNegInf, kNegInf, kNegInf};
            int from[2] = {0, 0};
            for (int l = 0; l < (sub < a.groups ? group_lanes : 0); ++l)
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    const float v = of[l][k];
                    const int e = (sub * group_lanes + l) * N + (int)place_of<false>(v);
                    if (v > best[0]) {
                        best[2] = best[1], best[1] = best[0], from[1] = from[0];
                        best[0] = v, from[0] = e;
                    } else if (v > best[1]) {
                        best[2] = best[1], best[1] = v, from[1] = e;
                    } else {
                        best[2] = fmaxf(best[2], v);
                    }
                }
            const float in = a.group_best > 1 ? best[1] : best[0], out = a.group_best > 1 ? best[2] : best[1];
            const bool unsure = close && there(out) && in - out <= off(in);
            slow = slow || unsure;
            const double sum64 = sum_of();
            double worth64 = -__builtin_huge_val();
            if (there(best[0])) worth64 = exact_of(load1(row + from[0]), from[0], sum64);
            if (there(best[1]) && a.group_best > 1) worth64 += exact_of(load1(row + from[1]), from[1], sum64);
            kept = false;
#pragma unroll 1
            for (int k = 0; k < a.top_groups; ++k) {
                double most = worth64;
                for (int d = 1; d < G; d <<= 1) most = fmax(most, __shfl_xor(most, d));
                const bool mine = worth64 == most, owner = mine && !(half_of(__ballot(mine)) & below);
                kept = kept || owner;
                worth64 = owner ? -__builtin_huge_val() : worth64;
            }
        }
        // an expert of no such group is never the largest, so its lane's list never moves
        if (!__shfl(kept ? 1 : 0, token_lane + sub / group_lanes)) list[0] = kNegInf;
    }
    // lane j keeps the j-th key; its expert's lane leaves the expert
    float my_key = kNegInf;
    auto take = [&](int j) __attribute__((always_inline)) {
        // (a place in a lane says nothing of the order of lanes)
        const float first = without_place(list[0]), most = most_of(first);
        const bool mine = first == most && most != kNegInf;
        const bool owner = mine && !(half_of(__ballot(mine)) & below);
        my_key = sub == j ? most : my_key;
        chosen[owner ? j : nowhere] = e0 + (int)place_of<kExact>(list[0]);
#pragma unroll
        for (int i = 0; i + 1 < KEEP; ++i) list[i] = owner ? list[i + 1] : list[i];
        list[KEEP - 1] = owner ? kNegInf : list[KEEP - 1];
        return most;
    };
    const int rounds = kExact ? a.top : a.top + 1;
#pragma unroll 1
    for (int j = 0; j < rounds; ++j) take(j);
    wave_fence();
    bool has = there(my_key) && sub < rounds;
    int mine = has ? chosen[sub] : -1;
    float x = has ? load1(row + mine) : kNegInf;
    if (!kExact) {
        float b = SCORED && a.bias && has ? a.bias[mine] : 0.0f;
        const float next = __shfl(my_key, lane + 1), next_x = __shfl(x, lane + 1), next_b = __shfl(b, lane + 1);
        // (equals at the end of the choice may have others close behind them, and those
        // of negative keys are sorted the highest first)
        const bool same = x == next_x && b == next_b && sub + 1 < a.top && my_key > 0.0f;
        const bool close = on && has && sub < a.top && there(next) && !same && my_key - next <= off(my_key);
        if (__any(close && !slow)) {
            // candidates until the next one is far behind the last one chosen
            const float last = __shfl(my_key, token_lane + a.top - 1);
            const float behind = __shfl(my_key, token_lane + rounds - 1);
            int count = rounds;
            bool more = (half_of(__ballot(close)) & mask) != 0 && there(behind) && behind >= last - off(last);
#pragma unroll 1
            for (; count < G && __any(more && !slow); ++count) {
                // (a lane whose list has run out may have had more)
                if (KEEP < N)
                    slow = slow || (more && (half_of(__ballot(list[0] == kNegInf && list[1] == kNegInf)) & mask));
                const float after = take(count);
                more = more && there(after) && after >= last - off(last);
            }
            slow = slow || more;
            wave_fence();
            has = there(my_key) && sub < count;
            mine = has ? chosen[sub] : -1;
            x = has ? load1(row + mine) : kNegInf;
            double exact = x;
            if (SCORED) {
                const double sum64 = sum_of();
                if (has) exact = exact_of(x, mine, sum64);
            }
            int rank = 0;
#pragma unroll 1
            for (int c = 0; c < count; ++c) {
                const double other = __shfl(exact, token_lane + c);
                const int at = __shfl(has ? mine : INT32_MAX, token_lane + c);
                rank += at != INT32_MAX && (other > exact || (other == exact && at < mine)) ? 1 : 0;
            }
            wave_fence();
            if (has) chosen[rank] = mine;
            wave_fence();
            // as many as there were, in their order
            has = sub < __popcll(half_of(__ballot(has)) & mask);
            mine = has ? chosen[sub] : -1;
            x = has ? load1(row + mine) : kNegInf;
        }
    }
    has = has && sub < a.top;
    float weight;
    if (a.sigmoid)
        weight = has ? sigmoid_of(x) : 0.0f;
    else
        weight = has && (sums || !a.renormalize) ? expf(x - top) * (1.0f / sum) : 0.0f;
    if (a.renormalize) {
        float all = 0.0f;
        if (a.sigmoid) all = lanes_sum(weight, G);
        if (!a.sigmoid || all < kSmall) {
            const float best = most_of(has ? x : kNegInf);
            weight = has ? expf(x - best) : 0.0f;
            all = lanes_sum(weight, G);
        }
        weight = has ? weight / all : 0.0f;
    }
    uint64_t again = __ballot(slow && on);
    if (on && sub < a.top && !(half_of(again) & mask)) {
        put_index(a, t * a.top + sub, has ? mine : -1);
        put_weight(a, t * a.top + sub, a.scale * weight);
    }
    if (again == 0) return;
    double *const space = wave_space + (int64_t)wave * 2 * E;
    while (again) {
        const int l = __builtin_ctzll(again) & ~(G - 1);
        again &= ~(((G == 64 ? 0ull : 1ull << G) - 1) << l);
        route_token<T>(a, (w << tokens_log) + l / G, space, (int64_t *)(space + E));
    }
}

// `lanes` lanes take a token, a lane N experts that follow each other and, as entry
// lane, one of the token's choices.
template <typename T, int N>
__global__ __launch_bounds__(256) void k_route_back(RouteArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = a.lanes, sub = lane & (G - 1), first = lane - sub, E = a.experts, e0 = sub * N;
    const int tokens_at_once = 64 / G;
    const bool all_scores = !a.sigmoid && !a.renormalize;
    const uint64_t mask = ((G == 64 ? 0ull : 1ull << G) - 1) << first;
    const int64_t waves = (int64_t)gridDim.x * (blockDim.x >> 6);
    for (int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 6) + wave; w * tokens_at_once < a.tokens; w += waves) {
        const int64_t t = w * tokens_at_once + (lane / G);
        const bool on = t < a.tokens;
        const T *row = (const T *)a.logits + (on ? t : a.tokens - 1) * a.logit_stride;
        float d[N];
        float top = 0.0f, sum = 1.0f;
        if (all_scores) {
            float z[N];
            load_experts<T, N>(row, e0, E, z);
            top = kNegInf;
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, z[i]);
            top = lanes_max(top, G);
            top = top == kNegInf ? 0.0f : top;
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) sum += d[i] = expf(z[i] - top);
            sum = lanes_sum(sum, G);
        }
        int64_t index = -1;
        float g = 0.0f;
        if (on && sub < a.top) {
            index = load_int(a.index_in, t * a.top + sub, a.index64);
            if (index >= 0) g = a.scale * load_either(a.dweights, t * a.top + sub, a.weight_bf16);
        }
        const bool bad = (__ballot(index >= E) & mask) != 0;
        const bool has = index >= 0 && index < E;
        const float x = has ? load1(row + index) : kNegInf;
        float p = 0.0f;
        if (has && a.sigmoid) p = sigmoid_of(x);
        if (has && all_scores) p = expf(x - top) / sum;
        const float rest = !has || !a.sigmoid ? 1.0f : sigmoid_of(-x);  // 1 - p
        float term, all = 0.0f;
        if (a.renormalize) {
            const float total = lanes_sum(p, G);
            float q = p / total;
            if (!a.sigmoid || total < kSmall) {
                const float best = lanes_max(x, G);
                const float e = has ? expf(x - best) : 0.0f;
                q = e / lanes_sum(e, G);
            }
            q = has ? q : 0.0f;
            term = q * (g - lanes_sum(g * q, G)) * rest;
        } else {
            term = g * p * rest;
            if (all_scores) all = lanes_sum(term, G);
        }
#pragma unroll
        // (a row of nothing but minus infinity has no scores, and no gradient)
        for (int i = 0; i < N; ++i) d[i] = all != 0.0f ? -d[i] / sum * all : 0.0f;
        const int named = has ? (int)index : -1;  // (32 bits of another index may name an expert)
        for (int j = 0; j < a.top; ++j) {
            const int at = __shfl(named, first + j) - e0;
            const float add = __shfl(term, first + j);
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] += at == i ? add : 0.0f;
        }
        if (!on) continue;
        T *dz = (T *)a.dlogits + t * a.dlogits_stride;
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = bad ? __builtin_nanf("") : d[i];
        if (N >= 8) {
#pragma unroll
            for (int i = 0; i < N; i += 8) store_floats(dz + e0 + i, E - e0 - i, d + i);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (e0 + i < E) store1(dz + e0 + i, d[i]);
        }
    }
}

// Any number of experts: a wave takes a token.
template <typename T>
__global__ __launch_bounds__(64) void k_route_back_any(RouteArgs a) {
    const int lane = threadIdx.x, E = a.experts;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const T *z = (const T *)a.logits + t * a.logit_stride;
        T *dz = (T *)a.dlogits + t * a.dlogits_stride;
        float top = 0.0f, sum = 1.0f;
        if (!a.sigmoid && !a.renormalize) softmax_of(z, E, top, sum);
        int64_t index = -1;
        float g = 0.0f;
        if (lane < a.top) {
            index = load_int(a.index_in, t * a.top + lane, a.index64);
            if (index >= 0) g = a.scale * load_either(a.dweights, t * a.top + lane, a.weight_bf16);
        }
        const bool bad = __any(index >= E);
        const bool has = index >= 0 && index < E;
        const float x = has ? load1(z + index) : kNegInf;
        const float p = !has ? 0.0f : a.sigmoid ? sigmoid_of(x) : expf(x - top) / sum;
        const float rest = !has || !a.sigmoid ? 1.0f : sigmoid_of(-x);  // 1 - p
        float term, all = 0.0f;
        if (a.renormalize) {
            float q = p;
            const float total = wave_sum(p);
            if (!a.sigmoid || total < kSmall) {
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

// Lanes of a token and experts of a lane, 16 where the lanes' lists keep nine of them.
// The fewest lanes that the experts, the choice and the groups allow: 32,768 tokens of 256
// experts in groups take 18.9 us with 16 lanes of 16 and 26.4 with 32 of 8.
// 0 lanes: none.
struct Split {
    int lanes, each;
};
constexpr int kKept = 9;
Split split_of(const RouteArgs &a, int taken) {
    for (int lanes = 8; lanes <= 64; lanes *= 2) {
        int each = 1;
        while (lanes * each < a.experts) each *= 2;
        if (each <= (taken <= kKept ? 16 : 8) && taken <= lanes && (a.groups == 1 || a.experts / a.groups % each == 0))
            return {lanes, each};
    }
    return {0, 0};
}

template <typename T>
hipError_t launch_route_any(const RouteArgs &args, hipStream_t s) {
    RouteArgs a = args;
    const bool scored = a.bias || a.groups > 1;
    const Split split = split_of(a, a.top + (scored || sizeof(T) == 4));  // one more is looked at than is chosen
    const size_t space = (size_t)a.experts * 16;  // of a wave
    if (!split.lanes) {
        const dim3 grid((uint32_t)std::min<int64_t>(a.tokens, 1 << 20));
        hipLaunchKernelGGL((k_route_any<T>), grid, dim3(64), space, s, a);
        return hipGetLastError();
    }
    a.lanes = split.lanes;
    const int64_t items = (a.tokens + 64 / a.lanes - 1) / (64 / a.lanes);
    // waves of a block: as many as have LDS for the slow way, and no more than there is work for
    const int waves = a.experts > 512 || items < 1024 ? 1 : 4;
    auto go = [&](auto kernel) {
        // (a wave walks no tokens in turn: what a loop keeps for the rare ways would leave room for fewer waves)
        constexpr int64_t kMost = 1 << 22;
        for (a.first = 0; a.first < items; a.first += kMost) {
            const int64_t n = std::min(kMost, items - a.first);
            const dim3 grid((uint32_t)((n + waves - 1) / waves));
            hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), space * waves, s, a);
        }
    };
    auto pick = [&](auto n) {
        constexpr int N = decltype(n)::value, K = N < kKept ? N : kKept;
        if (split.lanes > 16)
            scored ? go(k_route_lanes<T, N, K, true, true>) : go(k_route_lanes<T, N, K, true, false>);
        else
            scored ? go(k_route_lanes<T, N, K, false, true>) : go(k_route_lanes<T, N, K, false, false>);
    };
    switch (split.each) {
        case 1: pick(std::integral_constant<int, 1>()); break;
        case 2: pick(std::integral_constant<int, 2>()); break;
        case 4: pick(std::integral_constant<int, 4>()); break;
        case 8: pick(std::integral_constant<int, 8>()); break;
        default: pick(std::integral_constant<int, 16>()); break;
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_back_any(const RouteArgs &args, hipStream_t s) {
    RouteArgs a = args;
    a.groups = 1;
    const Split split = split_of(a, a.top);
    if (!split.lanes) {
        const dim3 grid((uint32_t)std::min<int64_t>(a.tokens, 1 << 20));
        hipLaunchKernelGGL((k_route_back_any<T>), grid, dim3(64), 0, s, a);
        return hipGetLastError();
    }
    a.lanes = split.lanes;
    const int64_t items = (a.tokens + 64 / a.lanes - 1) / (64 / a.lanes);
    const int waves = items < 1024 ? 1 : 4;
    const dim3 grid((uint32_t)std::min<int64_t>((items + waves - 1) / waves, 256 * 32)), block(64 * waves);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
    switch (split.each) {
        case 1: go(k_route_back<T, 1>); break;
        case 2: go(k_route_back<T, 2>); break;
        case 4: go(k_route_back<T, 4>); break;
        case 8: go(k_route_back<T, 8>); break;
        default: go(k_route_back<T, 16>); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_route(const RouteArgs &a, bool bf16, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    return bf16 ? launch_route_any<uint16_t>(a, s) : launch_route_any<float>(a, s);
}

hipError_t launch_route_backward(const RouteArgs &a, bool bf16, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    return bf16 ? launch_back_any<uint16_t>(a, s) : launch_back_any<float>(a, s);
}

}  // namespace sdpops
