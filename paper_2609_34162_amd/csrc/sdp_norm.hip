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
#include <type_traits>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"

namespace sdpops {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float weight_at(const NormArgs &a, const void *w, int64_t i) {
    return w ? a.offset + load_either(w, i, a.weight_bf16) : 1.0f;
}

// A gate after its activation, and its slope by the gate's input: of a sigmoid s the slope
// is s (1 - s) = s^2 e, e = exp(-z), which loses nothing where s is close to one.
struct Gate {
    float act, slope;
};
__device__ __forceinline__ Gate gate_of(const NormArgs &a, float z) {
    if (!a.sigmoid) return {z, 1.0f};
    const float e = fminf(expf(-z), __FLT_MAX__), s = __builtin_amdgcn_rcpf(1.0f + e);
    return {z != z ? z : s, s * (s * e)};
}

// The gate of an element (or 1).
template <typename T>
__device__ __forceinline__ Gate gate_at(const NormArgs &a, int64_t t, int64_t i) {
    if (a.gate_form == SDP_GATE_NONE) return {1.0f, 1.0f};
    const int64_t at = a.gate_form == SDP_GATE_CHANNEL ? i : t * a.gate_stride + (a.gate_form == SDP_GATE_ELEMENT ? i : 0);
    return gate_of(a, load1((const T *)a.gate + at));
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

__device__ __forceinline__ int64_t sums_stride(const NormArgs &a) { return ((int64_t)a.hidden + 3) / 4 * 4; }

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
            float v = load1(h + i);
            if (y) {
                const float u = a.post_norm ? load1(y + i) * ry * weight_at(a, a.post_weight, i) : load1(y + i);
                v += a.scale * gate_at<T>(a, t, i).act * u;
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

template <typename S, typename T>
__global__ __launch_bounds__(kThreads) void k_norm_back_any(NormArgs a) {
    __shared__ float waves[kThreads / 64];
    const float inv = 1.0f / (float)a.hidden;
    float *sums[2];
    for (int k = 0; k < 2; ++k) {
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
            for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads)
                dot += a.scale * gate_at<T>(a, t, i).act * g_at(i) * weight_at(a, a.post_weight, i) * load1(y + i);
            dot = block_sum(dot, waves) * inv * ry * ry;
        }
        float gate_sum = 0.0f;
        for (int64_t i = threadIdx.x; i < a.hidden; i += kThreads) {
            const float g = g_at(i);
            const Gate gate = gate_at<T>(a, t, i);
            const float du = a.scale * gate.act * g;
            const float x = y ? load1(y + i) : 0.0f, w = a.post_norm ? weight_at(a, a.post_weight, i) : 1.0f;
            if (sums[0]) sums[0][i] += load1(dn + i) * load1(h + i) * r;
            if (sums[1]) sums[1][i] += (a.gate_form >= SDP_GATE_TOKEN ? gate.act : 1.0f) * x * ry * g;
            if (a.dgate) {
                const float d = a.scale * (x * ry * w) * g * gate.slope;
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

// ---- rows in registers -------------------------------------------------------------

// Rows of up to 8,192 channels: `team` lanes take a row (a power of two within a
// wave, or the whole block), a lane NV pieces of eight channels that are a team
// apart, always the same ones, so that the weights and the sums over tokens stay in
// registers.  The next row's pieces are loaded before this one is worked on.
struct Place {
    int lane, team;       // in the team, and the team in the block
    int teams;            // of the grid
    int first;            // the block's first team
};
// WIDE: the team is the whole block, so that its rows' addresses are the same for all
// of its lanes.
template <bool WIDE>
__device__ __forceinline__ Place place_of(int team) {
    if (WIDE) return {(int)threadIdx.x, 0, (int)gridDim.x, (int)blockIdx.x};
    Place p;
    const int per = blockDim.x / team;
    p.lane = threadIdx.x % team;
    p.team = threadIdx.x / team;
    p.teams = gridDim.x * per;
    p.first = blockIdx.x * per;
    return p;
}

constexpr int kMostWaves = 16;

// Sums of N values over a team, in every lane of it.  A team of several waves meets in
// `waves`, of which calls use two in turn, so that one barrier is enough.
template <int N, bool WIDE>
__device__ __forceinline__ void team_sums(float *v, int team, float (*waves)[kMostWaves], int wave_count) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum(v[k], WIDE ? 64 : team);
    if (!WIDE) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) waves[k][wave] = v[k];
    }
    __syncthreads();
    const int from = lane & (kMostWaves - 1);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum(from < wave_count ? waves[k][from] : 0.0f, kMostWaves);
}

// NV 2: the next row is not loaded ahead, for want of registers.
template <typename S, typename T, int NV, bool WIDE, bool ONCE, int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_rows(NormArgs a) {
    __shared__ float waves[2][2][1][kMostWaves];
    const Place at = place_of<WIDE>(a.team);
    const int wave_count = blockDim.x >> 6;
    const float inv = 1.0f / (float)a.hidden;
    const bool has_y = a.y.data, has_n = a.n_out.data, each = a.gate_form == SDP_GATE_ELEMENT;
    int c[NV], left[NV];
    float add[NV][8], pre[NV][8];  // what y is multiplied by, less its token's factor; and the stream
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        c[j] = (at.lane + j * (WIDE ? (int)blockDim.x : a.team)) * 8;
        left[j] = a.hidden - c[j];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool in = k < left[j];
            add[j][k] = in ? a.scale * (a.post_norm ? weight_at(a, a.post_weight, c[j] + k) : 1.0f) : 0.0f;
            if (in && a.gate_form == SDP_GATE_CHANNEL) add[j][k] *= gate_of(a, load1((const T *)a.gate + c[j] + k)).act;
            pre[j][k] = in ? weight_at(a, a.pre_weight, c[j] + k) : 0.0f;
        }
    }
    Eight<S> h[NV];
    Eight<T> y[NV], gate[NV];
    float token_gate = 1.0f;
    auto fetch = [&](int64_t t) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (left[j] <= 0) continue;
            h[j] = load_eight<ONCE>((const S *)a.h.data + t * a.h.stride + c[j], left[j]);
            if (has_y) y[j] = load_eight<ONCE>((const T *)a.y.data + t * a.y.stride + c[j], left[j]);
            if (each) gate[j] = load_eight<ONCE>((const T *)a.gate + t * a.gate_stride + c[j], left[j]);
        }
        if (a.gate_form == SDP_GATE_TOKEN) token_gate = load1((const T *)a.gate + t * a.gate_stride);
    };
#pragma unroll
    for (int j = 0; j < NV; ++j) h[j].clear(), y[j].clear(), gate[j].clear();
    constexpr bool kAhead = NV == 1;
    int64_t t = at.first + at.team;
    if (kAhead && t < a.tokens) fetch(t);
    // (the teams of a block go on together, as they meet at barriers)
    int parity = 0;
    for (int64_t t0 = at.first; t0 < a.tokens; t0 += at.teams, t += at.teams, parity ^= 1) {
        const bool on = t < a.tokens;
        if (!kAhead && on) fetch(t);
        float x[NV][8], u[NV][8];
        float factor = 1.0f, sq = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            h[j].floats(x[j]);
            y[j].floats(u[j]);
#pragma unroll
            for (int k = 0; k < 8; ++k) sq += u[j][k] * u[j][k];
            if (each) {
                float z[8];
                gate[j].floats(z);
#pragma unroll
                for (int k = 0; k < 8; ++k) u[j][k] *= gate_of(a, z[k]).act;
            }
        }
        if (a.gate_form == SDP_GATE_TOKEN) factor = gate_of(a, token_gate).act;
        if (kAhead && t + at.teams < a.tokens) fetch(t + at.teams);
        if (has_y && a.post_norm) {
            team_sums<1, WIDE>(&sq, a.team, waves[parity][0], wave_count);
            factor *= rsqrtf(sq * inv + a.eps);
        }
        sq = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (has_y) x[j][k] += u[j][k] * factor * add[j][k];
                sq += x[j][k] * x[j][k];
            }
            if (on && a.h_out.data) store_floats<ONCE>((S *)a.h_out.data + t * a.h_out.stride + c[j], left[j], x[j]);
        }
        if (has_n) {
            team_sums<1, WIDE>(&sq, a.team, waves[parity][1], wave_count);
            const float r = rsqrtf(sq * inv + a.eps);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[j][k] *= r * pre[j][k];
                if (on) store_floats<ONCE>((T *)a.n_out.data + t * a.n_out.stride + c[j], left[j], x[j]);
            }
        }
    }
}

// Backward everything that a token's channels have to sum comes from one pass over
// them.  With q the factor of y in scale a u (less the root), v = dn w_pre, H channels:
//   hh = sum h^2, vh = sum v h, yy = sum y^2, and of g = dh_out + r v - r^3 vh / H h
//   qyg = sum q y dh_out + r sum q y v - r^3 vh / H sum q y h
// so that a row needs one meeting of its lanes.
// Over the tokens only dn h r and y ry g (times the gate where it is a token's own)
// are summed: a gate and weights of channels are factors of the whole sum.
template <typename S, typename T>
struct BackRow {
    Eight<S> h, dh;
    Eight<T> y, dn, gate;
};

// EACH: the gate is an element's own.  AHEAD: the next row's pieces are loaded before
// this one is worked on (where their registers are there).
template <typename S, typename T, bool EACH, bool AHEAD, bool WIDE, bool ONCE, int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_back_rows(NormArgs a) {
    __shared__ float waves[2][6][kMostWaves];
    __shared__ float joined[WIDE ? 1 : 2][WIDE ? 1 : THREADS * 8];
    const Place at = place_of<WIDE>(a.team);
    const int wave_count = blockDim.x >> 6;
    const float inv = 1.0f / (float)a.hidden;
    const bool has_y = a.y.data, has_n = a.dn.data, has_h = a.dh_out.data, by_token = a.gate_form == SDP_GATE_TOKEN;
    const bool dots = has_y && ((a.post_norm && a.dy.data) || (by_token && a.dgate));
    const int c = at.lane * 8, left = a.hidden - c;
    float q[8], pre[8], sum_n[8], sum_y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const bool in = k < left;
        q[k] = in ? a.scale * (a.post_norm ? weight_at(a, a.post_weight, c + k) : 1.0f) : 0.0f;
        if (in && a.gate_form == SDP_GATE_CHANNEL) q[k] *= gate_of(a, load1((const T *)a.gate + c + k)).act;
        pre[k] = in ? weight_at(a, a.pre_weight, c + k) : 0.0f;
        sum_n[k] = sum_y[k] = 0.0f;
    }
    BackRow<S, T> row;
    auto fetch = [&](int64_t t, BackRow<S, T> &to) __attribute__((always_inline)) {
        if (left > 0) {
            if (has_n) {
                to.h = load_eight<ONCE>((const S *)a.h.data + t * a.h.stride + c, left);
                to.dn = load_eight<ONCE>((const T *)a.dn.data + t * a.dn.stride + c, left);
            }
            if (has_h) to.dh = load_eight<ONCE>((const S *)a.dh_out.data + t * a.dh_out.stride + c, left);
            if (has_y) to.y = load_eight<ONCE>((const T *)a.y.data + t * a.y.stride + c, left);
            if (EACH) to.gate = load_eight<ONCE>((const T *)a.gate + t * a.gate_stride + c, left);
        }
    };
    auto clear = [](BackRow<S, T> &r) __attribute__((always_inline)) {
        r.h.clear(), r.dh.clear(), r.y.clear(), r.dn.clear(), r.gate.clear();
    };
    int64_t t = at.first + at.team;
    BackRow<S, T> next;
    clear(row);
    clear(next);
    if (AHEAD && t < a.tokens) fetch(t, next);
    int parity = 0;
    for (int64_t t0 = at.first; t0 < a.tokens; t0 += at.teams, t += at.teams, parity ^= 1) {
        const bool on = t < a.tokens;
        if (AHEAD) {
            row = next;
            if (t + at.teams < a.tokens) fetch(t + at.teams, next);
        } else if (on) {
            fetch(t, row);
        }
        Gate of_token = {1.0f, 1.0f};
        if (by_token && on) of_token = gate_of(a, load1((const T *)a.gate + t * a.gate_stride));
        float s[6] = {};
        {
            float x[8], v[8], g[8], z[8], f[8];
            row.h.floats(x), row.dn.floats(v), row.dh.floats(g), row.y.floats(z);
            if (EACH) row.gate.floats(f);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float vw = v[k] * pre[k];
                s[0] += x[k] * x[k];
                s[1] += vw * x[k];
                s[2] += z[k] * z[k];
                float qy = q[k] * z[k];
                if (EACH) qy *= gate_of(a, f[k]).act;
                s[3] += qy * g[k];
                s[4] += qy * vw;
                s[5] += qy * x[k];
            }
        }
        row.h.forget(), row.dn.forget(), row.dh.forget(), row.y.forget();
        if (EACH) row.gate.forget();
        team_sums<6, WIDE>(s, a.team, waves[parity], wave_count);
        float r = 0.0f, along = 0.0f, ry = 1.0f, dot = 0.0f;
        if (has_n) {
            r = rsqrtf(s[0] * inv + a.eps);
            along = s[1] * inv * r * r;
        }
        if (a.post_norm && has_y) ry = rsqrtf(s[2] * inv + a.eps);
        if (dots) dot = s[3] + r * (s[4] - along * s[5]);  // sum of q y g
        if (by_token && a.dgate && on && at.lane == 0) store1((T *)a.dgate + t * a.dgate_stride, of_token.slope * ry * dot);
        const float back = a.post_norm ? of_token.act * dot * inv * ry * ry : 0.0f;
        if (!on) continue;
        float x[8], v[8], g[8], z[8], f[8];
        row.h.floats(x), row.dn.floats(v), row.dh.floats(g), row.y.floats(z);
        if (EACH) row.gate.floats(f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float gk = g[k] + r * (v[k] * pre[k] - x[k] * along);
            g[k] = gk;
            const float yg = z[k] * ry * gk;
            float mine = of_token.act;
            if (EACH) {
                const Gate of = gate_of(a, f[k]);
                mine = of.act;
                f[k] = q[k] * yg * of.slope;
            }
            sum_n[k] += v[k] * x[k] * r;
            sum_y[k] += mine * yg;
            v[k] = ry * (mine * q[k] * gk - z[k] * back);
        }
        if (a.dh.data) store_floats<ONCE>((S *)a.dh.data + t * a.dh.stride + c, left, g);
        if (a.dy.data) store_floats<ONCE>((T *)a.dy.data + t * a.dy.stride + c, left, v);
        if (EACH && a.dgate) store_floats<ONCE>((T *)a.dgate + t * a.dgate_stride + c, left, f);
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        if (!a.sums[w]) continue;
        float *out = a.sums[w] + blockIdx.x * sums_stride(a);
        if (WIDE) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) out[c + k] = w ? sum_y[k] : sum_n[k];
        } else {
            // the block's teams, added in their order
#pragma unroll
            for (int k = 0; k < 8; ++k) joined[w][threadIdx.x * 8 + k] = w ? sum_y[k] : sum_n[k];
            __syncthreads();
            for (int i = threadIdx.x; i < a.hidden; i += THREADS) {
                float s = 0.0f;
                for (int p = 0; p < THREADS / a.team; ++p) s += joined[w][p * a.team * 8 + i];
                out[i] = s;
            }
        }
    }
}

// The blocks' partial sums, added in their order: 32 channels to a block, eight threads
// of four channels to a row of them, 128 rows at a time.  blockIdx.y: which sums.
constexpr int kSumThreads = 1024, kSumLanes = 8, kSumRows = kSumThreads / kSumLanes;
template <typename T>
__global__ __launch_bounds__(kSumThreads) void k_norm_sums(NormArgs a) {
    __shared__ f32x4 part[kSumRows][kSumLanes];
    const int which = blockIdx.y, x = threadIdx.x % kSumLanes, y = threadIdx.x / kSumLanes;
    if (!a.sums[which]) return;
    const int64_t i = ((int64_t)blockIdx.x * kSumLanes + x) * 4;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i < a.hidden) {
        const float *from = a.sums[which] + i;
#pragma unroll 4
        for (int b = y; b < a.blocks; b += kSumRows) s += *(const f32x4 *)(from + b * sums_stride(a));
    }
    part[y][x] = s;
    for (int half = kSumRows / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (y < half) part[y][x] += part[y + half][x];
    }
    if (y > 0) return;
    s = part[0][x];
    for (int k = 0; k < 4 && i + k < a.hidden; ++k) {
        auto put = [&](void *w, float v) {
            if (a.weight_bf16)
                store1((uint16_t *)w + i + k, v);
            else
                ((float *)w)[i + k] = v;
        };
        if (which == 0) {
            put(a.dpre, s[k]);
            continue;
        }
        const bool channel = a.gate_form == SDP_GATE_CHANNEL;
        const Gate gate = channel ? gate_at<T>(a, 0, i + k) : Gate{1.0f, 1.0f};
        if (a.dpost) put(a.dpost, a.scale * gate.act * s[k]);
        if (a.dgate && channel)
            store1((T *)a.dgate + i + k,
                   a.scale * gate.slope * (a.post_norm ? weight_at(a, a.post_weight, i + k) : 1.0f) * s[k]);
    }
}

template <typename F>
void with_types(bool stream_bf16, bool bf16, F &&go) {
    if (stream_bf16)
        bf16 ? go((uint16_t *)nullptr, (uint16_t *)nullptr) : go((uint16_t *)nullptr, (float *)nullptr);
    else
        bf16 ? go((float *)nullptr, (uint16_t *)nullptr) : go((float *)nullptr, (float *)nullptr);
}

// How a call is split: lanes to a row and threads to a block; 0 lanes where rows do not
// fit the registers.
struct Split {
    int team, threads, pieces;  // pieces: of a lane
};
Split split_of(const NormArgs &a, bool backward) {
    const int n = (a.hidden - 1) / 8 + 1;
    if (n <= 64) {
        int team = 8;
        while (team < n) team *= 2;
        return {team, 256, 1};
    }
    for (int pieces = 1; pieces <= (backward ? 1 : 2); ++pieces) {
        const int lanes = ((n + pieces - 1) / pieces + 63) / 64 * 64;
        if (lanes <= 1024) return {lanes, lanes, pieces};
    }
    return {0, kThreads, 1};
}

// Blocks that a call's rows are walked by: at most as many as the compute units hold at
// once (forward eight waves to a SIMD, or what is left of them; backward three, or four of
// 16-bit tensors), and each as many rows as the others.
int blocks_of(const NormArgs &a, const Split &s, bool backward, bool wide_types) {
    const int64_t per = s.team ? s.threads / s.team : 1, waves = s.threads / 64;
    const int64_t held = !backward ? 32 : wide_types ? 12 : 16;
    const int64_t most = 256 * (s.team ? std::max<int64_t>(1, held / waves) : 4);
    const int64_t rows = (a.tokens + per - 1) / per, each = (rows + most - 1) / most;
    return (int)((rows + each - 1) / each);
}

// Whether a call's tensors are past the last-level cache.
bool past_cache(const NormArgs &a, int64_t bytes) { return a.tokens * a.hidden * bytes > (int64_t)256 << 20; }

}  // namespace

int norm_blocks(const NormArgs &a, bool stream_bf16, bool bf16) {
    return a.tokens ? blocks_of(a, split_of(a, true), true, !(stream_bf16 && bf16)) : 0;
}

hipError_t launch_norm(const NormArgs &args, bool stream_bf16, bool bf16, hipStream_t s) {
    NormArgs a = args;
    const Split split = split_of(a, false);
    a.team = split.team;
    const dim3 grid(blocks_of(a, split, false, false)), block(split.threads);
    const bool once = past_cache(a, 2 * ((stream_bf16 ? 2 : 4) + (bf16 ? 2 : 4)));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
    with_types(stream_bf16, bf16, [&](auto *st, auto *ty) {
        using S = std::remove_pointer_t<decltype(st)>;
        using T = std::remove_pointer_t<decltype(ty)>;
        if (!split.team) return go(k_norm_any<S, T>);
        if (split.team <= 64)
            return once ? go(k_norm_rows<S, T, 1, false, true, 256>) : go(k_norm_rows<S, T, 1, false, false, 256>);
        if (split.pieces == 1)
            return once ? go(k_norm_rows<S, T, 1, true, true, 1024>) : go(k_norm_rows<S, T, 1, true, false, 1024>);
        once ? go(k_norm_rows<S, T, 2, true, true, 1024>) : go(k_norm_rows<S, T, 2, true, false, 1024>);
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormArgs &args, bool stream_bf16, bool bf16, hipStream_t s) {
    NormArgs a = args;
    if (a.blocks > 0) {
        const Split split = split_of(a, true);
        a.team = split.team;
        const dim3 grid(a.blocks), block(split.threads);
        const bool once = past_cache(a, 3 * ((stream_bf16 ? 2 : 4) + (bf16 ? 2 : 4)));
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
        with_types(stream_bf16, bf16, [&](auto *st, auto *ty) {
            using S = std::remove_pointer_t<decltype(st)>;
            using T = std::remove_pointer_t<decltype(ty)>;
            if (!split.team) return go(k_norm_back_any<S, T>);
            auto pick = [&](auto each) {
                constexpr bool E = decltype(each)::value;
                auto go_once = [&](auto is_once) {
                    constexpr bool O = decltype(is_once)::value;
                    if (split.team <= 64) return go(k_norm_back_rows<S, T, E, true, false, O, 256>);
                    if (split.threads <= 768) return go(k_norm_back_rows<S, T, E, true, true, O, 768>);
                    go(k_norm_back_rows<S, T, E, false, true, O, 1024>);
                };
                once ? go_once(std::true_type()) : go_once(std::false_type());
            };
            a.gate_form == SDP_GATE_ELEMENT ? pick(std::true_type()) : pick(std::false_type());
        });
    }
    if (a.sums[0] || a.sums[1]) {
        const dim3 grid((a.hidden - 1) / (4 * kSumLanes) + 1, 2);
        if (bf16)
            hipLaunchKernelGGL((k_norm_sums<uint16_t>), grid, dim3(kSumThreads), 0, s, a);
        else
            hipLaunchKernelGGL((k_norm_sums<float>), grid, dim3(kSumThreads), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace sdpops
