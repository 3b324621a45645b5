// gfx950 kernels of sdp_block_norm and its backward.
//
// For a token's rows, ry = 1 / rms(y), r = 1 / rms(h_out), w the weights with their
// offset and a the gate:
//   u = y ry w_post;  h_out = h + s a u;  n = h_out r w_pre
// and backward, with v = dn w_pre and mean over the channels:
//   g = dh_out + r (v - h_out r^2 mean(v h_out));  dh = g;  du = s a g
//   dy = ry (du w_post - y ry^2 mean(du w_post y));  dgate = s u g (times a (1 - a))
//   dw_pre = sum of dn h_out r;  dw_post = sum of du y ry
// Memory bounds both: each tensor is read once and written once, at 5.4 TB/s for 32,768
// tokens of 5,120 BF16 channels (248 us; backward, with its sums over tokens, 398, 5.1).
#include <algorithm>
#include <type_traits>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"

namespace sdpops {
namespace {

__device__ __forceinline__ float weight_at(const NormArgs &a, const void *w, int64_t i) {
    return w ? a.offset + load_either(w, i, a.weight_bf16) : 1.0f;
}

// A gate after its activation, and its slope by the gate's input: of a sigmoid s the slope
// is s (1 - s) = s^2 e, e = exp(-z), which loses nothing where s is close to one.  Of a NaN
// both are NaN, which fminf loses.
struct Gate {
    float act, slope;
};
__device__ __forceinline__ Gate gate_of(const NormArgs &a, float z) {
    if (!a.sigmoid) return {z, 1.0f};
    const float e = fminf(expf(-z), __FLT_MAX__), s = __builtin_amdgcn_rcpf(1.0f + e);
    return {z != z ? z : s, z != z ? z : s * (s * e)};
}

// Eight of a norm's weights with their offset; zeros behind the row.
__device__ __forceinline__ void weights_of(const NormArgs &a, const void *w, int c, int left, float *out) {
#pragma unroll
    for (int k = 0; k < 8; ++k) out[k] = 0.0f;
    if (w && a.weight_bf16)
        load_floats((const uint16_t *)w + c, left, out);
    else if (w)
        load_floats((const float *)w + c, left, out);
#pragma unroll
    for (int k = 0; k < 8; ++k) out[k] = k < left ? (w ? a.offset + out[k] : 1.0f) : 0.0f;
}

// Of eight channels the factors that are not a token's: of y (the scale, the weight, a
// gate of channels) and of the stream's norm.
template <typename T>
__device__ __forceinline__ void factors_of(const NormArgs &a, int c, int left, float *of_y, float *of_n) {
    weights_of(a, a.pre_weight, c, left, of_n);
    weights_of(a, a.post_norm ? a.post_weight : nullptr, c, left, of_y);
    float z[8] = {};
    if (a.gate_form == SDP_GATE_CHANNEL) load_floats((const T *)a.gate + c, left, z);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        of_y[k] *= a.scale;
        if (a.gate_form == SDP_GATE_CHANNEL) of_y[k] *= k < left ? gate_of(a, z[k]).act : 0.0f;
    }
}

__device__ __forceinline__ int64_t sums_stride(const NormArgs &a) { return ((int64_t)a.hidden + 3) / 4 * 4; }

// ---- rows in registers -------------------------------------------------------------

// Rows of up to 8,192 channels (forward 16,384): `team` lanes take a row (a power of two
// within a wave, or the whole block), a lane NV pieces of eight channels that are a team
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
        factors_of<T>(a, c[j], left[j], add[j], pre[j]);
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
// Adds what eight channels have in those sums.  EACH: the gate is an element's own.
template <bool EACH>
__device__ __forceinline__ void add_dots(const NormArgs &a, const float *x, const float *v, const float *g,
                                         const float *z, const float *f, const float *q, const float *pre, float *s) {
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

struct BackToken {
    float r, along, ry, dot, back;  // dot: sum of q y g
    Gate gate;                      // the token's own, or 1
};
__device__ __forceinline__ BackToken token_of(const NormArgs &a, const float *s, float inv, Gate gate) {
    BackToken o = {0.0f, 0.0f, 1.0f, 0.0f, 0.0f, gate};
    const bool by_token = a.gate_form == SDP_GATE_TOKEN && a.dgate;
    if (a.dn.data) {
        o.r = rsqrtf(s[0] * inv + a.eps);
        o.along = s[1] * inv * o.r * o.r;
    }
    if (a.post_norm && a.y.data) o.ry = rsqrtf(s[2] * inv + a.eps);
    if (a.y.data && ((a.post_norm && a.dy.data) || by_token)) o.dot = s[3] + o.r * (s[4] - o.along * s[5]);
    if (a.post_norm) o.back = gate.act * o.dot * inv * o.ry * o.ry;
    return o;
}
template <typename T>
__device__ __forceinline__ void put_token_gate(const NormArgs &a, int64_t t, const BackToken &o) {
    store1((T *)a.dgate + t * a.dgate_stride, o.gate.slope * o.ry * o.dot);
}

// Eight channels' gradients: of the stream over g, of y over v, of their gates over f; and
// what the sums over tokens get.
template <bool EACH>
__device__ __forceinline__ void finish(const NormArgs &a, const BackToken &o, const float *x, float *v, float *g,
                                       const float *z, float *f, const float *q, const float *pre, float *sum_n,
                                       float *sum_y) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float gk = g[k] + o.r * (v[k] * pre[k] - x[k] * o.along);
        g[k] = gk;
        const float yg = z[k] * o.ry * gk;
        float mine = o.gate.act;
        if (EACH) {
            const Gate of = gate_of(a, f[k]);
            mine = of.act;
            f[k] = q[k] * yg * of.slope;
        }
        sum_n[k] += v[k] * x[k] * o.r;
        sum_y[k] += mine * yg;
        v[k] = o.ry * (mine * q[k] * gk - z[k] * o.back);
    }
}

template <typename S, typename T>
struct BackRow {
    Eight<S> h, dh;
    Eight<T> y, dn, gate;
};

// Waves that a SIMD is to hold of it at least.
template <typename S, typename T, bool EACH>
constexpr int kBackHeld = !EACH && sizeof(S) + sizeof(T) == 4 ? 4 : 1;

// AHEAD: the next row's pieces are loaded before
// this one is worked on (where their registers are there).
template <typename S, typename T, bool EACH, bool AHEAD, bool WIDE, bool ONCE, int THREADS>
__global__ __launch_bounds__(THREADS, (kBackHeld<S, T, EACH>)) void k_norm_back_rows(NormArgs a) {
    __shared__ float waves[2][6][kMostWaves];
    __shared__ float joined[WIDE ? 1 : 2][WIDE ? 1 : THREADS * 8];
    const Place at = place_of<WIDE>(a.team);
    const int wave_count = blockDim.x >> 6;
    const float inv = 1.0f / (float)a.hidden;
    const bool has_y = a.y.data, has_n = a.dn.data, has_h = a.dh_out.data, by_token = a.gate_form == SDP_GATE_TOKEN;
    const int c = at.lane * 8, left = a.hidden - c;
    float q[8], pre[8], sum_n[8], sum_y[8];
    factors_of<T>(a, c, left, q, pre);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum_n[k] = sum_y[k] = 0.0f;
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
    // (a wave's lanes have rows of their own unless WIDE: addresses of 32-bit rows take fewer registers)
    using Row = std::conditional_t<WIDE, int64_t, uint32_t>;
    const Row n = (Row)a.tokens;  // below 2^31
    Row t = at.first + at.team;
    BackRow<S, T> next;
    clear(row);
    clear(next);
    if (AHEAD && t < n) fetch(t, next);
    int parity = 0;
    for (Row t0 = at.first; t0 < n; t0 += at.teams, t += at.teams, parity ^= 1) {
        const bool on = t < n;
        if (AHEAD) {
            row = next;
            if (t + at.teams < n) fetch(t + at.teams, next);
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
            add_dots<EACH>(a, x, v, g, z, f, q, pre, s);
        }
        row.h.forget(), row.dn.forget(), row.dh.forget(), row.y.forget();
        if (EACH) row.gate.forget();
        team_sums<6, WIDE>(s, a.team, waves[parity], wave_count);
        const BackToken token = token_of(a, s, inv, of_token);
        if (by_token && a.dgate && on && at.lane == 0) put_token_gate<T>(a, t, token);
        if (!on) continue;
        float x[8], v[8], g[8], z[8], f[8];
        row.h.floats(x), row.dn.floats(v), row.dh.floats(g), row.y.floats(z);
        if (EACH) row.gate.floats(f);
        finish<EACH>(a, token, x, v, g, z, f, q, pre, sum_n, sum_y);
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

// ---- rows past the registers ---------------------------------------------------------

// A block walks a row's pieces once for each step of it; what it reads again comes from
// the caches (8,192 rows of 12,288 BF16 channels backward: 0.57 ms,
// 2.3 times what its bytes take; in single elements 2.3 ms).
constexpr int kAnyThreads = 512;

template <typename S, typename T>
__global__ __launch_bounds__(kAnyThreads) void k_norm_any(NormArgs a) {
    __shared__ float waves[2][1][kMostWaves];
    constexpr int kStep = kAnyThreads * 8, kWaves = kAnyThreads / 64;
    const float inv = 1.0f / (float)a.hidden;
    const bool each = a.gate_form == SDP_GATE_ELEMENT;
    const int c0 = threadIdx.x * 8;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const S *h = (const S *)a.h.data + t * a.h.stride;
        const T *y = (const T *)a.y.data + t * a.y.stride;
        float factor = 1.0f, sq = 0.0f;
        if (a.gate_form == SDP_GATE_TOKEN) factor = gate_of(a, load1((const T *)a.gate + t * a.gate_stride)).act;
        if (a.y.data && a.post_norm) {
            for (int64_t c = c0; c < a.hidden; c += kStep) {
                float v[8];
                load_floats(y + c, a.hidden - c, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) sq += v[k] * v[k];
            }
            team_sums<1, true>(&sq, 0, waves[0], kWaves);
            factor *= rsqrtf(sq * inv + a.eps);
        }
        // the stream's new piece, and the weights of its norm
        auto sum_at = [&](int c, int left, float *x, float *pre) __attribute__((always_inline)) {
            float u[8], add[8], z[8];
            load_floats(h + c, left, x);
            factors_of<T>(a, c, left, add, pre);
            if (!a.y.data) return;
            load_floats(y + c, left, u);
            if (each) load_floats((const T *)a.gate + t * a.gate_stride + c, left, z);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] += u[k] * (each ? gate_of(a, z[k]).act : 1.0f) * factor * add[k];
        };
        float r = 0.0f;
        if (a.n_out.data) {
            sq = 0.0f;
            for (int64_t c = c0; c < a.hidden; c += kStep) {
                float x[8], pre[8];
                sum_at((int)c, (int)(a.hidden - c), x, pre);
#pragma unroll
                for (int k = 0; k < 8; ++k) sq += x[k] * x[k];
            }
            team_sums<1, true>(&sq, 0, waves[1], kWaves);
            r = rsqrtf(sq * inv + a.eps);
        }
        __syncthreads();
        for (int64_t c = c0; c < a.hidden; c += kStep) {
            const int left = (int)(a.hidden - c);
            float x[8], pre[8];
            sum_at((int)c, left, x, pre);
            if (a.h_out.data) store_floats((S *)a.h_out.data + t * a.h_out.stride + c, left, x);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= r * pre[k];
            if (a.n_out.data) store_floats((T *)a.n_out.data + t * a.n_out.stride + c, left, x);
        }
    }
}

template <typename S, typename T, bool EACH>
__global__ __launch_bounds__(kAnyThreads) void k_norm_back_any(NormArgs a) {
    __shared__ float waves[2][6][kMostWaves];
    constexpr int kStep = kAnyThreads * 8, kWaves = kAnyThreads / 64;
    const float inv = 1.0f / (float)a.hidden;
    const int c0 = threadIdx.x * 8;
    // the block's sums over its tokens; a thread's columns are always its own
    float *sums[2];
    for (int w = 0; w < 2; ++w) sums[w] = a.sums[w] ? a.sums[w] + blockIdx.x * sums_stride(a) : nullptr;
    bool first = true;
    int parity = 0;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x, parity ^= 1, first = false) {
        auto fetch = [&](int64_t c, float *x, float *v, float *g, float *z, float *f) __attribute__((always_inline)) {
            const int left = (int)(a.hidden - c);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = v[k] = g[k] = z[k] = 0.0f;
            if (a.dn.data) {
                load_floats((const S *)a.h.data + t * a.h.stride + c, left, x);
                load_floats((const T *)a.dn.data + t * a.dn.stride + c, left, v);
            }
            if (a.dh_out.data) load_floats((const S *)a.dh_out.data + t * a.dh_out.stride + c, left, g);
            if (a.y.data) load_floats((const T *)a.y.data + t * a.y.stride + c, left, z);
            if (EACH) load_floats((const T *)a.gate + t * a.gate_stride + c, left, f);
        };
        float s[6] = {};
        for (int64_t c = c0; c < a.hidden; c += kStep) {
            float x[8], v[8], g[8], z[8], f[8], q[8], pre[8];
            fetch(c, x, v, g, z, f);
            factors_of<T>(a, (int)c, (int)(a.hidden - c), q, pre);
            add_dots<EACH>(a, x, v, g, z, f, q, pre, s);
        }
        team_sums<6, true>(s, 0, waves[parity], kWaves);
        Gate gate = {1.0f, 1.0f};
        if (a.gate_form == SDP_GATE_TOKEN) gate = gate_of(a, load1((const T *)a.gate + t * a.gate_stride));
        const BackToken token = token_of(a, s, inv, gate);
        if (a.gate_form == SDP_GATE_TOKEN && a.dgate && threadIdx.x == 0) put_token_gate<T>(a, t, token);
        for (int64_t c = c0; c < a.hidden; c += kStep) {
            const int left = (int)(a.hidden - c);
            float x[8], v[8], g[8], z[8], f[8], q[8], pre[8], sum[2][8] = {};
            fetch(c, x, v, g, z, f);
            factors_of<T>(a, (int)c, left, q, pre);
#pragma unroll
            for (int w = 0; w < 2; ++w)
                if (sums[w] && !first) load_floats(sums[w] + c, left, sum[w]);
            finish<EACH>(a, token, x, v, g, z, f, q, pre, sum[0], sum[1]);
#pragma unroll
            for (int w = 0; w < 2; ++w)
                if (sums[w]) store_floats(sums[w] + c, left, sum[w]);
            if (a.dh.data) store_floats((S *)a.dh.data + t * a.dh.stride + c, left, g);
            if (a.dy.data) store_floats((T *)a.dy.data + t * a.dy.stride + c, left, v);
            if (EACH && a.dgate) store_floats((T *)a.dgate + t * a.dgate_stride + c, left, f);
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
    // (without tokens the sums are zeros, whatever the gate and the weight hold: neither is read,
    // and the call has not looked where the weight lies)
    const bool some = a.tokens > 0;
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
        const Gate gate = channel && some ? gate_of(a, load1((const T *)a.gate + i + k)) : Gate{1.0f, 1.0f};
        if (a.dpost) put(a.dpost, a.scale * gate.act * s[k]);
        if (a.dgate && channel)
            store1((T *)a.dgate + i + k,
                   a.scale * gate.slope * (a.post_norm && some ? weight_at(a, a.post_weight, i + k) : 1.0f) * s[k]);
    }
}

// Rows without channels: a token's gate has a gradient, the sum over nothing.
template <typename T>
__global__ __launch_bounds__(kAnyThreads) void k_norm_no_channels(NormArgs a) {
    for (int64_t t = (int64_t)blockIdx.x * kAnyThreads + threadIdx.x; t < a.tokens; t += (int64_t)gridDim.x * kAnyThreads)
        store1((T *)a.dgate + t * a.dgate_stride, 0.0f);
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
    return {0, kAnyThreads, 1};
}

// Blocks that a call's rows are walked by: at most as many as the compute units hold at
// once (forward six waves to a SIMD, backward three, or four of 16-bit tensors), and each
// as many rows as the others.  One more block to a unit than it holds waits for the rest:
// 32,768 x 5,120 BF16 forward 247 us in 512 blocks, in 763 265.
int blocks_of(const NormArgs &a, const Split &s, bool backward, bool wide_types) {
    const int64_t per = s.team ? s.threads / s.team : 1, waves = s.threads / 64;
    const int64_t held = !backward ? 24 : wide_types ? 12 : 16;
    const int64_t most = 256 * std::max<int64_t>(1, held / waves);
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

hipError_t launch_norm_no_channels(const NormArgs &a, bool bf16, hipStream_t s) {
    if (a.tokens == 0 || !a.dgate || a.gate_form != SDP_GATE_TOKEN) return hipSuccess;
    const dim3 grid((uint32_t)std::min<int64_t>((a.tokens + kAnyThreads - 1) / kAnyThreads, 1 << 12));
    if (bf16)
        hipLaunchKernelGGL((k_norm_no_channels<uint16_t>), grid, dim3(kAnyThreads), 0, s, a);
    else
        hipLaunchKernelGGL((k_norm_no_channels<float>), grid, dim3(kAnyThreads), 0, s, a);
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
            auto pick = [&](auto each) {
                constexpr bool E = decltype(each)::value;
                if (!split.team) return go(k_norm_back_any<S, T, E>);
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
