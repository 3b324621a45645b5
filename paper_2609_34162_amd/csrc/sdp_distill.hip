// gfx950 kernels of sdp_distill_loss and its backward.
//
// A row needs its largest logit and the two sums S_tau = sum exp((z - max) / tau)
// and S_1 = sum exp(z - max) (one where tau = 1), then its loss from a few
// gathered logits, and its gradient
//   g (a tau (exp(z / tau - L_tau) - q) + b (exp(z - L_1) - [label]))
// The floor is the memory's: each logit read once and each gradient written
// once.  Two ways there:
//  - resident: a block holds a whole row in its registers (a compute unit's hold
//    512 KB, a row of 151,936 BF16 logits 304 KB), so the gradient needs no
//    second read.  While it writes a row's gradient it loads the next row.
//  - split: blocks share a row; one pass leaves each part's sums, a second one
//    joins them and writes the loss and, where it is wanted, the gradient.
// Rows of 151,936 BF16 logits: loss and gradient of 8,192 in one call 1087 us (4.6 TB/s
// of read and written bytes), the gradient alone of 4,096 from the forward's sums 500 us
// (5.0 TB/s), the loss alone of 301 30 us, 24 of them for the sums (3.9 TB/s).
// An exponential takes as long as four multiplications, and two for each logit and
// pass would bound the resident kernel.  Where tau is 2, 3 or 4 (kernels' POWER),
// exp(z) is that power of exp(z / tau) instead.
#include <algorithm>
#include <type_traits>

#include "sdp_ops_device.h"
#include "sdp_ops_internal.h"

namespace sdpops {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- 16 bytes of a row ---------------------------------------------------------

// A row starts wherever its stride puts it, so 16-byte accesses are only aligned
// to an element.
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

template <typename T>
constexpr int kPer = 16 / (int)sizeof(T);

// ONCE: with the non-temporal hint.
template <bool ONCE, typename T>
__device__ __forceinline__ u32x4 load_piece(const T *p) {
    return ONCE ? __builtin_nontemporal_load((const u32x4_any *)p) : *(const u32x4_any *)p;
}
__device__ __forceinline__ void floats_of(u32x4 r, const uint16_t *, float *v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[2 * k] = bf16_lo(r[k]), v[2 * k + 1] = bf16_hi(r[k]);
}
__device__ __forceinline__ void floats_of(u32x4 r, const float *, float *v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void store_piece(uint16_t *p, const float *v) {
    u32x4 u;
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = pack2(v[2 * k], v[2 * k + 1]);
    __builtin_nontemporal_store(u, (u32x4_any *)p);
}
__device__ __forceinline__ void store_piece(float *p, const float *v) {
    u32x4 u;
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = __float_as_uint(v[k]);
    __builtin_nontemporal_store(u, (u32x4_any *)p);
}
// The compiler is not to keep a piece's floats from one use of it to the next:
// a held row has registers for its pieces only.
__device__ __forceinline__ void forget(u32x4 &r) { asm volatile("" : "+v"(r)); }

// Eight or four times minus infinity.
template <typename T>
__device__ __forceinline__ u32x4 nothing() {
    const uint32_t u = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    return u32x4{u, u, u, u};
}

// ---- sums ------------------------------------------------------------------------

// What a kernel does with the two exponents z / tau and z.  POWER 0: only one of
// them is needed; 1: both, two exponentials; 2, 3, 4: both, tau being that number.
template <int POWER>
__device__ __forceinline__ float power(float e) {
    if (POWER == 2) return e * e;
    if (POWER == 3) return e * e * e;
    return (e * e) * (e * e);
}

// The largest of some logits and the sums of 2^((z - top) c) for c = log2(e) / tau
// and log2(e); top = -inf (nothing but -inf) goes with sums of 0 against 0.
// Differences come first: logits as low as the type goes overflow in a product.
struct Sums {
    float top, tau, one;
};

__device__ __forceinline__ float against(float top) { return top == kNegInf ? 0.0f : top; }

__device__ __forceinline__ Sums join(Sums a, Sums b, float c_tau) {
    const float top = fmaxf(a.top, b.top), ref = against(top);
    const float da = a.top - ref, db = b.top - ref;
    return {top, a.tau * exp2_of(da * c_tau) + b.tau * exp2_of(db * c_tau),
            a.one * exp2_of(da * kLog2e) + b.one * exp2_of(db * kLog2e)};
}

__device__ __forceinline__ Sums wave_join(Sums s, float c_tau) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        s = join(s, {__shfl_xor(s.top, d), __shfl_xor(s.tau, d), __shfl_xor(s.one, d)}, c_tau);
    return s;
}

// ---- the teacher and the label of a row --------------------------------------------

struct Row {
    float t_ref;       // the teacher's largest t, and
    float log_sum;     // the logarithm of its sum of exp((t - t_ref) / tau)
    bool has_teacher, has_label, bad;
    int32_t label;     // -1: none
};

// Found by one whole wave.
__device__ Row row_of(const DistillArgs &a, int64_t row) {
    const int lane = threadIdx.x & 63, K = a.k;
    float top = kNegInf, bad = 0.0f;
    for (int j = lane; j < K; j += 64) {
        const int64_t idx = load_int(a.teacher_index, row * K + j, a.index64);
        if (idx >= a.vocab) bad = 1.0f;
        if (idx >= 0) top = fmaxf(top, load_either(a.teacher_logits, row * K + j, a.teacher_bf16));
    }
    top = wave_max(top);
    Row r;
    r.t_ref = against(top);
    const float c_tau = a.inv_tau * kLog2e;
    float sum = 0.0f;
    for (int j = lane; j < K; j += 64)
        if (load_int(a.teacher_index, row * K + j, a.index64) >= 0)
            sum += exp2_of((load_either(a.teacher_logits, row * K + j, a.teacher_bf16) - r.t_ref) * c_tau);
    sum = wave_sum(sum);
    r.log_sum = logf(sum);
    // a NaN among the teacher's logits leaves top alone and makes the sum NaN
    r.has_teacher = a.distill_weight != 0.0f && (top != kNegInf || sum != 0.0f);
    int64_t label = a.labels && a.label_weight != 0.0f ? load_int(a.labels, row, a.index64) : -1;
    if (label >= a.vocab) bad = 1.0f, label = -1;
    r.label = (int32_t)label;
    r.has_label = label >= 0;
    r.bad = wave_max(bad) != 0.0f;
    return r;
}

// Entry j: its place in the row (-1: not there, or past the vocabulary), q and tau log q.
__device__ __forceinline__ int32_t entry(const DistillArgs &a, int64_t row, const Row &r, int j, float *q,
                                         float *tau_log_q) {
    const int64_t idx = load_int(a.teacher_index, row * a.k + j, a.index64);
    const float t = load_either(a.teacher_logits, row * a.k + j, a.teacher_bf16) - r.t_ref;
    *tau_log_q = t - a.tau * r.log_sum;
    *q = idx >= 0 ? exp2_of((t * a.inv_tau - r.log_sum) * kLog2e) : 0.0f;
    return idx >= 0 && idx < a.vocab ? (int32_t)idx : -1;
}

// What one part of a row says to its loss: sum of q (tau log q - (z - ref)) and of q
// over the entries in [v0, v1), and the label's logit less ref.  A loss comes from
// differences to the row's largest logit alone: L - z would lose what the logits'
// distance from zero leaves no bits for, and a row of the type's lowest value has no L.
struct Terms {
    float dot, q, z_label;
};

template <typename T>
__device__ Terms wave_terms(const DistillArgs &a, int64_t row, const Row &r, const T *z, int64_t v0, int64_t v1,
                            float ref) {
    const int lane = threadIdx.x & 63;
    Terms t{0.0f, 0.0f, 0.0f};
    if (r.has_teacher)
        for (int j = lane; j < a.k; j += 64) {
            float q, tau_log_q;
            const int32_t v = entry(a, row, r, j, &q, &tau_log_q);
            if (v < v0 || v >= v1 || q == 0.0f) continue;
            t.dot += q * (tau_log_q - (load1(z + v) - ref));
            t.q += q;
        }
    t.dot = wave_sum(t.dot);
    t.q = wave_sum(t.q);
    if (r.label >= v0 && r.label < v1) t.z_label = load1(z + r.label) - ref;
    return t;
}

// log_tau, log_one: of the sums against the row's largest logit, as the terms are.
__device__ float loss_of(const DistillArgs &a, const Row &r, const Terms &t, float log_tau, float log_one) {
    float loss = 0.0f;
    if (r.has_teacher) loss = a.distill_weight * a.tau * (t.dot + t.q * (a.tau * log_tau));
    if (r.has_label) loss += a.label_weight * (log_one - t.z_label);
    return r.bad ? __builtin_nanf("") : loss;
}

// ---- the gradient --------------------------------------------------------------------

// d = k_tau 2^((z s - r_tau) c) + k_one 2^((z - r_one) log2(e)), before the terms of
// the entries and the label; POWER 0: the first alone, 2 to 4: the second is that
// power of the first.  From the sums of the row r = top, s = 1 and c = log2(e) / tau;
// from their logarithms (BACK) r_tau = L_tau, r_one = L_1, s = 1 / tau and c = log2(e).
struct Slope {
    float s, r_tau, c, k_tau, r_one, k_one;
    float g_tau, g_one;  // what the entries' q and the label's 1 are multiplied by
};

template <int POWER, bool BACK>
__device__ Slope slope_of(const DistillArgs &a, const Row &r, float g, Sums sums, float l_tau, float l_one) {
    Slope d;
    g = r.bad && g != 0.0f ? __builtin_nanf("") : g;
    d.g_tau = r.has_teacher || r.bad ? g * a.distill_weight * a.tau : 0.0f;
    d.g_one = r.has_label || r.bad ? g * a.label_weight : 0.0f;
    const float ref = against(sums.top);
    d.s = BACK ? a.inv_tau : 1.0f;
    d.c = BACK ? kLog2e : a.inv_tau * kLog2e;
    d.r_tau = BACK ? l_tau : ref;
    d.r_one = BACK ? l_one : ref;
    d.k_tau = d.g_tau == 0.0f ? 0.0f : BACK ? d.g_tau : d.g_tau / sums.tau;
    d.k_one = d.g_one == 0.0f ? 0.0f : BACK ? d.g_one : d.g_one / sums.one;
    if (POWER == 0) {
        // one of the terms is off, or both have the same exponent
        if (d.g_tau == 0.0f && d.g_one != 0.0f) d.s = 1.0f, d.c = kLog2e, d.r_tau = d.r_one;
        d.k_tau += d.k_one;
    }
    // exp(z - L_1) = exp(z / tau - L_tau)^tau exp(tau L_tau - L_1)
    if (BACK && POWER >= 2 && d.k_one != 0.0f)
        d.k_one *= exp2_of(__builtin_fmaf((float)POWER, l_tau, -l_one) * kLog2e);
    return d;
}

template <int POWER, bool BACK>
__device__ __forceinline__ float slope_at(const Slope &d, float z) {
    const float diff = BACK ? __builtin_fmaf(z, d.s, -d.r_tau) : z - d.r_tau;
    const float e = exp2_of(diff * d.c);
    if (POWER == 0) return d.k_tau * e;
    if (POWER == 1) return d.k_tau * e + d.k_one * exp2_of((BACK ? z - d.r_one : diff) * kLog2e);
    return d.k_tau * e + d.k_one * power<POWER>(e);
}

// The entries of a row that a block's gradient has to correct, in LDS.
struct Entries {
    int32_t index[SDP_DISTILL_MAX_K + 1];  // -1: not in the block's part; [k]: the label
    float q[SDP_DISTILL_MAX_K + 1];
    float z[SDP_DISTILL_MAX_K + 1];
};

// By one whole wave, before the block writes anything: dlogits may be logits.
template <typename T>
__device__ void gather_entries(const DistillArgs &a, int64_t row, const Row &r, const T *z, int64_t v0, int64_t v1,
                               Entries &e) {
    for (int j = threadIdx.x & 63; j <= a.k; j += 64) {
        float q = 0.0f, tau_log_q;
        int32_t v = r.label;
        if (j < a.k) v = r.has_teacher ? entry(a, row, r, j, &q, &tau_log_q) : -1;
        if (v < v0 || v >= v1) v = -1;
        e.index[j] = v;
        e.q[j] = q;
        e.z[j] = v >= 0 ? load1(z + v) : 0.0f;
    }
}

// After the block has written its part (and met): the entries' elements anew,
// each with all that names it, so that elements named twice are written alike.
template <typename T, int POWER, bool BACK>
__device__ void correct_entries(const DistillArgs &a, const Row &r, const Slope &d, const Entries &e, T *dz) {
    for (int j = threadIdx.x; j <= a.k; j += blockDim.x) {
        const int32_t v = e.index[j];
        if (v < 0) continue;
        float q = 0.0f;
        for (int i = 0; i < a.k; ++i) q += e.index[i] == v ? e.q[i] : 0.0f;
        float s = slope_at<POWER, BACK>(d, e.z[j]);
        if (q != 0.0f) s -= d.g_tau * q;  // (a NaN in the teacher's sum is not the label's)
        if (v == r.label) s -= d.g_one;
        store1(dz + v, s);
    }
}

// ---- split rows ------------------------------------------------------------------------

constexpr int kSplitThreads = 256, kSplitAhead = 4;

struct Part {
    int64_t p0, p1;  // 16-byte pieces
    int64_t v0, v1;  // elements (the last part has the row's last few)
};
template <typename T>
__device__ __forceinline__ Part part_of(const DistillArgs &a, int part, int parts) {
    const int64_t pieces = a.vocab / kPer<T>, each = (pieces + parts - 1) / parts;
    Part p;
    p.p0 = part * each < pieces ? part * each : pieces;
    p.p1 = p.p0 + each < pieces ? p.p0 + each : pieces;
    p.v0 = p.p0 * kPer<T>;
    p.v1 = part == parts - 1 ? a.vocab : p.p1 * kPer<T>;
    return p;
}

// Adds kN logits, the largest of them and of s.top being `top`, to sums against it.
template <int kN, int POWER>
__device__ __forceinline__ void add_against(Sums &s, const float *z, float ref, float c_tau) {
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        const float d = z[k] - ref, e = exp2_of(d * c_tau);
        s.tau += e;
        if (POWER == 1) s.one += exp2_of(d * kLog2e);
        if (POWER >= 2) s.one += power<POWER>(e);
    }
}

// Adds kN logits to a thread's running sums.
template <int kN, int POWER>
__device__ __forceinline__ void add(Sums &s, const float *z, float c_tau) {
    float top = s.top;
#pragma unroll
    for (int k = 0; k < kN; ++k) top = fmaxf(top, z[k]);
    const float ref = against(top);
    if (top > s.top) {
        s.tau *= exp2_of((s.top - ref) * c_tau);
        s.one *= exp2_of((s.top - ref) * kLog2e);
        s.top = top;
    }
    add_against<kN, POWER>(s, z, ref, c_tau);
}

// The sums of part blockIdx.y of row blockIdx.x and, where a gradient follows (it
// may overwrite the logits), what the part says to the loss.
template <typename T, int POWER>
__global__ __launch_bounds__(kSplitThreads) void k_distill_sums(DistillArgs a) {
    constexpr int kN = kPer<T>;
    __shared__ Sums waves[kSplitThreads / 64];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T *z = (const T *)a.logits + row * a.logit_stride;
    const Part p = part_of<T>(a, blockIdx.y, a.splits);
    const float c_tau = a.inv_tau * kLog2e;
    Sums s{kNegInf, 0.0f, 0.0f};
    for (int64_t i = p.p0 + tid; i < p.p1; i += kSplitThreads * kSplitAhead) {
        u32x4 r[kSplitAhead];
#pragma unroll
        for (int u = 0; u < kSplitAhead; ++u)
            r[u] = i + u * kSplitThreads < p.p1 ? load_piece<false>(z + (i + u * kSplitThreads) * kN) : nothing<T>();
#pragma unroll
        for (int u = 0; u < kSplitAhead; ++u) {
            float v[kN];
            floats_of(r[u], z, v);
            add<kN, POWER>(s, v, c_tau);
        }
    }
    const int64_t rest = p.p1 * kN + tid;
    if (rest < p.v1) {
        const float v = load1(z + rest);
        add<1, POWER>(s, &v, c_tau);
    }
    if (POWER == 0) s.one = s.tau;
    s = wave_join(s, c_tau);
    if ((tid & 63) == 0) waves[tid >> 6] = s;
    __syncthreads();
    if (tid >= 64) return;
    s = waves[0];
#pragma unroll
    for (int w = 1; w < kSplitThreads / 64; ++w) s = join(s, waves[w], c_tau);
    Terms t{0.0f, 0.0f, 0.0f};
    bool label_here = false;
    if (a.dlogits) {
        const Row r = row_of(a, row);
        t = wave_terms<T>(a, row, r, z, p.v0, p.v1, against(s.top));
        label_here = r.label >= p.v0 && r.label < p.v1;
    }
    if (tid == 0) {
        float *out = a.partials + (row * a.splits + blockIdx.y) * kDistillPartials;
        out[0] = s.top, out[1] = s.tau, out[2] = s.one;
        out[3] = t.dot, out[4] = t.q, out[5] = t.z_label, out[6] = label_here ? 1.0f : 0.0f;
    }
}

// The parts of a row joined, by one whole wave, a lane to each part (parts_of: 64 at most).
__device__ void join_parts(const DistillArgs &a, int64_t row, Sums *s, Terms *t) {
    const int part = threadIdx.x & 63;
    Sums mine{kNegInf, 0.0f, 0.0f};
    *t = Terms{0.0f, 0.0f, 0.0f};
    bool label_here = false;
    if (part < a.splits) {
        const float *p = a.partials + (row * a.splits + part) * kDistillPartials;
        mine = Sums{p[0], p[1], p[2]};
        *t = Terms{p[3], p[4], p[5]};
        label_here = p[6] != 0.0f;
    }
    *s = wave_join(mine, a.inv_tau * kLog2e);
    // the terms from the part's largest logit to the row's
    const float up = against(mine.top) - against(s->top);
    if (t->q != 0.0f) t->dot -= t->q * up;
    if (label_here) t->z_label += up;
    t->dot = wave_sum(t->dot), t->q = wave_sum(t->q), t->z_label = wave_sum(t->z_label);
}

__device__ void write_loss(const DistillArgs &a, int64_t row, const Row &r, const Sums &s, const Terms &t) {
    const float log_tau = logf(s.tau), log_one = logf(s.one), ref = against(s.top);
    a.loss[row] = loss_of(a, r, t, log_tau, log_one);
    if (a.lse) {
        a.lse[2 * row] = log_tau + ref * a.inv_tau;
        a.lse[2 * row + 1] = log_one + ref;
    }
}

// The loss alone: a wave joins a row's parts.
template <typename T>
__global__ __launch_bounds__(64) void k_distill_loss(DistillArgs a) {
    const int64_t row = blockIdx.x;
    const Row r = row_of(a, row);
    Sums s;
    Terms t;
    join_parts(a, row, &s, &t);
    t = wave_terms<T>(a, row, r, (const T *)a.logits + row * a.logit_stride, 0, a.vocab, against(s.top));
    if (threadIdx.x == 0) write_loss(a, row, r, s, t);
}

// The gradient of part blockIdx.y of row blockIdx.x, from the joined parts (and
// the loss, by part 0) or, backward, from lse.
template <typename T, int POWER, bool BACK, bool ONCE>
__global__ __launch_bounds__(kSplitThreads) void k_distill_gradient(DistillArgs a) {
    constexpr int kN = kPer<T>;
    __shared__ Entries entries;
    __shared__ Slope shared_slope;
    __shared__ Row shared_row;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T *z = (const T *)a.logits + row * a.logit_stride;
    T *dz = (T *)a.dlogits + row * a.dlogits_stride;
    const Part p = part_of<T>(a, blockIdx.y, a.parts);
    if (tid < 64) {
        const Row r = row_of(a, row);
        const float g = a.row_grad[row];
        Slope d;
        if (BACK) {
            d = slope_of<POWER, true>(a, r, g, {}, a.lse_in[2 * row], a.lse_in[2 * row + 1]);
        } else {
            Sums s;
            Terms t;
            join_parts(a, row, &s, &t);
            d = slope_of<POWER, false>(a, r, g, s, 0.0f, 0.0f);
            if (blockIdx.y == 0 && tid == 0) write_loss(a, row, r, s, t);
        }
        gather_entries(a, row, r, z, p.v0, p.v1, entries);
        if (tid == 0) shared_slope = d, shared_row = r;
    }
    __syncthreads();
    const Slope d = shared_slope;
    const Row r = shared_row;
    if (d.k_tau == 0.0f && d.k_one == 0.0f) {
        // nothing here is learned from: zeros, whatever the logits hold
        const float zero[kN] = {};
        for (int64_t i = p.p0 + tid; i < p.p1; i += kSplitThreads) store_piece(dz + i * kN, zero);
        if (p.p1 * kN + tid < p.v1) store1(dz + p.p1 * kN + tid, 0.0f);
        return;
    }
    for (int64_t i = p.p0 + tid; i < p.p1; i += kSplitThreads * kSplitAhead) {
        u32x4 raw[kSplitAhead];
#pragma unroll
        for (int u = 0; u < kSplitAhead; ++u)
            raw[u] = i + u * kSplitThreads < p.p1 ? load_piece<ONCE>(z + (i + u * kSplitThreads) * kN) : nothing<T>();
#pragma unroll
        for (int u = 0; u < kSplitAhead; ++u) {
            if (i + u * kSplitThreads >= p.p1) break;
            float v[kN];
            floats_of(raw[u], z, v);
#pragma unroll
            for (int k = 0; k < kN; ++k) v[k] = slope_at<POWER, BACK>(d, v[k]);
            store_piece(dz + (i + u * kSplitThreads) * kN, v);
        }
    }
    const int64_t rest = p.p1 * kN + tid;
    if (rest < p.v1) store1(dz + rest, slope_at<POWER, BACK>(d, load1(z + rest)));
    __syncthreads();
    correct_entries<T, POWER, BACK>(a, r, d, entries, dz);
}

// ---- resident rows ------------------------------------------------------------------------

// The largest of 8 BF16 values at a time as 16-bit integers: right if it is not
// negative, as then the order of the bits is that of the values (a NaN with its
// sign clear comes out largest, and makes the sums NaN as it should).
typedef __attribute__((ext_vector_type(8))) short s16x8;
__device__ __forceinline__ s16x8 top_bits(s16x8 m, u32x4 r) {
    return __builtin_elementwise_max(m, __builtin_bit_cast(s16x8, r));
}
__device__ __forceinline__ float top_of_bits(s16x8 m) {
    short t = m[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) t = t > m[k] ? t : m[k];
    return t >= 0 ? __uint_as_float((uint32_t)t << 16) : kNegInf;
}

// A block of THREADS holds a row in up to NV 16-byte pieces a thread.  SUMS and
// POWER: the sums' and the gradient's.
template <typename T, int THREADS, int NV, int SUMS, int POWER>
__global__ __launch_bounds__(THREADS) void k_distill_resident(DistillArgs a) {
    constexpr int kN = kPer<T>, kWaves = THREADS / 64;
    // the entries (q: t at first, then q times t_sum) of this row and the next;
    // entry j, and the label as entry k, belong to thread j mod THREADS
    __shared__ Entries both[2];
    __shared__ float red[4][kWaves];
    __shared__ int bad_waves[kWaves];
    const int tid = threadIdx.x, wave = tid >> 6;
    const int pieces = a.vocab / kN, rest = pieces * kN + tid;
    const float c_tau = a.inv_tau * kLog2e;
    const bool labels = a.labels && a.label_weight != 0.0f, teacher = a.distill_weight != 0.0f;
    const T *const type = nullptr;
    u32x4 held[NV];
    float last = kNegInf;
    int64_t row = blockIdx.x;
    // a thread's pieces are THREADS apart: one offset, and a scalar base for each
    const uint32_t at = (uint32_t)tid * kN;
    // places and t of a row's entries (-inf where their term is off); an index past
    // the vocabulary is kept as its size
    auto fetch_entries = [&](int64_t of, Entries &en) __attribute__((always_inline)) {
#pragma unroll 1
        for (int j = tid; j <= a.k; j += THREADS) {
            int64_t v = -1;
            float t = kNegInf;
            if (j < a.k) {
                v = load_int(a.teacher_index, of * a.k + j, a.index64);
                if (teacher) t = load_either(a.teacher_logits, of * a.k + j, a.teacher_bf16);
            } else if (labels) {
                v = load_int(a.labels, of, a.index64);
            }
            en.index[j] = v < 0 ? -1 : v < a.vocab ? (int32_t)v : a.vocab;
            en.q[j] = v < 0 ? kNegInf : t;
        }
    };
    // and their logits, from the same thread
    auto fetch_logits = [&](const T *z, Entries &en) __attribute__((always_inline)) {
#pragma unroll 1
        for (int j = tid; j <= a.k; j += THREADS) {
            const int32_t v = en.index[j];
            en.z[j] = v >= 0 && v < a.vocab ? load1(z + v) : 0.0f;
        }
    };
    {
        const T *z = (const T *)a.logits + row * a.logit_stride;
        fetch_entries(row, both[0]);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            held[j] = tid + j * THREADS < pieces ? load_piece<true>(z + j * THREADS * kN + at) : nothing<T>();
        if (rest < a.vocab) last = load1(z + rest);
        fetch_logits(z, both[0]);
    }
    // over the block's threads: the largest x, and y
    auto block_top = [&](float x, float y, float *y_top) __attribute__((always_inline)) {
        x = wave_max(x), y = wave_max(y);
        __syncthreads();
        if ((tid & 63) == 0) red[0][wave] = x, red[1][wave] = y;
        __syncthreads();
        x = red[0][tid & (kWaves - 1)], y = red[1][tid & (kWaves - 1)];
#pragma unroll
        for (int w = 1; w < kWaves; w <<= 1) x = fmaxf(x, __shfl_xor(x, w)), y = fmaxf(y, __shfl_xor(y, w));
        *y_top = y;
        return x;
    };
    auto block_sum = [&](const float *of) __attribute__((always_inline)) {
        float x = of[tid & (kWaves - 1)];
#pragma unroll
        for (int w = 1; w < kWaves; w <<= 1) x += __shfl_xor(x, w);
        return x;
    };
    for (int parity = 0; row < a.rows; row += gridDim.x, parity ^= 1) {
        Entries &entries = both[parity], &entries_next = both[parity ^ 1];
        float t_top = kNegInf;
        bool bad = false;
#pragma unroll 1
        for (int j = tid; j <= a.k; j += THREADS) {
            t_top = fmaxf(t_top, entries.q[j]);
            bad = bad || entries.index[j] == a.vocab;
        }
        const bool wave_bad = __any(bad);
        if ((tid & 63) == 0) bad_waves[wave] = wave_bad;
        float top = kNegInf;
        if constexpr (kN == 8) {
            s16x8 m = (short)-32768;
#pragma unroll
            for (int j = 0; j < NV; ++j) m = top_bits(m, held[j]);
            const float own = top_of_bits(m);
            // a negative one says nothing while pieces may hold larger ones unseen
            top = block_top(last >= 0.0f ? fmaxf(own, last) : own, t_top, &t_top);
        }
        if (kN != 8 || top == kNegInf) {
            // 32 bits, or no value in the row that is not negative
            top = last;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float v[kN];
                floats_of(held[j], type, v);
#pragma unroll
                for (int k = 0; k < kN; ++k) top = fmaxf(top, v[k]);
                forget(held[j]);
            }
            top = block_top(top, t_top, &t_top);
        }
        const float ref = against(top), t_ref = against(t_top);
        // the teacher's sum of exp((t - t_ref) / tau), and of that times t - t_ref - (z - ref)
        float t_sum = 0.0f, t_dot = 0.0f;
#pragma unroll 1
        for (int j = tid; j <= a.k; j += THREADS) {
            const float t = entries.q[j];
            const float q = t != kNegInf ? exp2_of((t - t_ref) * c_tau) : 0.0f;
            t_sum += q;
            if (q != 0.0f) t_dot += q * (t - t_ref - (entries.z[j] - ref));
            entries.q[j] = q;
            if (entries.index[j] == a.vocab) entries.index[j] = -1;
        }
        Sums mine{top, 0.0f, 0.0f};
        add_against<1, SUMS>(mine, &last, ref, c_tau);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float v[kN];
            floats_of(held[j], type, v);
            add_against<kN, SUMS>(mine, v, ref, c_tau);
            forget(held[j]);
        }
        const float w_tau = wave_sum(mine.tau), w_one = SUMS ? wave_sum(mine.one) : 0.0f;
        t_sum = wave_sum(t_sum), t_dot = wave_sum(t_dot);
        __syncthreads();
        if ((tid & 63) == 0) red[0][wave] = w_tau, red[1][wave] = w_one, red[2][wave] = t_sum, red[3][wave] = t_dot;
        __syncthreads();
        Sums s{top, block_sum(red[0]), SUMS ? block_sum(red[1]) : 0.0f};
        t_sum = block_sum(red[2]), t_dot = block_sum(red[3]);
        Row r;
        r.bad = __any(bad_waves[tid & (kWaves - 1)]);
        if (!SUMS) s.one = s.tau;
        r.has_teacher = teacher && (t_top != kNegInf || t_sum != 0.0f);
        r.label = labels ? entries.index[a.k] : -1;
        r.has_label = r.label >= 0;
        if (tid == 0) {
            // sum of q (tau log q - (z - ref)), the q's sum being 1
            Terms terms{t_dot / t_sum - a.tau * logf(t_sum), 1.0f, entries.z[a.k] - ref};
            write_loss(a, row, r, s, terms);
        }
        Slope d = slope_of<POWER, false>(a, r, a.row_grad[row], s, 0.0f, 0.0f);
        const bool zeros = d.k_tau == 0.0f && d.k_one == 0.0f;

        T *dz = (T *)a.dlogits + row * a.dlogits_stride;
        const int64_t next = row + gridDim.x;
        const T *zn = (const T *)a.logits + (next < a.rows ? next : row) * a.logit_stride;
        const int pieces_next = next < a.rows ? pieces : 0;
        if (next < a.rows) fetch_entries(next, entries_next);
        if (rest < a.vocab) store1(dz + rest, zeros ? 0.0f : slope_at<POWER, false>(d, last));
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = tid + j * THREADS;
            float v[kN];
            floats_of(held[j], type, v);
#pragma unroll
            for (int k = 0; k < kN; ++k) v[k] = zeros ? 0.0f : slope_at<POWER, false>(d, v[k]);
            if (i < pieces) store_piece(dz + j * THREADS * kN + at, v);
            // its register takes the next row's piece
            held[j] = i < pieces_next ? load_piece<true>(zn + j * THREADS * kN + at) : nothing<T>();
        }
        last = rest < a.vocab && next < a.rows ? load1(zn + rest) : kNegInf;
        if (next < a.rows) fetch_logits(zn, entries_next);
        __syncthreads();
        // entries.q is q times t_sum
        if (r.has_teacher) d.g_tau /= t_sum;
        if (!zeros) correct_entries<T, POWER, false>(a, r, d, entries, dz);
        __syncthreads();
    }
}

// POWER of the sums (both are wanted: lse holds both), and of the gradient.
int sums_power(const DistillArgs &a) {
    if (a.tau == 1.0f) return 0;
    return a.tau == 2.0f ? 2 : a.tau == 3.0f ? 3 : a.tau == 4.0f ? 4 : 1;
}
int gradient_power(const DistillArgs &a) {
    return a.distill_weight != 0.0f && a.label_weight != 0.0f && a.labels ? sums_power(a) : 0;
}

constexpr int kMostHeld = 19;  // pieces a thread, of 1,024: what 128 registers hold beside the work on them

template <typename T, int THREADS, int NV>
void launch_resident(const DistillArgs &a, int per_cu, hipStream_t s) {
    const dim3 grid((uint32_t)std::min<int64_t>(a.rows, 256 * per_cu));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(THREADS), 0, s, a); };
    switch (gradient_power(a)) {
        case 1: return go(k_distill_resident<T, THREADS, NV, 1, 1>);
        case 2: return go(k_distill_resident<T, THREADS, NV, 2, 2>);
        case 3: return go(k_distill_resident<T, THREADS, NV, 3, 3>);
        case 4: return go(k_distill_resident<T, THREADS, NV, 4, 4>);
        default: break;
    }
    if (sums_power(a) == 0)
        go(k_distill_resident<T, THREADS, NV, 0, 0>);
    else
        go(k_distill_resident<T, THREADS, NV, 1, 0>);
}

// 16-byte pieces of a row.
int64_t pieces_of(const DistillArgs &a, bool bf16) { return a.vocab / (bf16 ? 8 : 4); }

// Whether rows stay in registers: a gradient is wanted, a row fits a compute
// unit's, and there are rows enough to give most units one.  Loss and gradient of
// 4,096 BF16 rows of 155,648 (held): 587 us, of 155,660 (read twice): 810; of 151,936
// and 192 rows: 37 us, 191 rows (shared by blocks): 48.
bool resident(const DistillArgs &a, bool bf16) {
    return a.dlogits && pieces_of(a, bf16) <= kMostHeld * 1024 && a.rows >= 192;
}

template <typename T>
void launch_resident_any(const DistillArgs &a, hipStream_t s) {
    const int64_t n = pieces_of(a, sizeof(T) == 2);
    if (n <= 4 * 256) return launch_resident<T, 256, 4>(a, 6, s);
    if (n <= 8 * 256) return launch_resident<T, 256, 8>(a, 6, s);
    if (n <= 16 * 256) return launch_resident<T, 256, 16>(a, 4, s);
    if (n <= 8 * 1024) return launch_resident<T, 1024, 8>(a, 1, s);
    if (n <= 12 * 1024) return launch_resident<T, 1024, 12>(a, 1, s);
    if (n <= 16 * 1024) return launch_resident<T, 1024, 16>(a, 1, s);
    return launch_resident<T, 1024, kMostHeld>(a, 1, s);
}

// Parts of a row so that the grid fills the compute units several times, none
// smaller than a block's loads.
int parts_of(const DistillArgs &a, bool bf16) {
    const int64_t want = (2048 + a.rows - 1) / std::max<int64_t>(1, a.rows);
    const int64_t most = std::max<int64_t>(1, pieces_of(a, bf16) / (kSplitThreads * kSplitAhead));
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, most, 64}));
}

template <typename T, bool BACK>
void launch_gradient(const DistillArgs &a, hipStream_t s) {
    const dim3 grid((uint32_t)a.rows, a.parts);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSplitThreads), 0, s, a); };
    // from 256 MB of logits and gradients on, the last-level cache's size, with the
    // non-temporal hint (4,096 rows of 151,936 in BF16: 496 us against 508)
    const bool once = a.rows * a.vocab * (int64_t)(2 * sizeof(T)) > (int64_t)256 << 20;
    auto pick = [&](auto power) {
        constexpr int P = decltype(power)::value;
        once ? go(k_distill_gradient<T, P, BACK, true>) : go(k_distill_gradient<T, P, BACK, false>);
    };
    switch (gradient_power(a)) {
        case 0: return pick(std::integral_constant<int, 0>{});
        case 2: return pick(std::integral_constant<int, 2>{});
        case 3: return pick(std::integral_constant<int, 3>{});
        case 4: return pick(std::integral_constant<int, 4>{});
        default: return pick(std::integral_constant<int, 1>{});
    }
}

template <typename T>
hipError_t launch_forward(const DistillArgs &a, hipStream_t s) {
    if (a.splits == 0) {
        launch_resident_any<T>(a, s);
        return hipGetLastError();
    }
    const dim3 grid((uint32_t)a.rows, a.splits);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSplitThreads), 0, s, a); };
    switch (sums_power(a)) {
        case 0: go(k_distill_sums<T, 0>); break;
        case 2: go(k_distill_sums<T, 2>); break;
        case 3: go(k_distill_sums<T, 3>); break;
        case 4: go(k_distill_sums<T, 4>); break;
        default: go(k_distill_sums<T, 1>); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.dlogits)
        launch_gradient<T, false>(a, s);
    else
        hipLaunchKernelGGL((k_distill_loss<T>), dim3((uint32_t)a.rows), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int distill_splits(const DistillArgs &a, bool bf16) { return resident(a, bf16) ? 0 : parts_of(a, bf16); }

hipError_t launch_distill(const DistillArgs &args, bool bf16, hipStream_t s) {
    if (args.rows == 0) return hipSuccess;
    DistillArgs a = args;
    a.parts = parts_of(a, bf16);
    return bf16 ? launch_forward<uint16_t>(a, s) : launch_forward<float>(a, s);
}

hipError_t launch_distill_backward(const DistillArgs &args, bool bf16, hipStream_t s) {
    if (args.rows == 0) return hipSuccess;
    DistillArgs a = args;
    // parts of about 16 KB and more
    a.parts = (int)std::max<int64_t>(parts_of(a, bf16), std::min<int64_t>(8, pieces_of(a, bf16) / (2 * kSplitThreads * kSplitAhead)));
    bf16 ? launch_gradient<uint16_t, true>(a, s) : launch_gradient<float, true>(a, s);
    return hipGetLastError();
}

}  // namespace sdpops
