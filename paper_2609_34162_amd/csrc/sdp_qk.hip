// gfx950 kernels of sdp_qk_norm_rope and its backward.
//
// For a head's row x of D elements, r = 1 / sqrt(mean(x^2) + eps):
//   n = x r w;  each rotated pair (a, b) of n becomes (a c - b s, b c + a s)
// and backward, with dn the rotation's transpose of dy and u = dn w:
//   dx = r (u - x r mean(u x r)),  dw = sum over rows of dn x r
// Every element is read once and written once: HBM bounds both directions.
// 32,768 tokens of 48 heads of 128 in BF16, views of a fused projection: forward
// 160 us (5.1 TB/s of the tensors' bytes), backward 251 us (4.8 TB/s); a copy of
// 4 GiB reaches 4.7 to 4.8.
#include <algorithm>

#include "sdp_ops_device.h"
#include "sdp_ops_internal.h"

namespace sdpops {
namespace {

constexpr int kRowWaves = 4;  // of a block, in both kernels

// Where element i of a row finds the other one of its rotated pair, the
// pair's angle and the sign of the partner's sine term.
struct Pair {
    int other, angle;
    float sign;
};

__device__ __forceinline__ Pair pair_of(int i, int rotary, int interleaved) {
    const int half = rotary / 2;
    if (interleaved) return {i ^ 1, i >> 1, (i & 1) ? 1.0f : -1.0f};
    return i < half ? Pair{i + half, i, -1.0f} : Pair{i - half, i - half, 1.0f};
}

// Any head size, stride and alignment: a wave takes a row, a lane the elements
// lane, lane + 64, ...; partners of a rotated pair meet in LDS.  Backward, each
// block walks rows a grid apart and keeps its sums of dn x r in registers.
template <typename T, bool BACK>
__global__ __launch_bounds__(64 * kRowWaves) void k_qk_rows(QkArgs a) {
    constexpr int kPer = SDP_QK_MAX_HEAD_DIM / 64;
    __shared__ float row_of[kRowWaves][SDP_QK_MAX_HEAD_DIM];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int which = (int)blockIdx.x < a.blocks[0] ? 0 : 1;
    const QkSide &side = a.side[which];
    const int block = (int)blockIdx.x - (which ? a.blocks[0] : 0);
    const int D = a.dim;
    float *buf = row_of[wave];
    float sums[kPer];
    for (int k = 0; k < kPer; ++k) sums[k] = 0.0f;

    for (int64_t first = (int64_t)block * kRowWaves; first < a.rows_total[which];
         first += (int64_t)a.blocks[which] * kRowWaves) {
        const int64_t row = first + wave;
        const bool on = row < a.rows_total[which];
        float x[kPer], y[kPer];
        int64_t at = 0;
        float r = 0.0f;
        T *out = nullptr;
        if (on) {
            const int64_t token = row / side.heads;
            const int64_t h = row - token * side.heads, b = token / a.tokens, s = token - b * a.tokens;
            at = a.positions ? load_int(a.positions, token, a.positions64) : s;
            const T *px = (const T *)side.x.data + b * side.x.b + s * side.x.s + h * side.x.h;
            out = (T *)side.out.data + b * side.out.b + s * side.out.s + h * side.out.h;
            float sq = 0.0f;
            for (int k = 0; k < kPer; ++k) {
                const int i = lane + 64 * k;
                x[k] = i < D ? load1(px + i) : 0.0f;
                sq += x[k] * x[k];
            }
            r = rsqrtf(wave_sum(sq) / (float)D + a.eps);
            if (BACK) {
                const T *py = (const T *)side.y.data + b * side.y.b + s * side.y.s + h * side.y.h;
                for (int k = 0; k < kPer; ++k) {
                    const int i = lane + 64 * k;
                    y[k] = i < D ? load1(py + i) : 0.0f;
                }
            } else {
                for (int k = 0; k < kPer; ++k) {
                    const int i = lane + 64 * k;
                    const float w = side.weight && i < D ? load_either(side.weight, i, a.weight_bf16) : 1.0f;
                    y[k] = x[k] * r * w;
                }
            }
            for (int k = 0; k < kPer; ++k) {
                const int i = lane + 64 * k;
                if (i < D) buf[i] = y[k];
            }
        }
        __syncthreads();
        if (on) {
            const bool in_table = a.rotary == 0 || (at >= 0 && at < a.table_rows);
            for (int k = 0; k < kPer; ++k) {
                const int i = lane + 64 * k;
                if (i < a.rotary) {
                    const Pair p = pair_of(i, a.rotary, a.interleaved);
                    float c = __builtin_nanf(""), s = c;
                    if (in_table) {
                        c = a.cos[at * (a.rotary / 2) + p.angle];
                        s = a.sin[at * (a.rotary / 2) + p.angle];
                    }
                    y[k] = y[k] * c + (BACK ? -p.sign : p.sign) * s * buf[p.other];
                } else if (!in_table) {
                    y[k] = __builtin_nanf("");
                }
            }
            if (BACK) {
                float dot = 0.0f;
                for (int k = 0; k < kPer; ++k) {
                    const int i = lane + 64 * k;
                    if (i >= D) continue;
                    const float unit = x[k] * r;
                    sums[k] += y[k] * unit;
                    y[k] *= side.weight ? load_either(side.weight, i, a.weight_bf16) : 1.0f;
                    dot += y[k] * unit;
                }
                dot = wave_sum(dot) / (float)D;
                for (int k = 0; k < kPer; ++k) y[k] = r * (y[k] - x[k] * r * dot);
            }
            for (int k = 0; k < kPer; ++k) {
                const int i = lane + 64 * k;
                if (i < D) store1(out + i, y[k]);
            }
        }
        __syncthreads();
    }
    if (BACK && side.partials) {
        for (int k = 0; k < kPer; ++k) {
            const int i = lane + 64 * k;
            if (i < D) buf[i] = sums[k];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < D; i += 64 * kRowWaves) {
            float s = 0.0f;
            for (int w = 0; w < kRowWaves; ++w) s += row_of[w][i];
            side.partials[(int64_t)block * D + i] = s;
        }
    }
}

// Rows whose 8-element pieces are 16-byte aligned: G lanes take a row, a lane a
// piece of 8, so that a wave reads 64 / G rows at once; the partners of a lane's
// elements are in the same lane (interleaved), or each half piece's rotary / 8
// half pieces on.  A wave takes a
// run of heads of one token (of several where a token has fewer heads than rows
// fit), so that it reads a token's position and angles once and steps from row to
// row by additions; the norm's weight goes into the angles:
// y = r (x (w c) -+ x' (w' s)).
// Loads and stores of 16 bytes, with the non-temporal hint where a call's data
// does not fit the last-level cache (see split).
template <bool STREAM, typename V>
__device__ __forceinline__ V load16(const void *p) {
    return STREAM ? __builtin_nontemporal_load((const V *)p) : *(const V *)p;
}
template <bool STREAM, typename V>
__device__ __forceinline__ void store16(void *p, V v) {
    if (STREAM)
        __builtin_nontemporal_store(v, (V *)p);
    else
        *(V *)p = v;
}

// 8 elements of a row as they are stored, and as floats.
template <typename T>
struct Piece;
template <>
struct Piece<uint16_t> {
    u32x4 raw;
    template <bool STREAM>
    __device__ __forceinline__ void load(const uint16_t *p) { raw = load16<STREAM, u32x4>(p); }
    __device__ __forceinline__ void clear() { raw = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void floats(float *v) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[2 * k] = bf16_lo(raw[k]), v[2 * k + 1] = bf16_hi(raw[k]);
    }
    // each half from another lane, SWAP: the other half there
    template <bool SWAP>
    __device__ __forceinline__ Piece partners(const int *lane) const {
        Piece o;
#pragma unroll
        for (int k = 0; k < 4; ++k) o.raw[k] = __shfl(raw[SWAP ? k ^ 2 : k], lane[SWAP ? k / 2 : 0]);
        return o;
    }
    template <bool STREAM>
    static __device__ __forceinline__ void store(uint16_t *p, const float *v) {
        u32x4 u;
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = pack2(v[2 * k], v[2 * k + 1]);
        store16<STREAM>(p, u);
    }
};
template <>
struct Piece<float> {
    f32x4 a, b;
    template <bool STREAM>
    __device__ __forceinline__ void load(const float *p) {
        a = load16<STREAM, f32x4>(p), b = load16<STREAM, f32x4>(p + 4);
    }
    __device__ __forceinline__ void clear() { a = b = f32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void floats(float *v) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
    }
    template <bool SWAP>
    __device__ __forceinline__ Piece partners(const int *lane) const {
        Piece o;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            o.a[k] = __shfl(SWAP ? b[k] : a[k], lane[0]);
            o.b[k] = __shfl(SWAP ? a[k] : b[k], lane[SWAP ? 1 : 0]);
        }
        return o;
    }
    template <bool STREAM>
    static __device__ __forceinline__ void store(float *p, const float *v) {
        store16<STREAM>(p, f32x4{v[0], v[1], v[2], v[3]});
        store16<STREAM>(p + 4, f32x4{v[4], v[5], v[6], v[7]});
    }
};

// Sum over the G lanes of a row.
template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int d = G / 2; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// How a rotated pair lies in a row: neighbours; or half the rotated dimensions
// apart, an even or an odd number of half pieces.
enum Pairs { kNeighbours, kHalves, kHalvesOdd };

template <typename T, int G, Pairs PAIRS, bool BACK, bool STREAM>
__global__ __launch_bounds__(256) void k_qk_tokens(QkArgs a) {
    constexpr bool INTERLEAVED = PAIRS == kNeighbours, kSwap = PAIRS == kHalvesOdd;
    constexpr int kAhead = 4;  // how many wavefuls of rows are loaded before they are worked on
    const int lane = threadIdx.x & 63, piece = lane % G, i = piece * 8;
    const int D = a.dim, half = a.rotary / 2;
    const bool in_row = i < D, turned = i < a.rotary;
    // of each half piece (of both where they cannot differ): whether it comes first
    // in its pairs, and the lane that has its partner
    constexpr int kOwn = kSwap ? 1 : 0;
    const bool first[2] = {i < half, i + 4 < half};
    int partner[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
        partner[j] = lane - piece + (first[j] ? 2 * piece + j + half / 4 : 2 * piece + j - half / 4) / 2;
    const int which = (int)blockIdx.x < a.blocks[0] ? 0 : 1;
    const QkSide &side = a.side[which];
    const int block = (int)blockIdx.x - (which ? a.blocks[0] : 0);
    float sums[8] = {};
    // the wave's 64 / G rows: `at_once` heads (a power of two) of each of several tokens
    const int at_once = 1 << a.heads_log[which], tokens_log = __builtin_ctz(64 / G) - a.heads_log[which];
    const int head = lane / G & (at_once - 1), token_in_wave = lane / G >> a.heads_log[which];
    const int64_t all_tokens = (int64_t)a.batch * a.tokens;
    const int64_t chunks = a.chunks[which];
    const int64_t waves = (int64_t)a.blocks[which] * 4;
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = side.weight && in_row ? load_either(side.weight, i + k, a.weight_bf16) : 1.0f;
    // the wave's item: a run of heads of the tokens from (b0, s0) on; from one
    // item to the next by additions, as divisions would cost more than a row
    int64_t item = (int64_t)block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t group0 = item / chunks, left = all_tokens - (group0 << tokens_log);  // tokens from the first one on
    int chunk = (int)(item - group0 * chunks);
    int64_t b0 = (group0 << tokens_log) / a.tokens, s0 = (group0 << tokens_log) - b0 * a.tokens;
    const int64_t more_groups = waves / chunks, more_b = (more_groups << tokens_log) / a.tokens,
                  more_s = (more_groups << tokens_log) - more_b * a.tokens;
    const int more_chunks = (int)(waves - more_groups * chunks);
    for (; left > 0;
         chunk += more_chunks, left -= more_groups << tokens_log, b0 += more_b, s0 += more_s) {
        if (chunk >= chunks) {
            chunk -= (int)chunks;
            left -= 1 << tokens_log;
            s0 += 1 << tokens_log;
        }
        for (; s0 >= a.tokens; ++b0) s0 -= a.tokens;
        if (left <= 0) break;
        const bool has_token = token_in_wave < left;
        int64_t b = b0, s = s0;
        if (tokens_log > 0) {
            s += has_token ? token_in_wave : 0;
            for (; s >= a.tokens; ++b) s -= a.tokens;
        }
        const int64_t at = a.positions ? load_int(a.positions, b * a.tokens + s, a.positions64) : s;
        const int h0 = chunk * a.chunk_heads, h1 = min(h0 + a.chunk_heads, side.heads);
        const T *px = (const T *)side.x.data + b * side.x.b + s * side.x.s + i;
        const T *py = BACK ? (const T *)side.y.data + b * side.y.b + s * side.y.s + i : nullptr;
        T *po = (T *)side.out.data + b * side.out.b + s * side.out.s + i;

        const bool lost = a.rotary > 0 && (at < 0 || at >= a.table_rows);
        float c[8], sn[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = 1.0f, sn[k] = 0.0f;
        if (turned && !lost) {
#pragma unroll
            for (int k = 0; k < (INTERLEAVED ? 4 : 8); k += 4) {
                const int64_t angle = at * half + (INTERLEAVED ? i / 2 : first[k / 4 * kOwn] ? i + k : i + k - half);
                const f32x4 cv = *(const f32x4 *)(a.cos + angle), sv = *(const f32x4 *)(a.sin + angle);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (INTERLEAVED) {
                        c[2 * e] = c[2 * e + 1] = cv[e];
                        sn[2 * e] = -sv[e], sn[2 * e + 1] = sv[e];
                    } else {
                        c[k + e] = cv[e];
                        sn[k + e] = first[k / 4 * kOwn] ? -sv[e] : sv[e];
                    }
                }
            }
        }
        if (!BACK) {
            // the weights into the angles: its own with the cosine, its partner's with the sine
            float wp[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) wp[k] = INTERLEAVED ? w[k ^ 1] : __shfl(w[kSwap ? k ^ 4 : k], partner[k / 4 * kOwn]);
#pragma unroll
            for (int k = 0; k < 8; ++k) c[k] *= w[k], sn[k] *= wp[k];
        }

        for (int hb = h0; hb < h1; hb += kAhead * at_once) {
            Piece<T> xr[kAhead], yr[kAhead];
            bool on[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int h = hb + u * at_once + head;
                on[u] = h < h1 && in_row && has_token;
                xr[u].clear();
                yr[u].clear();
                if (on[u]) {
                    xr[u].template load<STREAM>(px + h * side.x.h);
                    if (BACK) yr[u].template load<STREAM>(py + h * side.y.h);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (u > 0 && hb + u * at_once >= h1) break;  // the same for the whole wave
                float x[8], y[8], o[8];
                xr[u].floats(x);
                float sq = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) sq += x[k] * x[k];
                float r = rsqrtf(group_sum<G>(sq) * (1.0f / (float)D) + a.eps);
                if (lost) r = __builtin_nanf("");
                if (BACK) {
                    yr[u].floats(y);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = x[k];
                }
                if (INTERLEAVED) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) o[k] = y[k ^ 1];
                } else {
                    (BACK ? yr[u] : xr[u]).template partners<kSwap>(partner).floats(o);
                }
                // backward the transpose: the sine's other sign
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    y[k] = y[k] * c[k] + (turned ? (BACK ? -sn[k] : sn[k]) * o[k] : 0.0f);
                if (!BACK) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] *= r;
                } else {
                    float dot = 0.0f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        x[k] *= r;
                        sums[k] += on[u] ? y[k] * x[k] : 0.0f;
                        y[k] *= w[k];
                        dot += y[k] * x[k];
                    }
                    dot = group_sum<G>(dot) * (1.0f / (float)D);
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = r * (y[k] - x[k] * dot);
                }
                if (on[u]) Piece<T>::template store<STREAM>(po + (hb + u * at_once + head) * side.out.h, y);
            }
        }
    }
    if (BACK && side.partials) {
        // the block's lanes of each piece, added in a fixed order
        __shared__ float part[4][G * 8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float v = sums[k];
#pragma unroll
            for (int d = G; d < 64; d <<= 1) v += __shfl_xor(v, d);
            if (lane < G) part[threadIdx.x >> 6][i + k] = v;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < D; e += 256)
            side.partials[(int64_t)block * D + e] = part[0][e] + part[1][e] + (part[2][e] + part[3][e]);
    }
}

// dw: the blocks' partial sums, added in a fixed order: four columns to a block,
// its 1,024 threads a partial row each in turn, 16 bytes at a time (2,047 rows of 128:
// 5.9 us; 256 threads, element by element: 9.5); the second grid dimension the side.
constexpr int kColumns = 4, kDweightThreads = 1024;
__global__ __launch_bounds__(kDweightThreads) void k_qk_dweight(QkArgs a) {
    __shared__ float part[kDweightThreads / 64][kColumns];
    const QkSide &side = a.side[blockIdx.y];
    if (!side.dweight) return;
    const int i = blockIdx.x * kColumns, rows = a.blocks[blockIdx.y];
    const float *from = side.partials + i;
    float s[kColumns] = {};
    if (a.dim % kColumns == 0) {
#pragma unroll 2
        for (int b = threadIdx.x; b < rows; b += kDweightThreads) {
            const f32x4 v = *(const f32x4 *)(from + (int64_t)b * a.dim);
#pragma unroll
            for (int c = 0; c < kColumns; ++c) s[c] += v[c];
        }
    } else {
        for (int b = threadIdx.x; b < rows; b += kDweightThreads)
#pragma unroll
            for (int c = 0; c < kColumns; ++c) s[c] += i + c < a.dim ? from[(int64_t)b * a.dim + c] : 0.0f;
    }
#pragma unroll
    for (int c = 0; c < kColumns; ++c) {
        const float v = wave_sum(s[c]);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][c] = v;
    }
    __syncthreads();
    if (threadIdx.x < kColumns && i + (int)threadIdx.x < a.dim) {
        const int c = threadIdx.x;
        float v = 0.0f;
        for (int w = 0; w < kDweightThreads / 64; ++w) v += part[w][c];
        if (a.weight_bf16)
            store1((uint16_t *)side.dweight + i + c, v);
        else
            ((float *)side.dweight)[i + c] = v;
    }
}

template <typename T, bool BACK>
void launch_rows(const QkArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((k_qk_rows<T, BACK>), dim3(a.blocks[0] + a.blocks[1]), dim3(64 * kRowWaves), 0, s, a);
}

template <typename T, int G, bool BACK>
void launch_tokens(const QkArgs &a, hipStream_t s) {
    const dim3 grid(a.blocks[0] + a.blocks[1]);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
    const bool odd = a.rotary / 8 % 2 != 0;
    if (a.stream)
        a.interleaved ? go(k_qk_tokens<T, G, kNeighbours, BACK, true>)
        : odd         ? go(k_qk_tokens<T, G, kHalvesOdd, BACK, true>)
                      : go(k_qk_tokens<T, G, kHalves, BACK, true>);
    else
        a.interleaved ? go(k_qk_tokens<T, G, kNeighbours, BACK, false>)
        : odd         ? go(k_qk_tokens<T, G, kHalvesOdd, BACK, false>)
                      : go(k_qk_tokens<T, G, kHalves, BACK, false>);
}

// Lanes to a row of the tokens kernel: the power of two that holds the row.
int lanes_of(int dim) {
    int g = 4;
    while (g * 8 < dim) g *= 2;
    return g;
}

// Whether the tokens kernel takes the call: whole pieces, partners whole half
// pieces apart, and every row (and the tables') at a 16-byte boundary.
bool in_pieces(const QkArgs &a, bool bf16, bool backward) {
    const int64_t per16 = bf16 ? 8 : 4;
    auto aligned = [&](const Heads &h) {
        return (uintptr_t)h.data % 16 == 0 && h.b % per16 == 0 && h.s % per16 == 0 && h.h % per16 == 0;
    };
    if (a.dim % 8 != 0 || a.dim > 512 || a.rotary % 8 != 0) return false;
    if (a.rotary > 0 && ((uintptr_t)a.cos % 16 != 0 || (uintptr_t)a.sin % 16 != 0)) return false;
    for (int k = 0; k < 2; ++k) {
        const QkSide &d = a.side[k];
        if (a.rows_total[k] > 0 && !(aligned(d.x) && aligned(d.out) && (!backward || aligned(d.y)))) return false;
    }
    return true;
}

// How a call is split, in `a`: the blocks of each side and, for the tokens
// kernel, the runs of heads that a wave takes.  Forward 8,192 blocks of four waves,
// each walking its share (32,768 tokens of 48 heads of 128, BF16: 157 us; 4,096
// blocks 176, 16,384 169), four wavefuls of rows loaded ahead (two: 159 us with
// this split).  Backward 2,048, as each leaves a row of partial sums and holds
// more registers (256 us; 1,024: 279; half as many again: 251, but 40 instead of 34 us on
// 4,101 tokens of 16 heads).  Non-temporal loads and stores from 256 MB on, the
// last-level cache's size: 157 against 163 us and 256 against 274; below it they
// cost (34 against 32 us).
void split(QkArgs &a, bool bf16, bool backward) {
    const int64_t tokens = (int64_t)a.batch * a.tokens, both = a.rows_total[0] + a.rows_total[1];
    const int64_t most = backward ? 2048 : 8192;
    const bool pieces = in_pieces(a, bf16, backward);
    a.stream = both * a.dim * (bf16 ? 2 : 4) * (backward ? 3 : 2) > (int64_t)256 << 20;
    // runs as long as leave every wave of the grid one, in whole wavefuls of rows
    const int fit = pieces ? 64 / lanes_of(a.dim) : 1;
    const int64_t run = (both + 4 * most - 1) / (4 * most);
    a.chunk_heads = (int)std::min<int64_t>((run + fit - 1) / fit * fit, SDP_QK_MAX_HEADS);
    for (int k = 0; k < 2; ++k) {
        a.heads_log[k] = 0;
        while ((1 << a.heads_log[k]) < std::min(fit, a.side[k].heads)) ++a.heads_log[k];
        const int tokens_at_once = fit >> a.heads_log[k];
        a.chunks[k] = (a.side[k].heads + a.chunk_heads - 1) / a.chunk_heads;
        const int64_t items = pieces ? (tokens + tokens_at_once - 1) / tokens_at_once * a.chunks[k] : a.rows_total[k];
        const int64_t share = a.rows_total[k] ? std::max<int64_t>(1, most * a.rows_total[k] / both) : 0;
        a.blocks[k] = (int)std::min<int64_t>((items + 3) / 4, share);
    }
}

template <typename T, bool BACK>
void launch_any(const QkArgs &a, hipStream_t s) {
    if (!in_pieces(a, sizeof(T) == 2, BACK)) return launch_rows<T, BACK>(a, s);
    switch (lanes_of(a.dim)) {
        case 4: return launch_tokens<T, 4, BACK>(a, s);
        case 8: return launch_tokens<T, 8, BACK>(a, s);
        case 16: return launch_tokens<T, 16, BACK>(a, s);
        case 32: return launch_tokens<T, 32, BACK>(a, s);
        default: return launch_tokens<T, 64, BACK>(a, s);
    }
}

}  // namespace

void qk_split(QkArgs &a, bool bf16, bool backward) {
    a.blocks[0] = a.blocks[1] = a.chunks[0] = a.chunks[1] = 0;
    a.chunk_heads = 1;
    if (a.rows_total[0] + a.rows_total[1] > 0) split(a, bf16, backward);
}

hipError_t launch_qk(const QkArgs &a, bool bf16, bool backward, hipStream_t s) {
    if (a.blocks[0] + a.blocks[1] > 0) {
        if (bf16)
            backward ? launch_any<uint16_t, true>(a, s) : launch_any<uint16_t, false>(a, s);
        else
            backward ? launch_any<float, true>(a, s) : launch_any<float, false>(a, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (backward && (a.side[0].dweight || a.side[1].dweight)) {
        hipLaunchKernelGGL(k_qk_dweight, dim3((a.dim + kColumns - 1) / kColumns, 2), dim3(kDweightThreads), 0, s, a);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace sdpops
