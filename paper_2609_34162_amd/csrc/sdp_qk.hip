// gfx950 kernels of sdp_qk_norm_rope and its backward.
//
// For a head's row x of D elements, r = 1 / sqrt(mean(x^2) + eps):
//   n = x r w;  each rotated pair (a, b) of n becomes (a c - b s, b c + a s)
// and backward, with dn the rotation's transpose of dy and u = dn w:
//   dx = r (u - x r mean(u x r)),  dw = sum over rows of dn x r
// Every element is read once and written once: HBM bounds both directions.
#include "sdp_ops_device.h"
#include "sdp_ops_internal.h"

namespace sdpops {
namespace {

constexpr int kRowWaves = 4;

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

// dw: the blocks' partial sums, added in a fixed order: 64 threads to a
// column, 16 columns to a block, the second grid dimension the side.
__global__ __launch_bounds__(1024) void k_qk_dweight(QkArgs a) {
    __shared__ float part[64][17];
    const QkSide &side = a.side[blockIdx.y];
    if (!side.dweight) return;
    const int c = threadIdx.x & 15, t = threadIdx.x >> 4;
    const int i = blockIdx.x * 16 + c;
    float s = 0.0f;
    if (i < a.dim)
        for (int b = t; b < a.blocks[blockIdx.y]; b += 64) s += side.partials[(int64_t)b * a.dim + i];
    part[t][c] = s;
    __syncthreads();
    for (int half = 32; half > 0; half >>= 1) {
        if (t < half) part[t][c] += part[t + half][c];
        __syncthreads();
    }
    if (t == 0 && i < a.dim) {
        if (a.weight_bf16)
            store1((uint16_t *)side.dweight + i, part[0][c]);
        else
            ((float *)side.dweight)[i] = part[0][c];
    }
}

template <typename T, bool BACK>
void launch_rows(const QkArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((k_qk_rows<T, BACK>), dim3(a.blocks[0] + a.blocks[1]), dim3(64 * kRowWaves), 0, s, a);
}

int64_t blocks_for(int64_t rows, int64_t most) {
    const int64_t n = (rows + kRowWaves - 1) / kRowWaves;
    return n < most ? n : most;
}

}  // namespace

int qk_backward_blocks(const QkArgs &a, int side) { return (int)blocks_for(a.rows_total[side], 1024); }

hipError_t launch_qk(const QkArgs &args, bool bf16, bool backward, hipStream_t s) {
    QkArgs a = args;
    for (int k = 0; k < 2; ++k)
        a.blocks[k] = backward ? qk_backward_blocks(a, k) : (int)blocks_for(a.rows_total[k], 1 << 20);
    if (a.blocks[0] + a.blocks[1] > 0) {
        if (bf16)
            backward ? launch_rows<uint16_t, true>(a, s) : launch_rows<uint16_t, false>(a, s);
        else
            backward ? launch_rows<float, true>(a, s) : launch_rows<float, false>(a, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (backward && (a.side[0].dweight || a.side[1].dweight) && a.dim > 0) {
        hipLaunchKernelGGL(k_qk_dweight, dim3((a.dim + 15) / 16, 2), dim3(1024), 0, s, a);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace sdpops
