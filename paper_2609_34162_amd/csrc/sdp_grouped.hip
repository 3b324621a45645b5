// gfx950 kernels of sdp_grouped_matmul and its backward.
//
// Three products over the groups' rows t:
//   forward  y[t, n]  = sum_k x[t, k] w[e][n, k]
//   dx       dx[t, k] = sum_n dy[t, n] w[e][n, k]
//   dw       dw[e][n, k] = sum_t dy[t, n] x[t, k]
// each C[m, n] = sum_c A(m, c) B(n, c) with one of the outer dimensions
// (forward, dx) or the contraction (dw) ragged.  The groups' ends lie in device
// memory, so a block finds its tile there itself and the grid is an upper bound.
#include "sdp_ops_device.h"
#include "sdp_ops_internal.h"

namespace sdpops {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

enum Mode { kForward = 0, kDx = 1, kDw = 2 };

struct RowTile {
    int group;      // groups: rows of no group; -1: nothing to do
    int64_t first, end;
    int64_t tiles;  // row tiles in all
};

__device__ __forceinline__ int64_t shfl64(int64_t v, int lane) {
    const int lo = __shfl((int)(uint32_t)v, lane), hi = __shfl((int)(v >> 32), lane);
    return (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
}
__device__ __forceinline__ int64_t shfl_up64(int64_t v, int d) {
    const int lo = __shfl_up((int)(uint32_t)v, d), hi = __shfl_up((int)(v >> 32), d);
    return (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
}

// The end of group e as the groups use it: the largest of the values up to e,
// within 0..rows (group `groups`, the rows of no group, ends at rows).
// A wave takes 64 groups at a time; `run` is the largest value before them.
__device__ __forceinline__ int64_t group_end(const GroupedArgs &a, int e, int64_t run) {
    int64_t end = e < a.groups ? load_int(a.ends, e, a.ends64) : e == a.groups ? a.rows : 0;
    end = end < 0 ? 0 : end > a.rows ? a.rows : end;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t before = shfl_up64(end, d);
        if ((int)(threadIdx.x & 63) >= d && before > end) end = before;
    }
    return end > run ? end : run;
}

// Row tile `want` of the tiles of BM rows that cover each group (and the rows
// of no group) from its first row: every wave of the block finds it by a scan
// over the groups' ends.  want < 0: only the number of tiles.
template <int BM>
__device__ RowTile find_row_tile(const GroupedArgs &a, int64_t want) {
    const int lane = threadIdx.x & 63;
    RowTile found{-1, 0, 0, 0};
    int64_t run = 0, tiles = 0;
    for (int base = 0; base <= a.groups; base += 64) {
        const int e = base + lane;
        const int64_t end = group_end(a, e, run);
        int64_t start = shfl_up64(end, 1);
        if (lane == 0) start = run;
        const int64_t mine = e <= a.groups ? (end - start + BM - 1) / BM : 0;
        int64_t upto = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t before = shfl_up64(upto, d);
            if (lane >= d) upto += before;
        }
        const int64_t from = tiles + upto - mine;
        const uint64_t hit = __ballot(want >= from && want < tiles + upto);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            found.group = base + l;
            found.first = shfl64(start, l) + (want - shfl64(from, l)) * BM;
            found.end = shfl64(end, l);
        }
        run = shfl64(end, 63);
        tiles += shfl64(upto, 63);
    }
    found.tiles = tiles;
    return found;
}

// Rows of group e.
__device__ void group_rows(const GroupedArgs &a, int want, int64_t *start_out, int64_t *end_out) {
    const int lane = threadIdx.x & 63;
    int64_t run = 0;
    for (int base = 0;; base += 64) {
        const int64_t end = group_end(a, base + lane, run);
        int64_t start = shfl_up64(end, 1);
        if (lane == 0) start = run;
        if (want < base + 64) {
            *start_out = shfl64(start, want - base);
            *end_out = shfl64(end, want - base);
            return;
        }
        run = shfl64(end, 63);
    }
}

// ---- any size, stride and alignment ----------------------------------------

// A 64 x 64 tile of C, four waves of 32 x 32, 32 of the contraction at a time
// through LDS, loaded element by element.
constexpr int kAnyTile = 64, kAnyDepth = 32, kAnyPitch = kAnyDepth + 8;

// 64 x 32 elements (i, c) of base[i * si + c * sc] into LDS, zero outside.
__device__ void load_any(const uint16_t *base, int64_t si, int64_t sc, int64_t n_i, int64_t n_c,
                         uint16_t (*lds)[kAnyPitch]) {
    for (int k = threadIdx.x; k < kAnyTile * kAnyDepth; k += 256) {
        // neighbouring threads along the contiguous dimension
        const int i = sc == 1 ? k / kAnyDepth : k % kAnyTile, c = sc == 1 ? k % kAnyDepth : k / kAnyTile;
        lds[i][c] = i < n_i && c < n_c ? base[i * si + c * sc] : (uint16_t)0;
    }
}

template <Mode MODE>
__global__ __launch_bounds__(256) void k_grouped_any(GroupedArgs a) {
    __shared__ uint16_t la[kAnyTile][kAnyPitch], lb[kAnyTile][kAnyPitch];
    int64_t m0, m1, n0, n1, depth;
    const uint16_t *A = nullptr, *B = nullptr;
    int64_t sai, sac, sbi, sbc;
    char *C;
    int64_t c_stride;
    bool f32 = a.out_f32 != 0;
    bool empty = false;
    const int64_t n_in = a.n_in, n_out = a.n_out;
    if (MODE == kDw) {
        const int64_t tm = (n_out + kAnyTile - 1) / kAnyTile, tn = (n_in + kAnyTile - 1) / kAnyTile;
        const int64_t id = blockIdx.x;
        const int e = (int)(id / (tm * tn));
        m0 = (id / tn) % tm * kAnyTile, m1 = n_out;
        n0 = id % tn * kAnyTile, n1 = n_in;
        int64_t t0, t1;
        group_rows(a, e, &t0, &t1);
        depth = t1 - t0;
        A = a.dy + t0 * a.y_stride + m0, sai = 1, sac = a.y_stride;
        B = a.x + t0 * a.x_stride + n0, sbi = 1, sbc = a.x_stride;
        c_stride = n_in;
        C = (char *)a.dw + (f32 ? 4 : 2) * ((int64_t)e * n_out * n_in);
    } else {
        const int64_t cols = MODE == kForward ? n_out : n_in;
        const int64_t tn = (cols + kAnyTile - 1) / kAnyTile;
        const RowTile t = find_row_tile<kAnyTile>(a, (int64_t)blockIdx.x / tn);
        if (t.group < 0) return;
        empty = t.group == a.groups;
        const uint16_t *w = a.w + (empty ? 0 : (int64_t)t.group * n_out * n_in);
        m0 = t.first, m1 = t.end;
        n0 = (int64_t)blockIdx.x % tn * kAnyTile, n1 = cols;
        depth = empty ? 0 : MODE == kForward ? n_in : n_out;
        if (MODE == kForward) {
            A = a.x + m0 * a.x_stride, sai = a.x_stride, sac = 1;
            B = w + n0 * n_in, sbi = n_in, sbc = 1;
            C = (char *)a.y, c_stride = a.y_stride;
        } else {
            A = a.dy + m0 * a.y_stride, sai = a.y_stride, sac = 1;
            B = w + n0, sbi = 1, sbc = n_in;
            C = (char *)a.dx, c_stride = a.dx_stride;
            f32 = false;
        }
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32, sub = lane & 15, quad = lane >> 4;
    f32x4 acc[2][2] = {};
    for (int64_t c0 = 0; c0 < depth; c0 += kAnyDepth) {
        load_any(A + c0 * sac, sai, sac, m1 - m0, depth - c0, la);
        load_any(B + c0 * sbc, sbi, sbc, n1 - n0, depth - c0, lb);
        __syncthreads();
        bf16x8 fa[2], fb[2];
        for (int i = 0; i < 2; ++i) {
            fa[i] = *(const bf16x8 *)&la[wm + 16 * i + sub][8 * quad];
            fb[i] = *(const bf16x8 *)&lb[wn + 16 * i + sub][8 * quad];
        }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
        __syncthreads();
    }
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            for (int r = 0; r < 4; ++r) {
                const int64_t m = m0 + wm + 16 * i + 4 * quad + r, n = n0 + wn + 16 * j + sub;
                if (m >= m1 || n >= n1) continue;
                if (f32)
                    ((float *)C)[m * c_stride + n] = acc[i][j][r];
                else
                    store1((uint16_t *)C + m * c_stride + n, acc[i][j][r]);
            }
}

int64_t ceil_div(int64_t a, int64_t b) { return a / b + (a % b != 0); }

// Most row tiles of bm rows that the groups and the rows of no group can make:
// each of them, if it has rows, adds at most one part tile.
int64_t row_tiles(const GroupedArgs &a, int64_t bm) {
    const int64_t parts = a.groups + 1 < a.rows ? a.groups + 1 : a.rows;
    const int64_t most = a.rows / bm + parts;
    return most < a.rows ? most : a.rows;
}

constexpr int64_t kMaxBlocks = 0xffffffffll / 256;

int64_t blocks_any(const GroupedArgs &a, Mode mode) {
    if (mode == kDw) return (int64_t)a.groups * ceil_div(a.n_out, kAnyTile) * ceil_div(a.n_in, kAnyTile);
    return row_tiles(a, kAnyTile) * ceil_div(mode == kForward ? a.n_out : a.n_in, kAnyTile);
}

template <Mode MODE>
hipError_t launch_any(const GroupedArgs &a, hipStream_t s) {
    const int64_t blocks = blocks_any(a, MODE);
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL((k_grouped_any<MODE>), dim3((uint32_t)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

bool grouped_fits(const GroupedArgs &a, bool forward, bool dx, bool dw) {
    return (!forward || blocks_any(a, kForward) <= kMaxBlocks) && (!dx || blocks_any(a, kDx) <= kMaxBlocks) &&
           (!dw || blocks_any(a, kDw) <= kMaxBlocks);
}

hipError_t launch_grouped_forward(const GroupedArgs &a, hipStream_t s) { return launch_any<kForward>(a, s); }
hipError_t launch_grouped_dx(const GroupedArgs &a, hipStream_t s) { return launch_any<kDx>(a, s); }
hipError_t launch_grouped_dw(const GroupedArgs &a, hipStream_t s) { return launch_any<kDw>(a, s); }

}  // namespace sdpops
