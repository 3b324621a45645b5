// gfx950 kernels of sdp_grouped_matmul and its backward.
//
// Three products over the groups' rows t:
//   forward  y[t, n]  = sum_k x[t, k] w[e][n, k]
//   dx       dx[t, k] = sum_n dy[t, n] w[e][n, k]
//   dw       dw[e][n, k] = sum_t dy[t, n] x[t, k]
// each C[m, n] = sum_c A(m, c) B(n, c) with one of the outer dimensions
// (forward, dx) or the contraction (dw) ragged.  The groups' ends lie in device
// memory, so a block finds its tile there itself and the grid is an upper bound.
#include <type_traits>

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

__device__ __forceinline__ int64_t uniform64(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
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
    // the same in every lane: keep them in scalar registers
    found.group = __builtin_amdgcn_readfirstlane(found.group);
    found.first = uniform64(found.first);
    found.end = uniform64(found.end);
    found.tiles = uniform64(tiles);
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
            *start_out = uniform64(shfl64(start, want - base));
            *end_out = uniform64(shfl64(end, want - base));
            return;
        }
        run = shfl64(end, 63);
    }
}

// Blocks go to the 8 XCDs in turn; neighbouring tiles share operands in an
// XCD's L2, so each XCD gets a run of tiles: the tile of block `b` of `n`.
__device__ __forceinline__ int64_t xcd_order(int64_t b, int64_t n) {
    const int64_t x = b & 7, each = n >> 3, more = n & 7;
    return x * each + (x < more ? x : more) + (b >> 3);
}

// Tile `id` of rows x columns tiles, in panels of 8 columns: the 32 blocks that
// an XCD runs at once (one to a compute unit) are then 4 rows by 8 columns, and
// load 12 tiles of operands from beyond the XCD's L2 instead of up to 33.
__device__ __forceinline__ void panel_order(int64_t id, int64_t rows, int columns, int64_t *row, int *column) {
    const int64_t panel = id / (8 * rows), in_panel = id - panel * 8 * rows;
    const int first = (int)panel * 8, width = columns - first < 8 ? columns - first : 8;
    *row = in_panel / width;
    *column = first + (int)(in_panel - *row * width);
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

// ---- rows of 16-byte pieces ---------------------------------------------------

// Where every row starts at a 16-byte boundary and holds whole pieces of 8
// elements, a block computes a BM x BN tile of C from tiles of 32 of the
// contraction in LDS, written there by the load instructions themselves.
//
// A tile whose rows run along the contraction ("by row": x and w forward, dy
// for dx) lies in LDS as [row][4 pieces], piece c of row r at place
// c ^ (r / 2 & 3): 8 neighbouring rows read at one c then fall on different
// banks.  One whose rows lie across it ("by depth": w for dx, dy and x for dw)
// lies as [depth][BM or BN elements], in segments of 16 elements, segment s of
// depth d at place s ^ f(d), f = d & 3 | (d / 8 & 1) * 4, and is read by the
// transposing LDS load: 16 lanes read 4 depths x 16 elements and each gets the 4
// depths of one element.
//
// NB buffers, step s in buffer s mod NB.  In step s the products of s run from
// registers, the operands of s + 1 are read from LDS, and loads of the steps up
// to s + NB are in flight, the last of them into the buffer that s has left: a
// load has NB - 1 steps to arrive.  One barrier a step.
constexpr int kDepth = 32;
constexpr uint32_t kRange = 0x7ffffff0u;  // bytes that a load's offset may reach

typedef __attribute__((address_space(3))) void *LdsPtr;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

// The wave of this thread in its block, in a scalar register.
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// How a segment's place depends on its depth (by depth; T / 16 segments a depth).
template <int T>
__device__ __forceinline__ int turn(int d) {
    const int f = (d & 3) | ((d >> 3) & 1) << 2;
    return T >= 128 ? f : f & (T / 16 - 1);
}

// One operand: T elements of its outer dimension (rows of C, or columns) by
// kDepth of the contraction.  BY_DEPTH: see above.  WAVES: of the block.
template <int T, bool BY_DEPTH, int WAVES>
struct Operand {
    static constexpr int kLoads = T * kDepth * 2 / 1024;  // wave-wide load instructions a step
    static constexpr int kEach = (kLoads + WAVES - 1) / WAVES;
    static constexpr int kBytes = T * kDepth * 2;
    static constexpr int kPieces = T / 8;  // by depth: pieces of a depth
    const char *base;      // element (first outer, depth 0) of the next step to load
    uint32_t off[kEach];   // bytes from it of this lane's piece of each load
    int64_t step;          // bytes to the step after

    // outer: how many outer elements exist from the first on (at least 1)
    __device__ __forceinline__ void init(const uint16_t *first, int64_t stride, int64_t outer) {
        const int lane = threadIdx.x & 63, wave = wave_id();
        base = (const char *)first;
        step = BY_DEPTH ? kDepth * stride * 2 : kDepth * 2;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int idx = j * WAVES + wave;
            if (BY_DEPTH) {
                const int d = (idx * 64 + lane) / kPieces, place = lane % kPieces;
                int piece = ((place >> 1) ^ turn<T>(d)) * 2 + (place & 1);
                // past the last element: any piece that exists, its results are not stored
                if (piece * 8 >= outer) piece = (int)(outer - 1) / 8;
                off[j] = (uint32_t)d * (uint32_t)(stride * 2) + piece * 16;
            } else {
                const int r = idx * 16 + lane / 4;
                const int piece = (lane & 3) ^ (lane >> 3 & 3);
                off[j] = (uint32_t)(r < outer ? r : (int)outer - 1) * (uint32_t)(stride * 2) + piece * 16;
            }
        }
    }

    // Load instructions of a wave in one step, USED outer elements being read (by
    // row, the others are not loaded).
    template <int USED>
    static constexpr int loads() {
        return BY_DEPTH || USED >= T ? kEach : (USED + WAVES * 16 - 1) / (WAVES * 16);
    }

    // Loads the next step into lds, `left` of the contraction being left; what
    // lies past it becomes 0: those lanes' offsets lie past the range that the
    // buffer descriptor allows, and such a load brings zeros.
    template <int USED>
    __device__ __forceinline__ void load(char *lds, int64_t left) {
        const int lane = threadIdx.x & 63, wave = wave_id();
        const __amdgpu_buffer_rsrc_t buffer =
            __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, kRange, 0x00020000);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int idx = j * WAVES + wave;
            if (!BY_DEPTH && j * WAVES * 16 >= USED) break;
            if (kLoads % WAVES != 0 && idx >= kLoads) break;
            uint32_t o = off[j];
            if (left < kDepth) {
                const int at = BY_DEPTH ? (idx * 64 + lane) / kPieces : ((lane & 3) ^ (lane >> 3 & 3)) * 8;
                o = at < left ? o : kRange;
            }
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (LdsPtr)(lds + idx * 1024), 16, o, 0, 0, 0);
        }
        // past the end the base stays: the loads bring zeros
        base += left > kDepth ? step : 0;
    }
};

// The 16 x 32 fragment of outer elements first + 16 STEP i + lane % 16 and
// depths 8 (lane / 16) + 0..7; the bits of first / 16 and of STEP i do not meet.
template <int T, bool BY_DEPTH, int STEP>
struct Reader {
    uint32_t at;
    __device__ __forceinline__ void init(int first) {
        const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
        if (BY_DEPTH) {
            const int d = 8 * g + (l >> 2);
            at = d * T * 2 + ((first / 16) ^ turn<T>(d)) * 32 + (l & 3) * 8;
        } else {
            const int r = first + l;
            at = r * 64 + ((g ^ (r >> 1 & 3)) * 16);
        }
    }
    __device__ __forceinline__ bf16x8 read(const char *lds, int i) const {
        if constexpr (BY_DEPTH) {
            typedef __attribute__((address_space(3))) s16x4 *P;
            // depths 4 apart turn alike, so one address serves both halves of the
            // fragment; worked out anew each time, as holding one for each i would
            // take registers that the tile needs
            uint32_t from = at;
            asm("" : "+v"(from));
            const char *p = lds + (from ^ (uint32_t)(i * STEP * 32));
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 4 * T * 2));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *(const bf16x8 *)(lds + at + i * STEP * 16 * 64);
        }
    }
};

// Waits until at most `loads` of this wave's loads are in flight and its LDS
// reads are done, then for the block's other waves.
template <int LOADS>
__device__ __forceinline__ void wait_and_meet() {
    static_assert(LOADS < 64, "the counter has 6 bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LOADS & 15) | 7 << 4 | (LOADS >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <Mode MODE, int BM, int BN, int WM, int WN, int NB>
__global__ __launch_bounds__(64 * WM * WN) void k_grouped(GroupedArgs a) {
    constexpr int kWaves = WM * WN, MT = BM / WM / 16, NT = BN / WN / 16;
    constexpr bool kADepth = MODE == kDw, kBDepth = MODE != kForward;
    using OpA = Operand<BM, kADepth, kWaves>;
    using OpB = Operand<BN, kBDepth, kWaves>;
    // an array for each buffer (A's tile, then B's), so that the compiler sees
    // which one a load writes and does not wait for it before it reads another
    constexpr int kBuffer = OpA::kBytes + OpB::kBytes;
    __shared__ __attribute__((aligned(1024))) char lds0[kBuffer], lds1[kBuffer], lds2[kBuffer];
    __shared__ __attribute__((aligned(1024))) char lds3[kBuffer], lds4[kBuffer], lds5[kBuffer];

    int64_t m0, m1, n0, n1, depth, c_stride;
    const uint16_t *A, *B;
    int64_t sa, sb;
    char *C;
    bool f32 = a.out_f32 != 0;
    const int64_t n_in = a.n_in, n_out = a.n_out;
    if constexpr (MODE == kDw) {
        const int tm = (int)((n_out + BM - 1) / BM), tn = (int)((n_in + BN - 1) / BN);
        const int64_t id = xcd_order(blockIdx.x, gridDim.x);
        const int e = (int)(id / (tm * tn)), in_group = (int)(id - (int64_t)e * (tm * tn));
        int64_t row;
        int column;
        panel_order(in_group, tm, tn, &row, &column);
        m0 = row * BM, m1 = n_out;
        n0 = (int64_t)column * BN, n1 = n_in;
        int64_t t0, t1;
        group_rows(a, e, &t0, &t1);
        depth = t1 - t0;
        A = a.dy + t0 * a.y_stride + m0, sa = a.y_stride;
        B = a.x + t0 * a.x_stride + n0, sb = a.x_stride;
        C = (char *)a.dw + (f32 ? 4 : 2) * ((int64_t)e * n_out * n_in), c_stride = n_in;
    } else {
        const int64_t cols = MODE == kForward ? n_out : n_in;
        const int tn = (int)((cols + BN - 1) / BN);
        const int64_t tm = find_row_tile<BM>(a, -1).tiles;
        if (blockIdx.x >= tm * tn) return;
        int64_t row;
        int column;
        panel_order(xcd_order(blockIdx.x, tm * tn), tm, tn, &row, &column);
        const RowTile t = find_row_tile<BM>(a, row);
        const bool empty = t.group == a.groups;
        const uint16_t *w = a.w + (empty ? 0 : (int64_t)t.group * n_out * n_in);
        m0 = t.first, m1 = t.end;
        n0 = (int64_t)column * BN, n1 = cols;
        depth = empty ? 0 : MODE == kForward ? n_in : n_out;
        if constexpr (MODE == kForward) {
            A = a.x + m0 * a.x_stride, sa = a.x_stride;
            B = w + n0 * n_in, sb = n_in;
            C = (char *)a.y, c_stride = a.y_stride;
        } else {
            A = a.dy + m0 * a.y_stride, sa = a.y_stride;
            B = w + n0, sb = n_in;
            C = (char *)a.dx, c_stride = a.dx_stride;
            f32 = false;
        }
    }

    // the waves' 16-row fragments alternate, so that a tile with few rows is
    // shared by all of them; their columns lie together
    const int wave = wave_id(), lane = threadIdx.x & 63;
    const int wm = wave / WN * 16, wn = wave % WN * (BN / WN);
    f32x4 acc[MT][NT] = {};
    const int steps = (int)((depth + kDepth - 1) / kDepth);
    // the whole contraction, over the first MU of a wave's row fragments
    auto contract = [&](auto used) __attribute__((always_inline)) {
        constexpr int MU = decltype(used)::value;
        constexpr int kLoads = OpA::template loads<MU * WM * 16>() + OpB::template loads<BN>();
        OpA oa;
        OpB ob;
        oa.init(A, sa, m1 - m0);
        ob.init(B, sb, n1 - n0);
        Reader<BM, kADepth, WM> ra;
        Reader<BN, kBDepth, 1> rb;
        ra.init(wm);
        rb.init(wn);
        bf16x8 fa[2][MU], fb[2][NT];
        auto read = [&](const char *lds, int f) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < NT; ++j) fb[f][j] = rb.read(lds + OpA::kBytes, j);
#pragma unroll
            for (int i = 0; i < MU; ++i) fa[f][i] = ra.read(lds, i);
        };
        int left = (int)depth;  // of the contraction, to load
        auto load = [&](char *lds) __attribute__((always_inline)) {
            oa.template load<MU * WM * 16>(lds, left);
            ob.template load<BN>(lds + OpA::kBytes, left);
            left = left > kDepth ? left - kDepth : 0;
        };
        // One step from registers f; `lds`: its buffer, `next`: the next step's.
        // Past the end of the contraction loads bring zeros, so that the number
        // in flight stays the same.
        auto step = [&](int f, char *lds, const char *next) __attribute__((always_inline)) {
            wait_and_meet<(NB - 2) * kLoads>();
            load(lds);
            read(next, f ^ 1);
#pragma unroll
            for (int i = 0; i < MU; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[f][j], fa[f][i], acc[i][j], 0, 0, 0);
            // one LDS read in front of each product until all are under way
            constexpr int kReads = MU * (kADepth ? 2 : 1) + NT * (kBDepth ? 2 : 1);
#pragma unroll
            for (int r = 0; r < (kReads < MU * NT ? kReads : MU * NT); ++r) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        char *const bufs[6] = {lds0, lds1, lds2, lds3, lds4, lds5};
#pragma unroll
        for (int k = 0; k < NB; ++k) load(bufs[k]);
        wait_and_meet<(NB - 1) * kLoads>();
        read(lds0, 0);
        constexpr int kUnroll = NB % 2 ? 2 * NB : NB;
        for (int k = 0; k < steps; k += kUnroll) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (u > 0 && k + u >= steps) break;
                step(u & 1, bufs[u % NB], bufs[(u + 1) % NB]);
            }
        }
        // no load may land after the block has given its LDS back
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(15 << 8 | 7 << 4);
    };
    if (steps > 0) {
        const int64_t rows = m1 - m0;
        if (MT >= 4 && rows <= MT / 4 * WM * 16)
            contract(std::integral_constant<int, (MT >= 4 ? MT / 4 : 1)>{});
        else if (MT >= 2 && rows <= MT / 2 * WM * 16)
            contract(std::integral_constant<int, (MT >= 2 ? MT / 2 : 1)>{});
        else
            contract(std::integral_constant<int, MT>{});
    }
    // a lane holds 4 neighbouring columns of row lane % 16 of each 16 x 16 tile
    auto store = [&](auto put) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = m0 + wm + 16 * WM * i + (lane & 15);
            if (m >= m1) continue;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int64_t n = n0 + wn + 16 * j + 4 * (lane >> 4);
                if (n < n1) put(m * c_stride + n, acc[i][j]);
            }
        }
    };
    if (f32)
        store([&](int64_t at, f32x4 v) { *(f32x4 *)((float *)C + at) = v; });
    else
        store([&](int64_t at, f32x4 v) {
            *(uint2 *)((uint16_t *)C + at) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
        });
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

// Whether the tiled kernels can take the call: whole 16-byte pieces in every
// row, rows and results at 16-byte boundaries, and a tile's offsets in 32 bits.
bool pieces(const void *p, int64_t stride, int64_t cols) {
    return (uintptr_t)p % 16 == 0 && stride % 8 == 0 && cols % 8 == 0 && stride < ((int64_t)1 << 22);
}
bool tiled(const GroupedArgs &a, Mode mode) {
    const bool w = mode == kDw || pieces(a.w, a.n_in, a.n_in);
    const bool x = mode == kDx || pieces(a.x, a.x_stride, a.n_in);
    const bool dy = mode == kForward || pieces(a.dy, a.y_stride, a.n_out);
    const void *c = mode == kForward ? a.y : mode == kDx ? (const void *)a.dx : a.dw;
    const int64_t cs = mode == kForward ? a.y_stride : mode == kDx ? a.dx_stride : a.n_in;
    return w && x && dy && (uintptr_t)c % 16 == 0 && cs % 4 == 0 && a.n_in % 8 == 0 && a.n_out % 8 == 0;
}

// Row tiles of bm rows that the groups make if each leaves half a tile, and the
// tiles of a product.
template <Mode MODE>
int64_t likely_tiles(const GroupedArgs &a, int64_t bm, int64_t bn) {
    if (MODE == kDw) return (int64_t)a.groups * ceil_div(a.n_out, bm) * ceil_div(a.n_in, bn);
    const int64_t parts = a.groups < a.rows ? a.groups : a.rows;
    return (ceil_div(a.rows, bm) + parts / 2) * ceil_div(MODE == kForward ? a.n_out : a.n_in, bn);
}

template <Mode MODE, int BM, int BN, int WM, int WN, int NB>
hipError_t launch_tiled(const GroupedArgs &a, hipStream_t s) {
    const int64_t blocks = MODE == kDw ? likely_tiles<kDw>(a, BM, BN)
                                       : row_tiles(a, BM) * ceil_div(MODE == kForward ? a.n_out : a.n_in, BN);
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL((k_grouped<MODE, BM, BN, WM, WN, NB>), dim3((uint32_t)blocks), dim3(64 * WM * WN), 0, s, a);
    return hipGetLastError();
}

// The largest tile whose tiles still occupy the 256 compute units (a large tile
// moves fewer operand bytes for its products, but takes a unit to itself; two
// blocks of the smaller ones share one).
template <Mode MODE>
hipError_t launch(const GroupedArgs &a, hipStream_t s) {
    if (!tiled(a, MODE)) return launch_any<MODE>(a, s);
    if (likely_tiles<MODE>(a, 256, 256) >= 512) return launch_tiled<MODE, 256, 256, 2, 4, 4>(a, s);
    if (likely_tiles<MODE>(a, 128, 128) >= 192) return launch_tiled<MODE, 128, 128, 2, 2, 4>(a, s);
    return launch_tiled<MODE, 64, 128, 2, 2, 6>(a, s);
}

}  // namespace

bool grouped_fits(const GroupedArgs &a, bool forward, bool dx, bool dw) {
    return (!forward || blocks_any(a, kForward) <= kMaxBlocks) && (!dx || blocks_any(a, kDx) <= kMaxBlocks) &&
           (!dw || blocks_any(a, kDw) <= kMaxBlocks);
}

hipError_t launch_grouped_forward(const GroupedArgs &a, hipStream_t s) { return launch<kForward>(a, s); }
hipError_t launch_grouped_dx(const GroupedArgs &a, hipStream_t s) { return launch<kDx>(a, s); }
hipError_t launch_grouped_dw(const GroupedArgs &a, hipStream_t s) { return launch<kDw>(a, s); }

}  // namespace sdpops
