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
#include "sdp_ops_plan.h"

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
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef u32x4 __attribute__((aligned(8))) u32x4_even;  // rows of C may start at any 4 elements

// The wave of this thread in its block, in a scalar register.
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// How a segment's place depends on its depth (by depth; T / 16 segments a depth).
template <int T>
__device__ __forceinline__ int turn(int d) {
    const int f = (d & 3) | ((d >> 3) & 1) << 2;
    return T >= 128 ? f : f & (T / 16 - 1);
}

// The lane, worked out where it is used: what depends on it is not to be kept in
// registers through the steps.
__device__ __forceinline__ int lane_anew() {
    int l = threadIdx.x & 63;
    asm volatile("" : "+v"(l));
    return l;
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

    // outer: how many outer elements exist from the first on; the others come as 0
    __device__ __forceinline__ void init(const uint16_t *first, int64_t stride, int64_t outer) {
        const int lane = lane_anew(), wave = wave_id();
        base = (const char *)first;
        step = BY_DEPTH ? kDepth * stride * 2 : kDepth * 2;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int idx = j * WAVES + wave;
            if (BY_DEPTH) {
                const int d = (idx * 64 + lane) / kPieces, place = lane % kPieces;
                const int piece = ((place >> 1) ^ turn<T>(d)) * 2 + (place & 1);
                off[j] = piece * 8 < outer ? (uint32_t)d * (uint32_t)(stride * 2) + piece * 16 : kRange;
            } else {
                const int r = idx * 16 + lane / 4;
                const int piece = (lane & 3) ^ (lane >> 3 & 3);
                off[j] = r < outer ? (uint32_t)r * (uint32_t)(stride * 2) + piece * 16 : kRange;
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

// Four neighbouring 16 x 16 tiles, of which a lane holds columns 4 (lane / 16) + 0..3
// of row lane % 16, as BF16 in pieces of 8 columns: columns 16 (lane / 16) +
// 8 (lane / 8 % 2) + 0..7 of row lane % 8 (`top`) and of row 8 + lane % 8 (`bottom`), so
// that 8 lanes store a row's 128 bytes, a whole cache line, in one instruction.  The
// tiles' order and the 16 lanes' are exchanged first, then a piece of each lane l with
// one of lane l ^ 8.
// (Stored as they lie, 8 bytes to a lane, 16 lines an instruction: 65,536 rows, 16
// groups, 1024 x 1024: 180 us against 160 forward.)
__device__ __forceinline__ void wide_rows(const f32x4 (&c)[4], u32x4 *top, u32x4 *bottom) {
    uint32_t r[4][2];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j][0] = pack2(c[j][0], c[j][1]), r[j][1] = pack2(c[j][2], c[j][3]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x2 s = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(r[j][h], r[j + 2][h], false, false));
            r[j][h] = s[0], r[j + 2][h] = s[1];
        }
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const u32x2 s = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(r[j][h], r[j + 1][h], false, false));
            r[j][h] = s[0], r[j + 1][h] = s[1];
        }
    }
    const bool upper = threadIdx.x & 8;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t first = r[k / 2][k & 1], second = r[2 + k / 2][k & 1];
        const uint32_t other = __builtin_amdgcn_mov_dpp(upper ? first : second, 0x128, 0xf, 0xf, false);
        (*top)[k] = upper ? other : first;
        (*bottom)[k] = upper ? second : other;
    }
}

// A block's tile of C and its operands.  With splits (dw only), blockIdx.y is a part
// of the rows, whose product goes to the partial sums.
struct Place {
    int64_t m0, m1, n0, n1;  // of C
    int32_t depth;
    const uint16_t *A, *B;   // elements (m0, 0) and (n0, 0)
    int64_t sa, sb;          // by row: from row to row; by depth: from depth to depth
    char *C;
    int64_t c_stride;
    bool f32, none;
};

template <Mode MODE, int BM, int BN>
__device__ __forceinline__ Place place_of(const GroupedArgs &a) {
    Place p;
    p.none = false;
    p.f32 = MODE != kDx && a.out_f32 != 0;
    const int64_t n_in = a.n_in, n_out = a.n_out;
    if constexpr (MODE == kDw) {
        const int tm = (int)((n_out + BM - 1) / BM), tn = (int)((n_in + BN - 1) / BN);
        const int64_t id = xcd_order(blockIdx.x, gridDim.x);
        const int e = (int)(id / (tm * tn)), in_group = (int)(id - (int64_t)e * (tm * tn));
        int64_t row;
        int column;
        panel_order(in_group, tm, tn, &row, &column);
        p.m0 = row * BM, p.m1 = n_out;
        p.n0 = (int64_t)column * BN, p.n1 = n_in;
        int64_t t0, t1;
        group_rows(a, e, &t0, &t1);
        p.depth = (int)(t1 - t0);
        p.A = a.dy + t0 * a.y_stride + p.m0, p.sa = a.y_stride;
        p.B = a.x + t0 * a.x_stride + p.n0, p.sb = a.x_stride;
        p.C = (char *)a.dw, p.c_stride = n_in;
        if (a.splits > 1) {
            const int steps = parts_of(p.depth, kDepth), each = parts_of(steps, a.splits);
            const int from = (int)blockIdx.y * each * kDepth;
            p.depth = from < p.depth ? min(p.depth - from, each * kDepth) : 0;
            p.A += p.depth ? from * p.sa : 0;
            p.B += p.depth ? from * p.sb : 0;
            p.C = (char *)(a.partials + blockIdx.y * (a.groups * n_out * n_in));
            p.f32 = true;
        }
        p.C += (p.f32 ? 4 : 2) * (e * n_out * n_in);
    } else {
        const int64_t cols = MODE == kForward ? n_out : n_in;
        const int tn = (int)((cols + BN - 1) / BN);
        const int64_t tm = find_row_tile<BM>(a, -1).tiles;
        if (blockIdx.x >= tm * tn) {
            p.none = true;
            return p;
        }
        int64_t row;
        int column;
        panel_order(xcd_order(blockIdx.x, tm * tn), tm, tn, &row, &column);
        const RowTile t = find_row_tile<BM>(a, row);
        const bool empty = t.group == a.groups;
        const uint16_t *w = a.w + (empty ? 0 : (int64_t)t.group * n_out * n_in);
        p.m0 = t.first, p.m1 = t.end;
        p.n0 = (int64_t)column * BN, p.n1 = cols;
        p.depth = empty ? 0 : MODE == kForward ? a.n_in : a.n_out;
        if constexpr (MODE == kForward) {
            p.A = a.x + p.m0 * a.x_stride, p.sa = a.x_stride;
            p.B = w + p.n0 * n_in, p.sb = n_in;
            p.C = (char *)a.y, p.c_stride = a.y_stride;
        } else {
            p.A = a.dy + p.m0 * a.y_stride, p.sa = a.y_stride;
            p.B = w + p.n0, p.sb = n_in;
            p.C = (char *)a.dx, p.c_stride = a.dx_stride;
        }
    }
    return p;
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

    const Place at = place_of<MODE, BM, BN>(a);
    if (at.none) return;
    const int64_t m0 = at.m0, m1 = at.m1, n0 = at.n0, n1 = at.n1;

    // the waves' 16-row fragments alternate, so that a tile with few rows is
    // shared by all of them; their columns lie together
    const int wave = wave_id(), lane = threadIdx.x & 63;
    const int wm = wave / WN * 16, wn = wave % WN * (BN / WN);
    f32x4 acc[MT][NT] = {};
    const int steps = parts_of(at.depth, kDepth);
    // the whole contraction, over the first MU of a wave's row fragments
    auto contract = [&](auto used) __attribute__((always_inline)) {
        constexpr int MU = decltype(used)::value;
        constexpr int kLoads = OpA::template loads<MU * WM * 16>() + OpB::template loads<BN>();
        OpA oa;
        OpB ob;
        oa.init(at.A, at.sa, m1 - m0);
        ob.init(at.B, at.sb, n1 - n0);
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
        int left = at.depth;  // of the contraction, to load
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
        static_assert(NB % 2 == 0, "a step's registers follow from its buffer");
        for (int k = 0; k < steps; k += NB) {
#pragma unroll
            for (int u = 0; u < NB; ++u) {
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
    const int g = lane >> 4;
    if constexpr (NT == 4) {
        if (!at.f32) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                u32x4 half[2];
                wide_rows(acc[i], half, half + 1);
                const int64_t n = n0 + wn + 16 * g + (lane & 8);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t m = m0 + wm + 16 * WM * i + 8 * h + (lane & 7);
                    if (m < m1 && n < n1) *(u32x4_even *)((uint16_t *)at.C + m * at.c_stride + n) = half[h];
                }
            }
            return;
        }
    }
    // a lane holds 4 neighbouring columns of row lane % 16 of each 16 x 16 tile
    auto store = [&](auto put) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = m0 + wm + 16 * WM * i + (lane & 15);
            if (m >= m1) continue;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int64_t n = n0 + wn + 16 * j + 4 * g;
                if (n < n1) put(m * at.c_stride + n, acc[i][j]);
            }
        }
    };
    if (NT == 4 || at.f32)
        store([&](int64_t i, f32x4 v) { *(f32x4 *)((float *)at.C + i) = v; });
    else
        store([&](int64_t i, f32x4 v) {
            *(uint2 *)((uint16_t *)at.C + i) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
        });
}

// ---- any size, stride and alignment ---------------------------------------------

typedef u32x4 __attribute__((aligned(2))) u32x4_any;

__device__ __attribute__((aligned(16))) const uint32_t zero_piece[4] = {0, 0, 0, 0};

// An operand whose rows start and end anywhere: the same tile in LDS, its 16-byte
// pieces loaded into registers and written there.  A piece past the tensor is loaded
// from a piece of zeros, and a row's last, shorter one with the elements before it,
// so that every load is the same instruction and none is waited for at a branch.
// SHORT: a row may have fewer than 8 elements; those pieces come element by element.
template <int T, bool BY_DEPTH, int THREADS, bool SHORT>
struct Loose {
    static constexpr int kEach = T * kDepth * 2 / 16 / THREADS;
    static constexpr int kBytes = T * kDepth * 2;
    static constexpr int kPieces = T / 8;
    const uint16_t *first;
    int64_t stride;
    int32_t outer;

    __device__ __forceinline__ void init(const uint16_t *first_, int64_t stride_, int64_t outer_) {
        first = first_, stride = stride_, outer = outer_ < T ? (int32_t)outer_ : T;
    }
    // Piece j of this thread: its row (or depth), its place in the row, and the
    // elements that it has (0 or less: none).
    __device__ __forceinline__ void piece_of(int j, int left, int *r, int *piece, int *n) const {
        const int q = j * THREADS + threadIdx.x;
        *r = BY_DEPTH ? q / kPieces : q / 4;
        const int place = BY_DEPTH ? q % kPieces : q & 3;
        *piece = BY_DEPTH ? ((place >> 1) ^ turn<T>(*r)) * 2 + (place & 1) : place ^ (*r >> 1 & 3);
        *n = *r < (BY_DEPTH ? left : outer) ? (BY_DEPTH ? outer : left) - *piece * 8 : 0;
    }
    // Depths from k on, `left` of them being there.
    __device__ __forceinline__ void load(u32x4 (&held)[kEach], int64_t k, int left) const {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            int r, piece, n;
            piece_of(j, left, &r, &piece, &n);
            const uint16_t *p = first + (BY_DEPTH ? (k + r) * stride : r * stride + k) + piece * 8;
            if constexpr (SHORT) {
                u32x4 v = {0, 0, 0, 0};
                for (int e = 0; e < 8; ++e)
                    if (e < n) v[e / 2] |= (uint32_t)p[e] << (e % 2 * 16);
                held[j] = v;
            } else {
                const uint16_t *from = n >= 8 ? p : n > 0 ? p - (8 - n) : (const uint16_t *)zero_piece;
                held[j] = *(const u32x4_any *)from;
            }
        }
    }
    __device__ __forceinline__ void write(const u32x4 (&held)[kEach], char *lds, int left) const {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            u32x4 v = held[j];
            if constexpr (!SHORT) {
                int r, piece, n;
                piece_of(j, left, &r, &piece, &n);
                if (n > 0 && n < 8) {
                    // the last n of the 8 elements to the front
                    const int s = 8 - n;
                    if (s & 4) v = u32x4{v[2], v[3], 0u, 0u};
                    if (s & 2) v = u32x4{v[1], v[2], v[3], 0u};
                    if (s & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
                }
            }
            *(u32x4 *)(lds + (j * THREADS + threadIdx.x) * 16) = v;
        }
    }
};

// T x T tiles, four waves; two buffers, and the next two steps' pieces on their way
// to registers while this one's products run.
template <Mode MODE, int T, bool SHORT>
__global__ __launch_bounds__(256) void k_grouped_loose(GroupedArgs a) {
    constexpr int kTiles = T / 2 / 16;  // 16 x 16 tiles of a wave, each way
    constexpr bool kADepth = MODE == kDw, kBDepth = MODE != kForward;
    using OpA = Loose<T, kADepth, 256, SHORT>;
    using OpB = Loose<T, kBDepth, 256, SHORT>;
    __shared__ __attribute__((aligned(1024))) char lds_a[2][OpA::kBytes], lds_b[2][OpB::kBytes];
    const Place at = place_of<MODE, T, T>(a);
    if (at.none) return;
    const int wave = wave_id(), lane = threadIdx.x & 63, wm = wave / 2 * (T / 2), wn = wave % 2 * (T / 2);
    OpA oa;
    OpB ob;
    oa.init(at.A, at.sa, at.m1 - at.m0);
    ob.init(at.B, at.sb, at.n1 - at.n0);
    Reader<T, kADepth, 1> ra;
    Reader<T, kBDepth, 1> rb;
    ra.init(wm);
    rb.init(wn);
    f32x4 acc[kTiles][kTiles] = {};
    const int steps = parts_of(at.depth, kDepth);
    u32x4 ha[2][OpA::kEach], hb[2][OpB::kEach];
    auto load = [&](int f, int k) __attribute__((always_inline)) {
        if (k >= steps) return;
        oa.load(ha[f], (int64_t)k * kDepth, at.depth - k * kDepth);
        ob.load(hb[f], (int64_t)k * kDepth, at.depth - k * kDepth);
    };
    load(0, 0);
    load(1, 1);
    for (int k0 = 0; k0 < steps; k0 += 2)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int k = k0 + f;
            if (k >= steps) break;
            oa.write(ha[f], lds_a[f], at.depth - k * kDepth);
            ob.write(hb[f], lds_b[f], at.depth - k * kDepth);
            __syncthreads();
            load(f, k + 2);
            bf16x8 fa[kTiles], fb[kTiles];
#pragma unroll
            for (int i = 0; i < kTiles; ++i) fa[i] = ra.read(lds_a[f], i), fb[i] = rb.read(lds_b[f], i);
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int j = 0; j < kTiles; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
        }
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int64_t m = at.m0 + wm + 16 * i + (lane & 15);
        if (m >= at.m1) continue;
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t n = at.n0 + wn + 16 * j + 4 * (lane >> 4) + r;
                if (n >= at.n1) continue;
                if (at.f32)
                    ((float *)at.C)[m * at.c_stride + n] = acc[i][j][r];
                else
                    store1((uint16_t *)at.C + m * at.c_stride + n, acc[i][j][r]);
            }
    }
}

// dw from its partial sums, added in order and rounded.
__global__ __launch_bounds__(256) void k_grouped_join(const float *partials, int splits, int64_t elems, void *dw,
                                                      int f32) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < elems; i += (int64_t)gridDim.x * 256) {
        float v = 0.0f;
        for (int k = 0; k < splits; ++k) v += partials[k * elems + i];
        if (f32)
            ((float *)dw)[i] = v;
        else
            store1((uint16_t *)dw + i, v);
    }
}

// ---- sizes and strides without whole pieces, laid out anew ---------------------------

// Groups of rows of `src_cols` elements into groups of rows of `dst_cols`, zeros where
// the source has no row or column: into whole pieces before the products, and out of
// them after.  A block takes `rows` rows, a thread 16 bytes at a time.
struct RowsCopy {
    const void *src;
    void *dst;
    int64_t src_stride, dst_stride, dst_rows;  // dst_rows: of all groups
    int32_t src_group, dst_group;              // rows of a group
    int32_t src_cols, dst_cols, rows;
};

template <typename T>
__global__ __launch_bounds__(256) void k_grouped_copy(RowsCopy c) {
    constexpr int kN = 16 / (int)sizeof(T);
    const int pieces = (c.dst_cols - 1) / kN + 1;
    const int64_t first = (int64_t)blockIdx.x * c.rows;
    const int rows = (int)min((int64_t)c.rows, c.dst_rows - first);
    for (uint32_t i = threadIdx.x; i < (uint32_t)rows * pieces; i += 256) {
        const uint32_t r = i / pieces, piece = i - r * pieces;
        const int64_t row = first + r, group = row / c.dst_group;
        const int in_group = (int)(row - group * c.dst_group), col = (int)piece * kN;
        const T *from = (const T *)c.src + (group * c.src_group + in_group) * c.src_stride + col;
        T *to = (T *)c.dst + row * c.dst_stride + col;
        const int n_src = in_group < c.src_group ? c.src_cols - col : 0, n_dst = c.dst_cols - col;
        union {
            u32x4 all;
            T each[kN];
        } v;
        v.all = u32x4{0, 0, 0, 0};
        if (n_src >= kN) {
            v.all = *(const u32x4_any *)from;
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (e < n_src) v.each[e] = from[e];
        }
        if (n_dst >= kN) {
            *(u32x4_any *)to = v.all;
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (e < n_dst) to[e] = v.each[e];
        }
    }
}

// ---- many tiles --------------------------------------------------------------------

// 256 x 256 tiles, one block to a compute unit, each block walking its share of the
// tiles as one stream of steps: the last steps of a tile load the first ones of
// the next, and a tile's results are stored while the next one's products run.
// 65,536 rows, 128 groups of unequal sizes, 2048 x 1536: forward 480 us, dx 470, dw 550
// (860, 880 and 750 TFLOP/s); forward the matrix units are busy for 42% of the time, at
// the 2.1 GHz that the card's power leaves; the rest is weights that come from memory
// and part tiles at the groups' ends.
constexpr int kStreamBlocks = 256, kStreamTile = 256, kStreamWm = 2, kStreamWn = 4, kStreamNb = 4;
constexpr int kSortedGroups = 256;  // dw: up to so many groups are taken largest first

template <Mode MODE>
__global__ __launch_bounds__(512) void k_grouped_stream(GroupedArgs a) {
    constexpr int BM = kStreamTile, BN = kStreamTile, WM = kStreamWm, WN = kStreamWn, NB = kStreamNb;
    constexpr int kWaves = WM * WN, MT = BM / WM / 16, NT = BN / WN / 16;
    constexpr bool kADepth = MODE == kDw, kBDepth = MODE != kForward;
    using OpA = Operand<BM, kADepth, kWaves>;
    using OpB = Operand<BN, kBDepth, kWaves>;
    constexpr int kBuffer = OpA::kBytes + OpB::kBytes;
    constexpr int kLoads = OpA::template loads<BM>() + OpB::template loads<BN>(), kStores32 = MT * NT, kStores16 = MT * 2;
    static_assert(NT == 4, "wide_rows");
    __shared__ __attribute__((aligned(1024))) char lds0[kBuffer], lds1[kBuffer], lds2[kBuffer], lds3[kBuffer];
    // of each group (the last: the rows of none): its end, and the row tiles before it
    __shared__ int32_t ends[SDP_GROUPED_MAX_GROUPS + 1], tiles_before[SDP_GROUPED_MAX_GROUPS + 2];
    __shared__ int16_t by_size[kSortedGroups];

    const int lane = threadIdx.x & 63, wave = wave_id();
    if (wave == 0) {
        int64_t run = 0;
        int32_t tiles = 0;
        for (int base = 0; base <= a.groups; base += 64) {
            const int e = base + lane;
            const int64_t end = group_end(a, e, run);
            int64_t start = shfl_up64(end, 1);
            if (lane == 0) start = run;
            const int32_t mine = e <= a.groups ? (int32_t)((end - start + BM - 1) / BM) : 0;
            int32_t upto = mine;
            for (int d = 1; d < 64; d <<= 1) {
                const int32_t before = __shfl_up(upto, d);
                if (lane >= d) upto += before;
            }
            if (e <= a.groups) ends[e] = (int32_t)end, tiles_before[e] = tiles + upto - mine;
            run = shfl64(end, 63);
            tiles += __shfl(upto, 63);
        }
        if (lane == 0) tiles_before[a.groups + 1] = tiles;
    }
    __syncthreads();
    const bool sorted = MODE == kDw && a.groups <= kSortedGroups;
    if (sorted) {
        for (int e = threadIdx.x; e < a.groups; e += 512) {
            const int32_t size = ends[e] - (e ? ends[e - 1] : 0);
            int rank = 0;
            for (int f = 0; f < a.groups; ++f) {
                const int32_t other = ends[f] - (f ? ends[f - 1] : 0);
                rank += other > size || (other == size && f < e);
            }
            by_size[rank] = (int16_t)e;
        }
        __syncthreads();
    }

    const int64_t n_in = a.n_in, n_out = a.n_out;
    const int64_t cols = MODE == kForward ? n_out : n_in;
    const int tn = (int)((cols + BN - 1) / BN);
    const int64_t tm = MODE == kDw ? (n_out + BM - 1) / BM
                                   : __builtin_amdgcn_readfirstlane(tiles_before[a.groups + 1]);
    const int64_t total = MODE == kDw ? tm * tn * a.groups : tm * tn;

    // The block's tile of round r.  A round's 256 tiles are neighbours, 32 of them
    // to an XCD; for dw, where the groups' sizes make tiles cost more or less and they
    // come sorted, every other round goes the other way round.
    auto tile_id = [&](int r) {
        const int place = (int)(blockIdx.x & 7) * (kStreamBlocks / 8) + (int)(blockIdx.x >> 3);
        return (int64_t)r * kStreamBlocks + (sorted && (r & 1) ? kStreamBlocks - 1 - place : place);
    };
    struct Tile {
        const uint16_t *A, *B;
        char *C;
        int32_t rows, columns, depth;  // that exist
    };
    const int64_t sa = MODE == kForward ? a.x_stride : a.y_stride, sb = MODE == kDw ? a.x_stride : n_in;
    const int64_t c_stride = MODE == kForward ? a.y_stride : MODE == kDx ? a.dx_stride : n_in;
    const bool f32 = MODE != kDx && a.out_f32;
    const int c_size = f32 ? 4 : 2;
    auto tile = [&](int64_t id) {
        Tile t;
        int64_t row;
        int column;
        if constexpr (MODE == kDw) {
            const int64_t g = id / (tm * tn);
            panel_order(id - g * (tm * tn), tm, tn, &row, &column);
            const int e = sorted ? __builtin_amdgcn_readfirstlane(by_size[g]) : (int)g;
            const int t0 = e ? __builtin_amdgcn_readfirstlane(ends[e - 1]) : 0;
            t.depth = __builtin_amdgcn_readfirstlane(ends[e]) - t0;
            t.A = a.dy + t0 * a.y_stride + row * BM;
            t.B = a.x + t0 * a.x_stride + (int64_t)column * BN;
            t.rows = (int)(n_out - row * BM);
            t.C = (char *)a.dw + c_size * ((e * n_out + row * BM) * n_in + (int64_t)column * BN);
        } else {
            panel_order(id, tm, tn, &row, &column);
            // the last group with at most `row` tiles before it, 64 at a time
            const int n = a.groups + 1, step = (n + 63) / 64;
            const int far = lane * step;
            const int hits = __popcll(__ballot(far < n && tiles_before[far < n ? far : 0] <= row));
            const int base = (hits - 1) * step, near = base + lane;
            const int more = __popcll(__ballot(lane < step && near < n && tiles_before[near < n ? near : 0] <= row));
            const int e = base + more - 1;
            const int start = e ? __builtin_amdgcn_readfirstlane(ends[e - 1]) : 0;
            const int64_t m0 = start + (row - __builtin_amdgcn_readfirstlane(tiles_before[e])) * BM;
            const bool empty = e == a.groups;
            const uint16_t *w = a.w + (empty ? 0 : e * n_out * n_in);
            t.rows = __builtin_amdgcn_readfirstlane(ends[e]) - (int)m0;
            t.depth = empty ? 0 : MODE == kForward ? a.n_in : a.n_out;
            if constexpr (MODE == kForward) {
                t.A = a.x + m0 * a.x_stride;
                t.B = w + (int64_t)column * BN * n_in;
                t.C = (char *)a.y + c_size * (m0 * a.y_stride + (int64_t)column * BN);
            } else {
                t.A = a.dy + m0 * a.y_stride;
                t.B = w + (int64_t)column * BN;
                t.C = (char *)a.dx + c_size * (m0 * a.dx_stride + (int64_t)column * BN);
            }
        }
        t.columns = (int)(cols - (int64_t)column * BN);
        return t;
    };

    int round = 0;
    if (tile_id(0) >= total) return;
    Tile cur = tile(tile_id(0));
    OpA oa;
    OpB ob;
    int left = cur.depth;  // of the contraction that is being loaded
    oa.init(cur.A, sa, cur.rows);
    ob.init(cur.B, sb, cur.columns);
    auto load = [&](char *lds) __attribute__((always_inline)) {
        oa.template load<BM>(lds, left);
        ob.template load<BN>(lds + OpA::kBytes, left);
        left = left > kDepth ? left - kDepth : 0;
    };
    const int wm = wave / WN * 16, wn = wave % WN * (BN / WN);
    Reader<BM, kADepth, WM> ra;
    Reader<BN, kBDepth, 1> rb;
    ra.init(wm);
    rb.init(wn);
    f32x4 acc[MT][NT] = {};
    bf16x8 fa[MT], fb[2][NT];
    int stores = 0;  // a tile's stores lie between the loads in flight: 1: kStores16, 2: kStores32 of them

    int used = MT;  // row fragments that have rows: MT, or a half or a quarter of them

    // Step u of four.  In the first three after a tile's stores those may still be
    // in flight, in front of none of the loads that are waited for.
    auto step = [&](int u, char *lds, const char *next) __attribute__((always_inline)) {
        // (the scalars are hidden from the compiler, which would otherwise make a loop
        // of its own for each value, and run out of registers between them)
        int mu = used, after = stores;
        asm volatile("" : "+s"(mu), "+s"(after));
        if (u < 3 && after == 2)
            wait_and_meet<(NB - 2) * kLoads + kStores32>();
        else if (u < 3 && after)
            wait_and_meet<(NB - 2) * kLoads + kStores16>();
        else
            wait_and_meet<(NB - 2) * kLoads>();
        load(lds);
        const int f = u & 1;
        // A row fragment is read anew for the next step as soon as its products are
        // under way; the last step reads all of them, for whatever tile comes next.
        auto rows = [&](int i0, int i1) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (i < i0 || i >= i1) continue;
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[f][j], fa[i], acc[i][j], 0, 0, 0);
                fa[i] = ra.read(next, i);
                if (i < NT / 2) {
                    fb[f ^ 1][2 * i] = rb.read(next + OpA::kBytes, 2 * i);
                    fb[f ^ 1][2 * i + 1] = rb.read(next + OpA::kBytes, 2 * i + 1);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto reread = [&](int i0, int i1) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if (i >= i0 && i < i1) fa[i] = ra.read(next, i);
        };
        rows(0, MT / 4);
        if (mu > MT / 4)
            rows(MT / 4, MT / 2);
        else if (u == 3)
            reread(MT / 4, MT / 2);
        if (mu > MT / 2)
            rows(MT / 2, MT);
        else if (u == 3)
            reread(MT / 2, MT);
    };

    load(lds0);
    load(lds1);
    load(lds2);
    load(lds3);
    wait_and_meet<(NB - 1) * kLoads>();
#pragma unroll
    for (int j = 0; j < NT; ++j) fb[0][j] = rb.read(lds0 + OpA::kBytes, j);
#pragma unroll
    for (int i = 0; i < MT; ++i) fa[i] = ra.read(lds0, i);

    for (;;) {
        // whole fours: past the contraction loads bring zeros
        const int fours = cur.depth > 0 ? parts_of(cur.depth, 4 * kDepth) : 1;
        const int64_t next_id = tile_id(round + 1);
        const bool has_next = next_id < total;
        Tile next = cur;
        used = cur.rows <= BM / 4 ? MT / 4 : cur.rows <= BM / 2 ? MT / 2 : MT;
        for (int k = 0; k < fours; ++k) {
            if (k == fours - 1) {
                // from here on the loads are the next tile's
                left = 0;
                if (has_next) {
                    next = tile(next_id);
                    oa.init(next.A, sa, next.rows);
                    ob.init(next.B, sb, next.columns);
                    left = next.depth;
                }
            }
            step(0, lds0, lds1);
            step(1, lds1, lds2);
            step(2, lds2, lds3);
            step(3, lds3, lds0);
            stores = 0;
        }
        // all the stores are issued, those past the tile's end to an offset out of range
        const __amdgpu_buffer_rsrc_t c = __builtin_amdgcn_make_buffer_rsrc(cur.C, 0, kRange, 0x00020000);
        const int l = lane_anew();
        const uint32_t row_bytes = (uint32_t)(c_stride * c_size);
        if (f32) {
            // a lane holds 4 neighbouring columns of row lane % 16 of each 16 x 16 tile
            const int m = wm + (l & 15), n = wn + 4 * (l >> 4);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int mi = m + 16 * WM * i;
                const uint32_t at = (uint32_t)mi * row_bytes + n * 4;
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[i][j]), c,
                                                           mi < cur.rows && n + 16 * j < cur.columns ? at + 64 * j : kRange,
                                                           0, 0);
            }
        } else {
            const int m = wm + (l & 7), n = wn + 16 * (l >> 4) + (l & 8);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                u32x4 half[2];
                wide_rows(acc[i], half, half + 1);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int mi = m + 16 * WM * i + 8 * h;
                    __builtin_amdgcn_raw_buffer_store_b128(
                        half[h], c, mi < cur.rows && n < cur.columns ? (uint32_t)mi * row_bytes + n * 2 : kRange, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
        if (!has_next) break;
        cur = next;
        ++round;
        stores = f32 ? 2 : 1;
    }
    // no load may land after the block has given its LDS back
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(15 << 8 | 7 << 4);
}

int64_t ceil_div(int64_t a, int64_t b) { return a / b + (a % b != 0); }

// Most row tiles of bm rows that the groups and the rows of no group can make:
// each of them, if it has rows, adds at most one part tile.
int64_t row_tiles(const GroupedArgs &a, int64_t bm) {
    const int64_t parts = a.groups + 1 < a.rows ? a.groups + 1 : a.rows;
    const int64_t most = a.rows / bm + parts;
    return most < a.rows ? most : a.rows;
}

constexpr int64_t kMaxBlocks = 0xffffffffll / 512;

// Whether the tiled kernels can take the call: whole 16-byte pieces in every
// row, rows and results at 16-byte boundaries, and a tile's offsets in 31 bits.
bool pieces(const void *p, int64_t stride, int64_t cols) {
    return (uintptr_t)p % 16 == 0 && stride % 8 == 0 && cols % 8 == 0 && stride < ((int64_t)1 << 21);
}
bool tiled(const GroupedArgs &a, Mode mode) {
    const bool w = mode == kDw || pieces(a.w, a.n_in, a.n_in);
    const bool x = mode == kDx || pieces(a.x, a.x_stride, a.n_in);
    const bool dy = mode == kForward || pieces(a.dy, a.y_stride, a.n_out);
    const void *c = mode == kForward ? a.y : mode == kDx ? (const void *)a.dx : a.dw;
    const int64_t cs = mode == kForward ? a.y_stride : mode == kDx ? a.dx_stride : a.n_in;
    return w && x && dy && (uintptr_t)c % 16 == 0 && cs % 4 == 0 && cs < ((int64_t)1 << 21) && a.n_in % 8 == 0 &&
           a.n_out % 8 == 0;
}

int64_t columns_of(const GroupedArgs &a, Mode mode) { return mode == kForward ? a.n_out : a.n_in; }
int64_t weights_of(const GroupedArgs &a) { return (int64_t)a.groups * a.n_out * a.n_in; }

// Tiles of t x t that a product makes if each group leaves half a row tile; and the
// most that it can make.
int64_t likely_tiles(const GroupedArgs &a, Mode mode, int64_t t) {
    if (mode == kDw) return (int64_t)a.groups * ceil_div(a.n_out, t) * ceil_div(a.n_in, t);
    const int64_t parts = a.groups < a.rows ? a.groups : a.rows;
    return (ceil_div(a.rows, t) + parts / 2) * ceil_div(columns_of(a, mode), t);
}
int64_t most_tiles(const GroupedArgs &a, Mode mode, int64_t t) {
    return mode == kDw ? likely_tiles(a, mode, t) : row_tiles(a, t) * ceil_div(columns_of(a, mode), t);
}

// How a product is done: in one stream of 256 x 256 tiles, in tiles of `tile`, or
// (loose) in tiles loaded through registers; and in how many parts of the
// contraction.
struct Way {
    bool stream, loose;
    int tile, splits;
};

// The largest tile that still occupies the 256 compute units, as it loads the fewest
// bytes for its products.  Measured with weights from memory, 256 against 128 against
// 64: 8,192 rows, 16 groups, 1024 x 1024, 160 tiles of 256: 36 us, 43, 57; 4,096 rows, 8
// groups, 2048 -> 1536, 120 tiles: 59, 48, 76; 1,000 rows, 16 groups, 2048 -> 1024, 128
// tiles of 128: 31 us (64: 33); 64 rows, one group, 2048 x 2048, 16 tiles of 128: 18 (64: 15).
//
// From 256 tiles of 256 on and with two groups or more they are walked as a stream.
// It evens out the groups' sizes in dw (16,384 rows, 8 groups of unequal sizes, 2048 x
// 2048: 163 us against 191 in blocks of one tile; 65,536 rows, 64 groups, 2048 x 1536:
// 466 against 500; with equal groups 136 against 123 and 464 against 410, which the
// host cannot see), and in the other products it hides the short contractions' ends
// (65,536 rows, 128 groups, 768 -> 2048: 278 us against 333).  Long ones of large groups
// fare better in blocks, whose tiles come to a compute unit as it gets free (16,384
// rows, 8 groups, 2048 x 2048: 169 us against 190; 40,000 rows, 4 groups, 4096 x 4096:
// 1101 against 1154; at 512 rows a group, 2048 -> 1536: 490 against 480).
//
// Where dw has few tiles even of 64 and many rows, parts of the rows are done by blocks
// of their own (30,000 rows, 3 groups, 256 x 256: 29 us against 90; 65,536 rows, 16
// groups, 136 x 200: 46 against 73); loose tiles of 128, four waves each, want it up to
// two a compute unit (65,536 rows, 8 groups, 261 x 1025: 280 us against 456; 16 groups,
// 255 x 777: 175 against 307).  The other products' contractions are shorter, and
// parts gained nothing there (16 rows over 16 groups, 4096 -> 1024: 32 us against 29; 64
// rows, 2048 x 2048: 15 against 15).
Way way_of(const GroupedArgs &a, Mode mode) {
    const int64_t t256 = likely_tiles(a, mode, 256), t128 = likely_tiles(a, mode, 128), t64 = likely_tiles(a, mode, 64);
    Way w{false, !tiled(a, mode), 64, 1};
    const bool long_large = mode != kDw && (mode == kForward ? a.n_in : a.n_out) >= 2048 &&
                            a.rows >= 768 * (int64_t)a.groups;
    if (!w.loose && t256 >= 150) {
        w.tile = 256;
        w.stream = a.groups >= 2 && t256 >= (mode == kDw ? 257 : 256) && !long_large;
    } else if (t128 >= 150) {
        w.tile = 128;
    }
    const int64_t tiles = w.tile == 64 ? t64 : t128, few = w.tile == 64 ? 384 : w.loose ? 513 : 0;
    if (mode == kDw && w.tile < 256 && tiles > 0 && tiles < few) {
        const int64_t depth = a.rows / a.groups;
        int64_t n = 1024 / tiles;
        n = n < depth / (8 * kDepth) ? n : depth / (8 * kDepth);
        if (depth < 64 * kDepth) n = 1;
        n = n < 16 ? n : 16;
        const int64_t bytes = 4 * weights_of(a), room = bytes ? ((int64_t)64 << 20) / bytes : 1;
        n = n < room ? n : room;
        w.splits = n > 1 ? (int)n : 1;
    }
    return w;
}

template <Mode MODE, int T, int WM, int WN, int NB>
void launch_tiled(const GroupedArgs &a, hipStream_t s) {
    const dim3 grid((uint32_t)most_tiles(a, MODE, T), a.splits);
    hipLaunchKernelGGL((k_grouped<MODE, T, T, WM, WN, NB>), grid, dim3(64 * WM * WN), 0, s, a);
}
template <Mode MODE, int T>
void launch_loose(const GroupedArgs &a, hipStream_t s) {
    const dim3 grid((uint32_t)most_tiles(a, MODE, T), a.splits);
    if (a.n_in < 8 || a.n_out < 8)
        hipLaunchKernelGGL((k_grouped_loose<MODE, T, true>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((k_grouped_loose<MODE, T, false>), grid, dim3(256), 0, s, a);
}

template <Mode MODE>
hipError_t launch(const GroupedArgs &args, hipStream_t s) {
    GroupedArgs a = args;
    const Way w = way_of(a, MODE);
    if (most_tiles(a, MODE, w.tile) == 0) return hipSuccess;
    a.splits = w.splits;
    if (w.stream)
        hipLaunchKernelGGL((k_grouped_stream<MODE>), dim3(kStreamBlocks), dim3(512), 0, s, a);
    else if (w.loose)
        w.tile == 128 ? launch_loose<MODE, 128>(a, s) : launch_loose<MODE, 64>(a, s);
    else if (w.tile == 256)
        launch_tiled<MODE, 256, 2, 4, 4>(a, s);
    else if (w.tile == 128)
        launch_tiled<MODE, 128, 2, 2, 4>(a, s);
    else
        launch_tiled<MODE, 64, 2, 2, 6>(a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || w.splits == 1) return e;
    const int64_t elems = weights_of(a), blocks = ceil_div(elems, 256);
    hipLaunchKernelGGL(k_grouped_join, dim3((uint32_t)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, a.partials,
                       w.splits, elems, a.dw, a.out_f32);
    return hipGetLastError();
}

// A call whose tensors are laid out anew for the tiled kernels: `to`, the call on the
// copies in the workspace (from its start; offsets until `base` is added).
struct Packed {
    bool any, x, w, dy, y, dx, dw;
    GroupedArgs to;
    size_t bytes;
};

// Which tensors have no whole pieces, and whether copies of them pay.  The loose kernel
// does 200 to 300 TFLOP/s and the tiled ones 500 to 900, and copies go at 5 TB/s and cost
// a launch each: they pay from some 110 operations for each byte that they move on.
// Both products of the backward, copies against none: 65,536 rows, 16 groups, 515 x
// 1025 (157 operations a byte for one product): 493 us against 700; 30,000 rows, 8 groups,
// 1023 x 2047 (288): 483 against 816.  dx alone of 57,617 rows, 105 groups, 328 x 2905
// (102): 451 against 338; forward of 8,192 rows, 32 groups, 1021 x 2047 (93): 175 against 142.
Packed pack_of(const GroupedArgs &a, bool forward, bool dx, bool dw) {
    Packed p{};
    p.to = a;
    GroupedArgs &b = p.to;
    const int64_t n_in = ceil_div(a.n_in, 8) * 8, n_out = ceil_div(a.n_out, 8) * 8;
    if (n_in >= (int64_t)1 << 21 || n_out >= (int64_t)1 << 21) return p;
    b.n_in = (int32_t)n_in, b.n_out = (int32_t)n_out;
    const bool same = n_in == a.n_in && n_out == a.n_out;
    const bool use_x = forward || dw, use_w = forward || dx, use_dy = dx || dw;
    const int out = a.out_f32 ? 4 : 2;
    auto result = [&](const void *c, int64_t stride, bool cols) {
        return !(cols && (uintptr_t)c % 16 == 0 && stride % 4 == 0 && stride < ((int64_t)1 << 21));
    };
    p.x = use_x && !pieces(a.x, a.x_stride, a.n_in);
    p.dy = use_dy && !pieces(a.dy, a.y_stride, a.n_out);
    p.w = use_w && !(same && (uintptr_t)a.w % 16 == 0);
    p.y = forward && result(a.y, a.y_stride, n_out == a.n_out);
    p.dx = dx && result(a.dx, a.dx_stride, n_in == a.n_in);
    p.dw = dw && result(a.dw, a.n_in, same);
    if (!(p.x || p.dy || p.w || p.y || p.dx || p.dw)) return p;
    size_t at = 0;
    int64_t moved = 0;
    auto place = [&](bool on, int64_t elems, int size) {
        const size_t here = at;
        if (on) at += ((size_t)elems * size + 255) / 256 * 256, moved += 2 * elems * size;
        return (uintptr_t)here;
    };
    const uintptr_t x = place(p.x, a.rows * n_in, 2), dy = place(p.dy, a.rows * n_out, 2);
    const uintptr_t w = place(p.w, a.groups * n_out * n_in, 2), y = place(p.y, a.rows * n_out, out);
    const uintptr_t gx = place(p.dx, a.rows * n_in, 2), gw = place(p.dw, a.groups * n_out * n_in, out);
    const double flops = 2.0 * a.rows * a.n_in * a.n_out * ((forward ? 1 : 0) + (dx ? 1 : 0) + (dw ? 1 : 0));
    if (p.x) b.x = (const uint16_t *)x, b.x_stride = n_in;
    if (p.dy) b.dy = (const uint16_t *)dy;
    if (p.w) b.w = (const uint16_t *)w;
    if (p.y) b.y = (void *)y;
    if (p.dx) b.dx = (uint16_t *)gx, b.dx_stride = n_in;
    if (p.dw) b.dw = (void *)gw;
    if (p.dy || p.y) b.y_stride = n_out;
    p.bytes = at;
    const bool large = (!forward || way_of(b, kForward).tile >= 128) && (!dx || way_of(b, kDx).tile >= 128) &&
                       (!dw || way_of(b, kDw).tile >= 128);
    p.any = large && flops > 110.0 * (double)moved + 5e9 && at <= ((size_t)2 << 30);
    return p;
}

template <typename T>
hipError_t copy_rows(const void *src, int64_t src_stride, int64_t src_group, int64_t src_cols, void *dst,
                     int64_t dst_stride, int64_t dst_group, int64_t dst_cols, int64_t groups, hipStream_t s) {
    RowsCopy c{src, dst, src_stride, dst_stride, groups * dst_group, (int32_t)src_group, (int32_t)dst_group,
               (int32_t)src_cols, (int32_t)dst_cols, 1};
    if (c.dst_rows == 0) return hipSuccess;
    // a thread does a few pieces, and there are some blocks for each compute unit
    const int64_t most = ceil_div(c.dst_rows, 2048);
    c.rows = (int32_t)(most < 32 ? most : 32);
    hipLaunchKernelGGL((k_grouped_copy<T>), dim3((uint32_t)ceil_div(c.dst_rows, c.rows)), dim3(256), 0, s, c);
    return hipGetLastError();
}

hipError_t copy_out(bool f32, const void *src, int64_t src_stride, int64_t src_group, int64_t src_cols, void *dst,
                    int64_t dst_stride, int64_t dst_group, int64_t dst_cols, int64_t groups, hipStream_t s) {
    return f32 ? copy_rows<float>(src, src_stride, src_group, src_cols, dst, dst_stride, dst_group, dst_cols, groups, s)
               : copy_rows<uint16_t>(src, src_stride, src_group, src_cols, dst, dst_stride, dst_group, dst_cols, groups, s);
}

bool fits(const GroupedArgs &a, Mode mode) { return most_tiles(a, mode, way_of(a, mode).tile) <= kMaxBlocks; }
}  // namespace

bool grouped_fits(const GroupedArgs &a, bool forward, bool dx, bool dw) {
    const Packed p = pack_of(a, forward, dx, dw);
    const GroupedArgs &b = p.any ? p.to : a;
    return (!forward || fits(b, kForward)) && (!dx || fits(b, kDx)) && (!dw || fits(b, kDw));
}

size_t grouped_workspace(const GroupedArgs &a, bool forward, bool dx, bool dw) {
    const Packed p = pack_of(a, forward, dx, dw);
    if (p.any) return p.bytes;
    const int splits = dw ? way_of(a, kDw).splits : 1;
    return splits > 1 ? (size_t)splits * (size_t)weights_of(a) * 4 : 0;
}

#define GROUPED_TRY(e)                              \
    do {                                            \
        const hipError_t e_ = (e);                  \
        if (e_ != hipSuccess) return e_;            \
    } while (0)

hipError_t launch_grouped(const GroupedArgs &a, bool forward, bool dx, bool dw, void *space, hipStream_t s) {
    const Packed p = pack_of(a, forward, dx, dw);
    GroupedArgs b = a;
    if (p.any) {
        b = p.to;
        char *base = (char *)space;
        if (p.x) b.x = (const uint16_t *)(base + (uintptr_t)b.x);
        if (p.dy) b.dy = (const uint16_t *)(base + (uintptr_t)b.dy);
        if (p.w) b.w = (const uint16_t *)(base + (uintptr_t)b.w);
        if (p.y) b.y = base + (uintptr_t)b.y;
        if (p.dx) b.dx = (uint16_t *)(base + (uintptr_t)b.dx);
        if (p.dw) b.dw = base + (uintptr_t)b.dw;
        if (p.x) GROUPED_TRY(copy_rows<uint16_t>(a.x, a.x_stride, a.rows, a.n_in, (void *)b.x, b.n_in, a.rows, b.n_in, 1, s));
        if (p.dy)
            GROUPED_TRY(copy_rows<uint16_t>(a.dy, a.y_stride, a.rows, a.n_out, (void *)b.dy, b.n_out, a.rows, b.n_out, 1, s));
        if (p.w)
            GROUPED_TRY(copy_rows<uint16_t>(a.w, a.n_in, a.n_out, a.n_in, (void *)b.w, b.n_in, b.n_out, b.n_in, a.groups, s));
    } else {
        b.partials = (float *)space;
    }
    if (forward) GROUPED_TRY(launch<kForward>(b, s));
    if (dx) GROUPED_TRY(launch<kDx>(b, s));
    if (dw) GROUPED_TRY(launch<kDw>(b, s));
    if (p.any && p.y)
        GROUPED_TRY(copy_out(a.out_f32, b.y, b.n_out, a.rows, b.n_out, a.y, a.y_stride, a.rows, a.n_out, 1, s));
    if (p.any && p.dx) GROUPED_TRY(copy_out(false, b.dx, b.n_in, a.rows, b.n_in, a.dx, a.dx_stride, a.rows, a.n_in, 1, s));
    if (p.any && p.dw)
        GROUPED_TRY(copy_out(a.out_f32, b.dw, b.n_in, b.n_out, b.n_in, a.dw, a.n_in, a.n_out, a.n_in, a.groups, s));
    return hipSuccess;
}

}  // namespace sdpops
