// gfx950 kernels of sdp_embed and its backward.
//
//   out[t] = s table[id_t];   dtable[v] = s sum over t with id_t = v of dout[t]
// Memory bounds both: the tokens' rows, and backward the whole table where it is
// written anew.  Backward the tokens are sorted by id (sdp_order.hip), so that each
// row of the table is one run of them.  Blocks take pieces of 128 places: a run within a
// piece is summed and written at once, of a longer one each piece leaves its sum, and
// the kernel that writes the rest of the table adds those in their order.  32,768 tokens
// of 4,096 BF16 channels, 151,936 rows: 97 us, backward 308, of which the sort takes 28.
#include <algorithm>
#include <type_traits>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"

namespace sdpops {
namespace {

constexpr int kWaves = 4;
constexpr int kColumns = 512;  // of a wave: eight to a lane
constexpr int kPieceWaves = 8, kWavePlaces = 16, kPiece = kPieceWaves * kWavePlaces;

__host__ __device__ inline int64_t pieces_of(const EmbedArgs &a) { return (a.tokens + kPiece - 1) / kPiece; }

template <typename T, typename R>
__global__ __launch_bounds__(64 * kWaves) void k_embed(EmbedArgs a, int slices) {
    const int lane = threadIdx.x & 63;
    for (int64_t w = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); w < a.tokens * slices;
         w += (int64_t)gridDim.x * kWaves) {
        const int64_t t = w / slices;
        const int c = (int)(w - t * slices) * kColumns + lane * 8, left = a.hidden - c;
        if (left <= 0) continue;
        const int64_t id = load_int(a.ids, t, a.ids64);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = id < 0 ? 0.0f : __builtin_nanf("");
        if (id >= 0 && id < a.vocab) {
            load_floats((const T *)a.table.data + id * a.table.stride + c, left, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= a.scale;
        }
        store_floats((R *)a.rows.data + t * a.rows.stride + c, left, v);
    }
}

// A row of the table's gradient: eight columns of it.
template <typename T, bool ONCE>
__device__ __forceinline__ void put_row(const EmbedArgs &a, int64_t v, int c, int left, float *sum) {
    T *out = (T *)a.table.data + v * a.table.stride + c;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] *= a.scale;
    if (a.accumulate) {
        float x[8];
        load_floats(out, left, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += x[k];
    }
    store_floats<ONCE>(out, left, sum);
}

// A block takes 512 columns of a piece's places, a wave of it 16 of them.  The sum of a
// run that goes on behind a wave's places stays with the wave it began in, and the others
// leave theirs for it to add.
template <typename T, typename R, bool ONCE>
__device__ __forceinline__ void add_piece(const EmbedArgs &a, int64_t piece, int c, float (*heads)[8][64]) {
    constexpr int kAhead = 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), left = a.hidden - c;
    const int64_t p0 = piece * kPiece + wave * kWavePlaces, n = a.tokens;
    // lane l has the wave's l-th place
    const bool on = lane < kWavePlaces && p0 + lane < n;
    const int32_t my_key = on ? a.key[p0 + lane] : a.vocab, my_entry = on ? a.order[p0 + lane] : 0;
    auto key_at = [&](int64_t p) { return p < n ? a.key[p] : a.vocab; };
    const int32_t key_before = p0 > 0 ? key_at(p0 - 1) : -1, key_after = key_at(p0 + kWavePlaces);
    // keys are in order, those of no row of the table last
    const int count = __popcll(__ballot(my_key < a.vocab));
    float sum[8] = {};
    bool first = true;   // the wave's first run
    int32_t going = -1;  // the id whose run it adds up behind its own places
    Eight<R> x[kAhead];
    auto fetch = [&](int i) __attribute__((always_inline)) {
        const int64_t t = __builtin_amdgcn_readlane(my_entry, i & 63);
        return load_eight<ONCE>((const R *)a.rows.data + t * a.rows.stride + c, i < count ? left : 0);
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = fetch(u);
    for (int i = 0; i < count; i += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= count) break;
            const int32_t id = __builtin_amdgcn_readlane(my_key, i + u);
            const bool ends = i + u + 1 == kWavePlaces,
                       last = i + u + 1 == count || __builtin_amdgcn_readlane(my_key, (i + u + 1) & 63) != id;
            float v[8];
            x[u].floats(v);
            x[u] = fetch(i + u + kAhead);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += v[k];
            if (!last) continue;
            const bool began = first && key_before == id, goes_on = ends && key_after == id;
            if (began && wave > 0) {
#pragma unroll
                for (int k = 0; k < 8; ++k) heads[wave - 1][k][lane] = sum[k];
            } else if (goes_on) {
                going = id;  // and sum stays
                first = began;
                break;
            } else if (began) {
                store_floats(a.sums + (2 * piece) * a.hidden + c, left, sum);
            } else if (left > 0) {
                put_row<T, ONCE>(a, id, c, left, sum);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
            first = false;
        }
    }
    __syncthreads();
    if (going < 0) return;
    int w = wave + 1;
    for (; w < kPieceWaves && key_at(piece * kPiece + w * kWavePlaces) == going; ++w)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += heads[w - 1][k][lane];
    if (first)
        store_floats(a.sums + (2 * piece) * a.hidden + c, left, sum);
    else if (w == kPieceWaves && key_at((piece + 1) * kPiece) == going)
        store_floats(a.sums + (2 * piece + 1) * a.hidden + c, left, sum);
    else if (left > 0)
        put_row<T, ONCE>(a, going, c, left, sum);
}

template <typename T, typename R, bool ONCE>
__global__ __launch_bounds__(64 * kPieceWaves) void k_embed_pieces(EmbedArgs a, int slices) {
    __shared__ float heads[kPieceWaves - 1][8][64];
    for (int64_t w = blockIdx.x; w < pieces_of(a) * slices; w += gridDim.x) {
        const int64_t piece = w / slices;
        __syncthreads();
        add_piece<T, R, ONCE>(a, piece, (int)(w - piece * slices) * kColumns + (threadIdx.x & 63) * 8, heads);
    }
}

// The first place whose key is v or more.
__device__ __forceinline__ int64_t lower_bound(const EmbedArgs &a, int64_t v) {
    int64_t lo = 0, hi = a.tokens;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (a.key[mid] < v)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

// What the pieces have not written: rows of no token, and of runs over several pieces.
// A block takes ROWS rows, whose 16-byte parts its threads walk one after the other
// (a wave to a row: 318 us for the call's 309 below).  Zeros are stored plainly, which is
// quicker than with the non-temporal hint (321).
constexpr int kTableThreads = 256;
template <typename T, int ROWS, bool ONCE>
__global__ __launch_bounds__(kTableThreads) void k_embed_table(EmbedArgs a) {
    constexpr int kPer = 16 / (int)sizeof(T), kAhead = 4;
    __shared__ int32_t first[ROWS + 1];
    const int parts = (a.hidden - 1) / kPer + 1;
    for (int64_t v0 = (int64_t)blockIdx.x * ROWS; v0 < a.vocab; v0 += (int64_t)gridDim.x * ROWS) {
        const int rows = (int)min((int64_t)ROWS, a.vocab - v0);
        __syncthreads();
        for (int r = threadIdx.x; r <= rows; r += kTableThreads) first[r] = (int32_t)lower_bound(a, v0 + r);
        __syncthreads();
        int row = threadIdx.x / parts, part = threadIdx.x - row * parts;
        const int more_rows = kTableThreads / parts, more_parts = kTableThreads - more_rows * parts;
        for (; row < rows; row += more_rows, part += more_parts) {
            if (part >= parts) {
                part -= parts;
                if (++row >= rows) break;
            }
            const int p0 = first[row], p1 = first[row + 1], r0 = p0 / kPiece, r1 = (p1 - 1) / kPiece;
            if (p0 == p1 ? a.accumulate : r0 == r1) continue;
            const int c = part * kPer, left = min(a.hidden - c, kPer);
            T *out = (T *)a.table.data + (v0 + row) * a.table.stride + c;
            if (p0 == p1) {
                if (left == kPer)
                    store_any16<false>(out, u32x4{0, 0, 0, 0});
                else
                    for (int k = 0; k < left; ++k) out[k] = 0;
                continue;
            }
            float sum[8] = {};
            for (int r = r0; r <= r1; r += kAhead) {
                float x[kAhead][8];
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    // in its first piece the run comes last
                    load_floats(a.sums + (2 * (int64_t)min(r + u, r1) + (r + u == r0 ? 1 : 0)) * a.hidden + c, left,
                                x[u]);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] += r + u <= r1 ? x[u][k] : 0.0f;
            }
            put_row<T, ONCE>(a, v0 + row, c, left, sum);
        }
    }
}

uint32_t grid_of(int64_t waves) { return (uint32_t)std::min<int64_t>((waves + kWaves - 1) / kWaves, 1 << 20); }
int slices_of(const EmbedArgs &a) { return a.hidden / kColumns + (a.hidden % kColumns != 0); }

// Keys are 0..vocab; each pass sorts by up to kMostBits of them.
constexpr int kMostBits = 11;
int key_bits(const EmbedArgs &a) {
    int b = 1;
    while ((int64_t)1 << b <= a.vocab) ++b;
    return b;
}
SortArgs sort_args(const EmbedArgs &a) {
    const int passes = (key_bits(a) + kMostBits - 1) / kMostBits;
    SortArgs s{};
    s.keys = a.ids;
    s.keys64 = a.ids64;
    s.limit = a.vocab;
    s.n = a.tokens;
    s.bits = (key_bits(a) + passes - 1) / passes;
    s.digits = 1 << s.bits;
    s.apart = true;
    sort_split(s);
    s.counts_stride = s.digits;
    return s;
}

}  // namespace

// The workspace's size and, with its address, where in it each part lies.
size_t embed_workspace(EmbedArgs &a, char *space) {
    size_t at = 0;
    auto part = [&](size_t bytes) {
        char *p = space + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    const SortArgs s = sort_args(a);
    for (int32_t **p : {&a.order, &a.order_spare, &a.key, &a.key_spare}) *p = (int32_t *)part((size_t)a.tokens * 4);
    a.counts = sort_needs_counts(s) ? (int32_t *)part((size_t)s.blocks * s.digits * 4) : nullptr;
    a.sums = (float *)part((size_t)pieces_of(a) * 2 * a.hidden * 4);
    return at + 256;
}

hipError_t launch_embed(const EmbedArgs &a, bool table_bf16, bool rows_bf16, hipStream_t s) {
    const int slices = slices_of(a);
    if (a.tokens * slices == 0) return hipSuccess;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid_of(a.tokens * slices)), dim3(64 * kWaves), 0, s, a, slices);
    };
    if (table_bf16)
        rows_bf16 ? go(k_embed<uint16_t, uint16_t>) : go(k_embed<uint16_t, float>);
    else
        rows_bf16 ? go(k_embed<float, uint16_t>) : go(k_embed<float, float>);
    return hipGetLastError();
}

hipError_t launch_embed_backward(const EmbedArgs &args, bool table_bf16, bool rows_bf16, hipStream_t s) {
    EmbedArgs a = args;
    const int slices = slices_of(a);
    SortArgs sort = sort_args(a);
    sort.counts = a.counts;
    const int bits = key_bits(a);
    for (int shift = 0; shift < bits && a.tokens > 0; shift += sort.bits) {
        sort.shift = shift;
        if (shift) sort.keys = a.key, sort.keys64 = 0, sort.order_in = a.order;
        sort.order_out = a.order_spare;
        sort.keys_out = a.key_spare;
        const hipError_t e = launch_sort(sort, s);
        if (e != hipSuccess) return e;
        std::swap(a.order, a.order_spare);
        std::swap(a.key, a.key_spare);
    }
    // past the last-level cache
    const bool once = a.tokens * a.hidden * (rows_bf16 ? 2 : 4) +
                          (a.accumulate ? 0 : (int64_t)a.vocab * a.hidden * (table_bf16 ? 2 : 4)) >
                      (int64_t)256 << 20;
    if (a.tokens > 0) {
        const dim3 grid((uint32_t)std::min<int64_t>(pieces_of(a) * slices, 1 << 20));
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * kPieceWaves), 0, s, a, slices); };
        auto pick = [&](auto is_once) {
            constexpr bool O = decltype(is_once)::value;
            if (table_bf16)
                rows_bf16 ? go(k_embed_pieces<uint16_t, uint16_t, O>) : go(k_embed_pieces<uint16_t, float, O>);
            else
                rows_bf16 ? go(k_embed_pieces<float, uint16_t, O>) : go(k_embed_pieces<float, float, O>);
        };
        once ? pick(std::true_type()) : pick(std::false_type());
    }
    auto table = [&](auto rows) {
        constexpr int ROWS = decltype(rows)::value;
        const dim3 grid((uint32_t)std::min<int64_t>(((int64_t)a.vocab + ROWS - 1) / ROWS, 1 << 20));
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kTableThreads), 0, s, a); };
        if (table_bf16)
            once ? go(k_embed_table<uint16_t, ROWS, true>) : go(k_embed_table<uint16_t, ROWS, false>);
        else
            once ? go(k_embed_table<float, ROWS, true>) : go(k_embed_table<float, ROWS, false>);
    };
    // rows of a block: few, so that blocks at work write close together, but enough of short
    // rows that finding them costs little (151,936 rows of 8 KB: 309 us in fours, 348 in 32s;
    // of 1.3 KB 123 and 94)
    if ((int64_t)a.hidden * (table_bf16 ? 2 : 4) > 1536)
        table(std::integral_constant<int, 4>());
    else
        table(std::integral_constant<int, 64>());
    return hipGetLastError();
}

}  // namespace sdpops
