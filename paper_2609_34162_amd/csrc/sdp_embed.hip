// gfx950 kernels of sdp_embed and its backward.
//
//   out[t] = s table[id_t];   dtable[v] = s sum over t with id_t = v of dout[t]
// Memory bounds both: the tokens' rows, and backward the whole table where it is
// written anew.  Backward the tokens are sorted by id (sdp_order.hip), so that each
// row of the table is one run of them, summed in the tokens' order and written once.
// Runs are cut at every 64th place: where one id fills all 64, their sum is made
// beforehand, by a wave of its own.
#include <algorithm>

#include "sdp_layer_device.h"
#include "sdp_layer_internal.h"

namespace sdpops {
namespace {

constexpr int kWaves = 4;
constexpr int kColumns = 512;  // of a wave: eight to a lane
constexpr int kTableRows = 64; // of a wave, backward

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

// Adds the rows of the tokens at places p0..p1 - 1.
template <typename R>
__device__ __forceinline__ void add_places(const EmbedArgs &a, int64_t p0, int64_t p1, int c, int left, float *sum) {
    for (int64_t p = p0; p < p1; ++p) {
        float v[8];
        load_floats((const R *)a.rows.data + (int64_t)a.order[p] * a.rows.stride + c, left, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += v[k];
    }
}

// The sums of aligned runs of places that one id fills.
template <typename R>
__global__ __launch_bounds__(64 * kWaves) void k_embed_runs(EmbedArgs a, int slices) {
    const int lane = threadIdx.x & 63;
    const int64_t runs = a.tokens / kEmbedRun;
    for (int64_t w = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); w < runs * slices;
         w += (int64_t)gridDim.x * kWaves) {
        const int64_t run = w / slices, p = run * kEmbedRun;
        const int c = (int)(w - run * slices) * kColumns + lane * 8, left = a.hidden - c;
        const int32_t id = a.key[p];
        if (id != a.key[p + kEmbedRun - 1] || id >= a.vocab || left <= 0) continue;
        float sum[8] = {};
        add_places<R>(a, p, p + kEmbedRun, c, left, sum);
        store_floats(a.runs + run * a.hidden + c, left, sum);
    }
}

// The first place whose key is v or more.
__device__ __forceinline__ int64_t lower_bound(const EmbedArgs &a, int32_t v) {
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

template <typename T, typename R>
__global__ __launch_bounds__(64 * kWaves) void k_embed_table(EmbedArgs a, int slices) {
    const int lane = threadIdx.x & 63;
    const int64_t parts = ((int64_t)a.vocab + kTableRows - 1) / kTableRows;
    for (int64_t w = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); w < parts * slices;
         w += (int64_t)gridDim.x * kWaves) {
        const int64_t part = w / slices;
        const int c = (int)(w - part * slices) * kColumns + lane * 8, left = a.hidden - c;
        const int64_t v0 = part * kTableRows, v1 = v0 + kTableRows < a.vocab ? v0 + kTableRows : a.vocab;
        const int64_t mine = v0 + lane + 1;
        // lane l has the end of row v0 + l
        const int64_t end = lower_bound(a, (int32_t)(mine < v1 ? mine : v1));
        int64_t p0 = lower_bound(a, (int32_t)v0);
        for (int64_t v = v0; v < v1; ++v) {
            const int64_t p1 = __shfl(end, (int)(v - v0));
            if (left > 0 && (p1 > p0 || !a.accumulate)) {
                float sum[8] = {};
                const int64_t r0 = (p0 + kEmbedRun - 1) / kEmbedRun, r1 = p1 / kEmbedRun;
                if (r1 > r0) {
                    add_places<R>(a, p0, r0 * kEmbedRun, c, left, sum);
                    for (int64_t r = r0; r < r1; ++r) {
                        float x[8];
                        load_floats(a.runs + r * a.hidden + c, left, x);
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum[k] += x[k];
                    }
                    add_places<R>(a, r1 * kEmbedRun, p1, c, left, sum);
                } else {
                    add_places<R>(a, p0, p1, c, left, sum);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] *= a.scale;
                T *out = (T *)a.table.data + v * a.table.stride + c;
                if (a.accumulate) {
                    float x[8];
                    load_floats(out, left, x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] += x[k];
                }
                store_floats(out, left, sum);
            }
            p0 = p1;
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
    a.order = (int32_t *)part((size_t)a.tokens * 4);
    a.spare = (int32_t *)part((size_t)a.tokens * 4);
    a.key = (int32_t *)part((size_t)a.tokens * 4);
    a.counts = (int32_t *)part((size_t)s.blocks * s.digits * 4);
    a.runs = (float *)part((size_t)(a.tokens / kEmbedRun) * a.hidden * 4);
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
        sort.order_in = shift ? a.order : nullptr;
        sort.order_out = a.spare;
        sort.keys_out = shift + sort.bits >= bits ? a.key : nullptr;
        const hipError_t e = launch_sort(sort, s);
        if (e != hipSuccess) return e;
        std::swap(a.order, a.spare);
    }
    if (a.tokens >= kEmbedRun) {
        const dim3 grid(grid_of(a.tokens / kEmbedRun * slices));
        if (rows_bf16)
            hipLaunchKernelGGL((k_embed_runs<uint16_t>), grid, dim3(64 * kWaves), 0, s, a, slices);
        else
            hipLaunchKernelGGL((k_embed_runs<float>), grid, dim3(64 * kWaves), 0, s, a, slices);
    }
    const int64_t waves = ((int64_t)a.vocab + kTableRows - 1) / kTableRows * slices;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid_of(waves)), dim3(64 * kWaves), 0, s, a, slices);
    };
    if (table_bf16)
        rows_bf16 ? go(k_embed_table<uint16_t, uint16_t>) : go(k_embed_table<uint16_t, float>);
    else
        rows_bf16 ? go(k_embed_table<float, uint16_t>) : go(k_embed_table<float, float>);
    return hipGetLastError();
}

}  // namespace sdpops
