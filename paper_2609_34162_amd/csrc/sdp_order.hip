// gfx950 kernels that sort entries by a small key, stably: sdp_expert_order, and
// the token ids of sdp_embed_backward digit by digit.
//
// A counting sort: an entry's place is the number of entries of lower digits,
// those of its own digit in earlier blocks, and those before it in its block.
// A block walks its entries in steps, each of its waves 64 entries of a step at a
// time; lanes of the same digit find each other by one ballot for each bit of it, so
// the counts need no atomics and the order of equals is kept.
//   count: the digits of each block's entries
//   scan:  one block turns them into the first place of each block and digit
//   place: the blocks walk their entries again
// Few entries are one block's work in one launch.
#include <algorithm>

#include "sdp_layer_internal.h"
#include "sdp_ops_device.h"

namespace sdpops {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kSteps = 4;                        // entries of a lane in a step
constexpr int kStep = kThreads * kSteps;         // entries of a block in a step

__device__ __forceinline__ int64_t entry_at(const SortArgs &a, int64_t i) { return a.order_in ? a.order_in[i] : i; }

__device__ __forceinline__ int32_t key_of(const SortArgs &a, int64_t entry) {
    const int64_t k = load_int(a.keys, entry, a.keys64);
    return k >= 0 && k < a.limit ? (int32_t)k : a.limit;
}

// The digits of up to kStep entries from i0 on, and their ranks among the equals
// before them in their wave's part; wave_count[wave][digit] becomes the waves' counts.
__device__ __forceinline__ void rank_step(const SortArgs &a, int64_t i0, int64_t i1, uint16_t *wave_count, int digits,
                                          int bits, int32_t *entry, int32_t *key, int *digit, int *rank) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < kWaves * digits; d += kThreads) wave_count[d] = 0;
    __syncthreads();
    uint16_t *mine = wave_count + wave * digits;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const int64_t i = i0 + (wave * kSteps + u) * 64 + lane;
        const bool on = i < i1;
        entry[u] = on ? (int32_t)entry_at(a, i) : -1;
        key[u] = on ? key_of(a, entry[u]) : 0;
        digit[u] = on ? (key[u] >> a.shift) & ((1 << a.bits) - 1) : 0;
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const bool on = entry[u] >= 0;
        uint64_t same = __ballot(on);
        for (int b = 0; b < bits; ++b) {
            const bool set = digit[u] >> b & 1;
            const uint64_t with = __ballot(set);
            same &= set ? with : ~with;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        int base = 0;
        if (on) base = mine[digit[u]];
        rank[u] = base + before;
        // (the wave's own reads come first: one wave's LDS accesses stay in order)
        if (on && before == 0) mine[digit[u]] = (uint16_t)(base + __popcll(same));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
}

__device__ __forceinline__ void put(const SortArgs &a, int64_t p, int32_t entry, int32_t key) {
    const bool absent = key == a.limit;
    if (a.order_out) a.order_out[p] = absent && a.place ? -1 : entry;
    if (a.place) a.place[entry] = absent ? -1 - (int32_t)p : (int32_t)p;
    if (a.keys_out) a.keys_out[p] = key;
}

// Bits that tell `digits` digits apart.
__device__ __forceinline__ int bits_of(int digits) { return digits > 1 ? 32 - __clz(digits - 1) : 0; }

// first[d] = base + the counts of lower digits, over one block; total[d] the counts.
__device__ void scan_digits(const int32_t *total, int32_t *first, int digits, int32_t *wave_sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    // each thread a run of digits
    const int each = (digits + blockDim.x - 1) / blockDim.x, d0 = threadIdx.x * each;
    int32_t sum = 0;
    for (int k = 0; k < each; ++k) sum += d0 + k < digits ? total[d0 + k] : 0;
    int32_t up = sum;
    for (int s = 1; s < 64; s <<= 1) {
        const int32_t v = __shfl_up(up, s);
        up += lane >= s ? v : 0;
    }
    if (lane == 63) wave_sums[wave] = up;
    __syncthreads();
    int32_t at = up - sum;
    for (int w = 0; w < waves; ++w) at += w < wave ? wave_sums[w] : 0;
    for (int k = 0; k < each; ++k)
        if (d0 + k < digits) {
            const int32_t c = total[d0 + k];
            first[d0 + k] = at;
            at += c;
        }
    __syncthreads();
}

__device__ void put_end(const SortArgs &a, int d, int32_t end) {
    if (!a.ends || d >= a.limit) return;
    if (a.ends64)
        ((int64_t *)a.ends)[d] = end;
    else
        ((int32_t *)a.ends)[d] = end;
}

struct Range {
    int64_t i0, i1;
};
__device__ __forceinline__ Range range_of(const SortArgs &a) {
    const int64_t i0 = (int64_t)blockIdx.x * a.chunk;
    return {i0, (int)blockIdx.x == a.blocks - 1 ? a.n : i0 + a.chunk};
}

// LDS of a block: counts of each wave, and two arrays of the digits'.
extern __shared__ char shared_memory[];
struct Shared {
    uint16_t *wave_count;
    int32_t *total, *base;
};
__device__ __forceinline__ Shared shared_of(int digits) {
    const int even = (digits + 1) & ~1;
    Shared s;
    s.total = (int32_t *)shared_memory;
    s.base = s.total + even;
    s.wave_count = (uint16_t *)(s.base + even);
    return s;
}
size_t shared_bytes(int digits) { return (size_t)((digits + 1) & ~1) * (2 * 4 + kWaves * 2); }

__device__ void count_range(const SortArgs &a, Range r, const Shared &s) {
    const int digits = a.digits, bits = bits_of(digits);
    for (int d = threadIdx.x; d < digits; d += kThreads) s.total[d] = 0;
    for (int64_t i = r.i0; i < r.i1; i += kStep) {
        int32_t entry[kSteps], key[kSteps];
        int digit[kSteps], rank[kSteps];
        rank_step(a, i, r.i1, s.wave_count, digits, bits, entry, key, digit, rank);
        for (int d = threadIdx.x; d < digits; d += kThreads)
            for (int w = 0; w < kWaves; ++w) s.total[d] += s.wave_count[w * digits + d];
        __syncthreads();
    }
}

__device__ void place_range(const SortArgs &a, Range r, const Shared &s) {
    const int digits = a.digits, bits = bits_of(digits), wave = threadIdx.x >> 6;
    for (int64_t i = r.i0; i < r.i1; i += kStep) {
        int32_t entry[kSteps], key[kSteps];
        int digit[kSteps], rank[kSteps];
        rank_step(a, i, r.i1, s.wave_count, digits, bits, entry, key, digit, rank);
        // counts of the waves to offsets within the step
        for (int d = threadIdx.x; d < digits; d += kThreads) {
            int sum = 0;
            for (int w = 0; w < kWaves; ++w) {
                const int c = s.wave_count[w * digits + d];
                s.wave_count[w * digits + d] = (uint16_t)sum;
                sum += c;
            }
            s.total[d] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            if (entry[u] >= 0)
                put(a, (int64_t)s.base[digit[u]] + s.wave_count[wave * digits + digit[u]] + rank[u], entry[u], key[u]);
        __syncthreads();
        for (int d = threadIdx.x; d < digits; d += kThreads) s.base[d] += s.total[d];
        __syncthreads();
    }
}

__global__ __launch_bounds__(kThreads) void k_sort_count(SortArgs a) {
    const Shared s = shared_of(a.digits);
    count_range(a, range_of(a), s);
    __syncthreads();
    for (int d = threadIdx.x; d < a.digits; d += kThreads) a.counts[blockIdx.x * a.counts_stride + d] = s.total[d];
}

__global__ __launch_bounds__(kThreads) void k_sort_scan(SortArgs a) {
    __shared__ int32_t wave_sums[kWaves];
    const Shared s = shared_of(a.digits);
    for (int d = threadIdx.x; d < a.digits; d += kThreads) {
        int32_t sum = 0;
        for (int b = 0; b < a.blocks; ++b) sum += a.counts[b * a.counts_stride + d];
        s.total[d] = sum;
    }
    __syncthreads();
    scan_digits(s.total, s.base, a.digits, wave_sums);
    for (int d = threadIdx.x; d < a.digits; d += kThreads) {
        int32_t at = s.base[d];
        put_end(a, d, at + s.total[d]);
        for (int b = 0; b < a.blocks; ++b) {
            const int32_t c = a.counts[b * a.counts_stride + d];
            a.counts[b * a.counts_stride + d] = at;
            at += c;
        }
    }
}

__global__ __launch_bounds__(kThreads) void k_sort_place(SortArgs a) {
    const Shared s = shared_of(a.digits);
    // all of the block's row is read before any of its places is written over it
    for (int d = threadIdx.x; d < a.digits; d += kThreads) s.base[d] = a.counts[blockIdx.x * a.counts_stride + d];
    __syncthreads();
    place_range(a, range_of(a), s);
}

__global__ __launch_bounds__(kThreads) void k_sort_one(SortArgs a) {
    __shared__ int32_t wave_sums[kWaves];
    const Shared s = shared_of(a.digits);
    const Range r{0, a.n};
    count_range(a, r, s);
    __syncthreads();
    scan_digits(s.total, s.base, a.digits, wave_sums);
    for (int d = threadIdx.x; d < a.digits; d += kThreads) put_end(a, d, s.base[d] + s.total[d]);
    __syncthreads();
    place_range(a, r, s);
}

}  // namespace

void sort_split(SortArgs &a) {
    // a block has at least as many entries as there are digits
    int64_t chunk = kStep;
    while (chunk < a.digits) chunk += kStep;
    while (a.n / chunk > 1024) chunk *= 2;
    a.chunk = chunk;
    a.blocks = (int32_t)std::max<int64_t>(1, a.n / chunk);  // the last one has the rest
}

hipError_t launch_sort(const SortArgs &a, hipStream_t s) {
    const size_t lds = shared_bytes(a.digits);
    if (a.blocks == 1) {
        hipLaunchKernelGGL(k_sort_one, dim3(1), dim3(kThreads), lds, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(k_sort_count, dim3(a.blocks), dim3(kThreads), lds, s, a);
    hipLaunchKernelGGL(k_sort_scan, dim3(1), dim3(kThreads), lds, s, a);
    hipLaunchKernelGGL(k_sort_place, dim3(a.blocks), dim3(kThreads), lds, s, a);
    return hipGetLastError();
}

}  // namespace sdpops
