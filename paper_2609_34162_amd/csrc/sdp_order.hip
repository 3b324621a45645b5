// gfx950 kernels that sort entries by a small key, stably: sdp_expert_order, and
// the token ids of sdp_embed_backward digit by digit.
//
// A counting sort: an entry's place is the number of entries of lower digits, those of
// its own digit in earlier blocks, and those before it in its block.  A block walks its
// entries in steps, each of its waves 64 entries of a step at a time; lanes of the same
// digit find each other by one ballot for each bit of it, so the order of equals is
// kept.  Where only numbers are wanted, LDS counters are added to: integers, whose sum
// has no order.
// Two ways:
//  - one launch: every block counts all of the entries itself, those before its own
//    apart from the rest (8,192 tokens' 8 of 128 experts each: 16.7 us; 8 tokens' 3.8).
//  - three launches, for more entries: each block's counts, their running sums by one
//    block, the places (13.8 us; 524,288 entries of 256 experts 28).  The counts of a
//    block lie where its places will (or in a workspace), so that the call needs no
//    memory of its own; where they lie apart, the second launch is part of the third.
#include <algorithm>

#include "sdp_layer_internal.h"
#include "sdp_ops_device.h"

namespace sdpops {
namespace {

constexpr int kStep = 2048;  // entries of a block in a step, kSteps of each lane
// 16 waves, where the counts of so many find room in LDS
constexpr int kManyWaves = 16, kFewWaves = 8, kMostDigitsOfMany = 1024;

__device__ __forceinline__ int64_t entry_at(const SortArgs &a, int64_t i) { return a.order_in ? a.order_in[i] : i; }

__device__ __forceinline__ int32_t key_of(const SortArgs &a, int64_t k) {
    return k >= 0 && k < a.limit ? (int32_t)k : a.limit;
}

// The key at place i before the pass.
__device__ __forceinline__ int32_t key_at(const SortArgs &a, int64_t i) {
    return key_of(a, load_int(a.keys, i, a.keys64));
}

__device__ __forceinline__ int digit_of(const SortArgs &a, int32_t key) {
    return (key >> a.shift) & ((1 << a.bits) - 1);
}

// The digits of up to kStep entries from i0 on, and their ranks among the equals
// before them in their wave's part; wave_count[wave][digit] becomes the waves' counts.
template <int WAVES, int kSteps>
__device__ __forceinline__ void rank_step(const SortArgs &a, int64_t i0, int64_t i1, uint16_t *wave_count, int digits,
                                          int bits, int32_t *entry, int32_t *key, int *digit, int *rank) {
    constexpr int kThreads = 64 * WAVES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < WAVES * digits; d += kThreads) wave_count[d] = 0;
    __syncthreads();
    uint16_t *mine = wave_count + wave * digits;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const int64_t i = i0 + (wave * kSteps + u) * 64 + lane;
        const bool on = i < i1;
        entry[u] = on ? (int32_t)entry_at(a, i) : -1;
        key[u] = on ? key_at(a, i) : 0;
        digit[u] = on ? digit_of(a, key[u]) : 0;
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

// Adds a digit of each lane that is on to counters in LDS; one that a quarter of the
// wave shares, once for all of them.
__device__ __forceinline__ void count_digit(int32_t *counts, int digit, bool on) {
    int32_t *const mine = counts + digit;
    const uint32_t at = (uint32_t)(uintptr_t)mine, first = __builtin_amdgcn_readfirstlane(at);
    const uint64_t same = __ballot(on && at == first);
    const int shared = __popcll(same);
    if (shared >= 16) {
        if ((threadIdx.x & 63) == __builtin_ctzll(same)) atomicAdd(mine, shared);
        on = on && at != first;
    }
    if (on) atomicAdd(mine, 1);
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

// LDS of a block: counts of each wave, and three arrays of the digits'.
extern __shared__ char shared_memory[];
struct Shared {
    uint16_t *wave_count;
    int32_t *total, *base, *before;
};
__device__ __forceinline__ Shared shared_of(int digits) {
    const int even = (digits + 1) & ~1;
    Shared s;
    s.total = (int32_t *)shared_memory;
    s.base = s.total + even;
    s.before = s.base + even;
    s.wave_count = (uint16_t *)(s.before + even);
    return s;
}
size_t shared_bytes(int digits, int waves) { return (size_t)((digits + 1) & ~1) * (3 * 4 + waves * 2); }

// Adds the entries' digits in [i0, i1) to counts: to before's up to entry `until`, to
// total's from there on.  i0 and until are multiples of four; keys are read as 16 bytes,
// the next ones before these are counted.
template <int WAVES>
__device__ void count_range(const SortArgs &a, int64_t i0, int64_t until, int64_t i1, int32_t *before, int32_t *total) {
    constexpr int kThreads = 64 * WAVES, kAhead = 2;
    typedef __attribute__((ext_vector_type(2))) int64_t i64x2;
    typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
    const bool aligned = (uintptr_t)a.keys % 16 == 0;
    const int64_t whole = aligned ? i0 + (i1 - i0) / 4 * 4 : i0;
    i32x4 next[kAhead];
    auto fetch = [&](int64_t i) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t at = i + (u * kThreads + (int)threadIdx.x) * 4;
            next[u] = i32x4{-1, -1, -1, -1};
            if (at >= whole) continue;
            if (a.keys64) {
                const i64x2 lo = *(const i64x2 *)((const int64_t *)a.keys + at),
                            hi = *(const i64x2 *)((const int64_t *)a.keys + at + 2);
                next[u] = i32x4{key_of(a, lo[0]), key_of(a, lo[1]), key_of(a, hi[0]), key_of(a, hi[1])};
            } else {
                const i32x4 v = *(const i32x4 *)((const int32_t *)a.keys + at);
                next[u] = i32x4{key_of(a, v[0]), key_of(a, v[1]), key_of(a, v[2]), key_of(a, v[3])};
            }
        }
    };
    fetch(i0);
    for (int64_t i = i0; i < whole; i += kThreads * 4 * kAhead) {
        i32x4 key[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) key[u] = next[u];
        fetch(i + kThreads * 4 * kAhead);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            int32_t *const counts = i + (u * kThreads + (int)threadIdx.x) * 4 < until ? before : total;
#pragma unroll
            for (int k = 0; k < 4; ++k) count_digit(counts, key[u][k] < 0 ? 0 : digit_of(a, key[u][k]), key[u][k] >= 0);
        }
    }
    for (int64_t i = whole; i < i1; i += kThreads) {
        const int64_t at = i + threadIdx.x;
        count_digit(at < until ? before : total, at < i1 ? digit_of(a, key_at(a, at)) : 0, at < i1);
    }
}

// A step's counts of each wave to their offsets within the step, and their total.
template <int WAVES>
__device__ __forceinline__ void step_offsets(const Shared &s, int digits) {
    for (int d = threadIdx.x; d < digits; d += 64 * WAVES) {
        int sum = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int c = s.wave_count[w * digits + d];
            s.wave_count[w * digits + d] = (uint16_t)sum;
            sum += c;
        }
        s.total[d] = sum;
    }
}

template <int WAVES>
__device__ void place_range(const SortArgs &a, Range r, const Shared &s) {
    constexpr int kThreads = 64 * WAVES, kSteps = kStep / kThreads;
    const int digits = a.digits, bits = bits_of(digits), wave = threadIdx.x >> 6;
    for (int64_t i = r.i0; i < r.i1; i += kStep) {
        int32_t entry[kSteps], key[kSteps];
        int digit[kSteps], rank[kSteps];
        rank_step<WAVES, kSteps>(a, i, r.i1, s.wave_count, digits, bits, entry, key, digit, rank);
        step_offsets<WAVES>(s, digits);
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

template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_sort_count(SortArgs a) {
    constexpr int kThreads = 64 * WAVES;
    const Shared s = shared_of(a.digits);
    const Range r = range_of(a);
    for (int d = threadIdx.x; d < a.digits; d += kThreads) s.total[d] = 0;
    __syncthreads();
    count_range<WAVES>(a, r.i0, r.i0, r.i1, s.total, s.total);
    __syncthreads();
    for (int d = threadIdx.x; d < a.digits; d += kThreads) a.counts[blockIdx.x * a.counts_stride + d] = s.total[d];
}

// Each wave takes its share of the blocks' rows, lanes the digits 64 at a time: sums of the
// shares, their running sums, then the rows again.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_sort_scan(SortArgs a) {
    constexpr int kThreads = 64 * WAVES, kAhead = 8;
    __shared__ int32_t wave_sums[WAVES];
    const Shared s = shared_of(a.digits);
    int32_t *const part = (int32_t *)s.wave_count;  // [WAVES][digits]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int each = (a.blocks + WAVES - 1) / WAVES;
    const int b0 = min(wave * each, a.blocks), b1 = min(b0 + each, a.blocks);
    for (int d = lane; d < a.digits; d += 64) {
        const int32_t *const row = a.counts + d;
        int32_t sum = 0;
        for (int b = b0; b < b1; b += kAhead) {
            int32_t c[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) c[u] = b + u < b1 ? row[(b + u) * a.counts_stride] : 0;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) sum += c[u];
        }
        part[wave * a.digits + d] = sum;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < a.digits; d += kThreads) {
        int32_t sum = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int32_t c = part[w * a.digits + d];
            part[w * a.digits + d] = sum;
            sum += c;
        }
        s.total[d] = sum;
    }
    __syncthreads();
    scan_digits(s.total, s.base, a.digits, wave_sums);
    for (int d = threadIdx.x; d < a.digits; d += kThreads) put_end(a, d, s.base[d] + s.total[d]);
    for (int d = lane; d < a.digits; d += 64) {
        int32_t *const row = a.counts + d;
        int32_t at = s.base[d] + part[wave * a.digits + d];
        for (int b = b0; b < b1; b += kAhead) {
            int32_t c[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) c[u] = b + u < b1 ? row[(b + u) * a.counts_stride] : 0;
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (b + u < b1) {
                    row[(b + u) * a.counts_stride] = at;
                    at += c[u];
                }
        }
    }
}

// SCANS: the counts are still the blocks' own, and each block adds up what it needs of them.
template <int WAVES, bool SCANS>
__global__ __launch_bounds__(64 * WAVES) void k_sort_place(SortArgs a) {
    constexpr int kThreads = 64 * WAVES, kAhead = 8;
    __shared__ int32_t wave_sums[WAVES];
    const Shared s = shared_of(a.digits);
    const int32_t *const mine = a.counts + (int64_t)blockIdx.x * a.counts_stride;
    if (SCANS) {
        for (int d = threadIdx.x; d < a.digits; d += kThreads) {
            int32_t before = 0, all = 0;
            for (int b = 0; b < a.blocks; b += kAhead) {
                int32_t c[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    c[u] = b + u < a.blocks ? a.counts[(b + u) * a.counts_stride + d] : 0;
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    all += c[u];
                    before += b + u < (int)blockIdx.x ? c[u] : 0;
                }
            }
            s.total[d] = all, s.before[d] = before;
        }
        __syncthreads();
        scan_digits(s.total, s.base, a.digits, wave_sums);
        for (int d = threadIdx.x; d < a.digits; d += kThreads) {
            if (blockIdx.x == 0) put_end(a, d, s.base[d] + s.total[d]);
            s.base[d] += s.before[d];
        }
    } else {
        // all of the block's row is read before any of its places is written over it
        for (int d = threadIdx.x; d < a.digits; d += kThreads) s.base[d] = mine[d];
    }
    __syncthreads();
    place_range<WAVES>(a, range_of(a), s);
}

// One step's entries: their ranks are all the counting there is.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_sort_few(SortArgs a) {
    constexpr int kThreads = 64 * WAVES;
    __shared__ int32_t wave_sums[WAVES];
    const Shared s = shared_of(a.digits);
    const int digits = a.digits, wave = threadIdx.x >> 6;
    int32_t entry[2], key[2];
    int digit[2], rank[2];
    rank_step<WAVES, 2>(a, 0, a.n, s.wave_count, digits, bits_of(digits), entry, key, digit, rank);
    step_offsets<WAVES>(s, digits);
    __syncthreads();
    scan_digits(s.total, s.base, digits, wave_sums);
    for (int d = threadIdx.x; d < digits; d += kThreads) put_end(a, d, s.base[d] + s.total[d]);
#pragma unroll
    for (int u = 0; u < 2; ++u)
        if (entry[u] >= 0)
            put(a, (int64_t)s.base[digit[u]] + s.wave_count[wave * digits + digit[u]] + rank[u], entry[u], key[u]);
}

// Counts of all entries by every block.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_sort_one(SortArgs a) {
    constexpr int kThreads = 64 * WAVES;
    __shared__ int32_t wave_sums[kManyWaves];
    const Shared s = shared_of(a.digits);
    const Range r = range_of(a);
    for (int d = threadIdx.x; d < a.digits; d += kThreads) s.total[d] = s.before[d] = 0;
    __syncthreads();
    count_range<WAVES>(a, 0, r.i0, a.n, s.before, s.total);
    __syncthreads();
    for (int d = threadIdx.x; d < a.digits; d += kThreads) s.total[d] += s.before[d];
    __syncthreads();
    scan_digits(s.total, s.base, a.digits, wave_sums);
    for (int d = threadIdx.x; d < a.digits; d += kThreads) {
        if (blockIdx.x == 0) put_end(a, d, s.base[d] + s.total[d]);
        s.base[d] += s.before[d];
    }
    __syncthreads();
    place_range<WAVES>(a, r, s);
}

}  // namespace

// Up to how many entries every block counts all of them (128 experts: 32,768 entries
// 11.4 us, 65,536 16.7, in three launches 13.8; 2,048 experts: 65,536 entries 33 us, in
// three launches 51, as its scan finds room for four waves only).
constexpr int kMostScannedWide = 512;
int64_t most_counted_by_all(const SortArgs &a) { return (a.digits <= kMostScannedWide ? 40 : 128) << 10; }

void sort_split(SortArgs &a) {
    // a block has at least as many entries as there are digits
    int64_t chunk = kStep;
    while (chunk < a.digits) chunk += kStep;
    while (a.n / chunk > 1024) chunk *= 2;
    a.chunk = chunk;
    a.blocks = (int32_t)std::max<int64_t>(1, a.n / chunk);  // the last one has the rest
}

// Up to how many blocks of entries each adds up the counts itself, where they lie apart.
// (Embedding gradients of a table of 151,936: 12,000 tokens' take 64.2 us so and 62.4 where
// every block counts, 20,000 tokens' 64.9 and 67.0.)
constexpr int kMostScannedByAll = 64;
constexpr int64_t kMostCountedApart = 16 << 10;

bool sort_needs_counts(const SortArgs &a) { return a.n > (a.apart ? kMostCountedApart : most_counted_by_all(a)); }

hipError_t launch_sort(const SortArgs &a, hipStream_t s) {
    auto go = [&](auto kernel, int blocks, int waves) {
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * waves), shared_bytes(a.digits, waves), s, a);
    };
    const bool many = a.digits <= kMostDigitsOfMany;
    if (a.n <= 128 * 2) {
        go(k_sort_few<2>, 1, 2);
        return hipGetLastError();
    }
    if (a.n <= 128 * 8) {
        go(k_sort_few<8>, 1, 8);
        return hipGetLastError();
    }
    if (!sort_needs_counts(a)) {
        many ? go(k_sort_one<kManyWaves>, a.blocks, kManyWaves) : go(k_sort_one<kFewWaves>, a.blocks, kFewWaves);
        return hipGetLastError();
    }
    constexpr int kScanWaves = 4;  // where there are many digits
    many ? go(k_sort_count<kManyWaves>, a.blocks, kManyWaves) : go(k_sort_count<kFewWaves>, a.blocks, kFewWaves);
    if (a.apart && a.blocks <= kMostScannedByAll) {
        many ? go(k_sort_place<kManyWaves, true>, a.blocks, kManyWaves)
             : go(k_sort_place<kFewWaves, true>, a.blocks, kFewWaves);
        return hipGetLastError();
    }
    // (its sums have 32 bits, the steps' counts 16)
    auto scan = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, dim3(1), dim3(64 * waves), shared_bytes(a.digits, 2 * waves), s, a);
    };
    a.digits <= kMostScannedWide ? scan(k_sort_scan<kManyWaves>, kManyWaves)
                                 : scan(k_sort_scan<kScanWaves>, kScanWaves);
    many ? go(k_sort_place<kManyWaves, false>, a.blocks, kManyWaves)
         : go(k_sort_place<kFewWaves, false>, a.blocks, kFewWaves);
    return hipGetLastError();
}

}  // namespace sdpops
