// Device helpers of the training operators around the experts' products: 16
// bytes of a row at a time, wherever the row starts.
#pragma once

#include "sdp_ops_device.h"

namespace sdpops {

// A row starts wherever its stride puts it, so 16-byte accesses are only aligned
// to an element.
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

// ONCE: with the non-temporal hint.
template <bool ONCE>
__device__ __forceinline__ u32x4 load_any16(const void *p) {
    return ONCE ? __builtin_nontemporal_load((const u32x4_any *)p) : *(const u32x4_any *)p;
}
template <bool ONCE>
__device__ __forceinline__ void store_any16(void *p, u32x4 v) {
    if (ONCE)
        __builtin_nontemporal_store(v, (u32x4_any *)p);
    else
        *(u32x4_any *)p = v;
}

// Eight elements of a row as they are stored.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    u32x4 raw;
    __device__ __forceinline__ void clear() { raw = u32x4{0, 0, 0, 0}; }
    template <bool ONCE = false>
    __device__ __forceinline__ void load(const uint16_t *p) { raw = load_any16<ONCE>(p); }
    // the first n, zeros behind them
    __device__ __forceinline__ void load_part(const uint16_t *p, int n) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t u = 0;
            if (2 * k < n) u = p[2 * k];
            if (2 * k + 1 < n) u |= (uint32_t)p[2 * k + 1] << 16;
            raw[k] = u;
        }
    }
    __device__ __forceinline__ void floats(float *v) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[2 * k] = bf16_lo(raw[k]), v[2 * k + 1] = bf16_hi(raw[k]);
    }
    __device__ __forceinline__ void set(const float *v) {
#pragma unroll
        for (int k = 0; k < 4; ++k) raw[k] = pack2(v[2 * k], v[2 * k + 1]);
    }
    // The compiler is not to keep floats of the piece past here.
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(raw)); }
    template <bool ONCE = false>
    __device__ __forceinline__ void store(uint16_t *p) const { store_any16<ONCE>(p, raw); }
};
template <>
struct Eight<float> {
    u32x4 a, b;
    __device__ __forceinline__ void clear() { a = b = u32x4{0, 0, 0, 0}; }
    template <bool ONCE = false>
    __device__ __forceinline__ void load(const float *p) { a = load_any16<ONCE>(p), b = load_any16<ONCE>(p + 4); }
    __device__ __forceinline__ void load_part(const float *p, int n) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a[k] = k < n ? __float_as_uint(p[k]) : 0;
            b[k] = 4 + k < n ? __float_as_uint(p[4 + k]) : 0;
        }
    }
    __device__ __forceinline__ void floats(float *v) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(a[k]), v[4 + k] = __uint_as_float(b[k]);
    }
    __device__ __forceinline__ void set(const float *v) {
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = __float_as_uint(v[k]), b[k] = __float_as_uint(v[4 + k]);
    }
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(a), "+v"(b)); }
    template <bool ONCE = false>
    __device__ __forceinline__ void store(float *p) const { store_any16<ONCE>(p, a), store_any16<ONCE>(p + 4, b); }
};

// n (any number) elements from p on, zeros where there are fewer than 8.
template <bool ONCE, typename T>
__device__ __forceinline__ Eight<T> load_eight(const T *p, int n) {
    Eight<T> e;
    if (n >= 8)
        e.template load<ONCE>(p);
    else
        e.load_part(p, n);
    return e;
}
template <bool ONCE = false, typename T>
__device__ __forceinline__ void load_floats(const T *p, int n, float *v) {
    load_eight<ONCE>(p, n).floats(v);
}
template <bool ONCE = false, typename T>
__device__ __forceinline__ void store_floats(T *p, int n, const float *v) {
    if (n >= 8) {
        Eight<T> e;
        e.set(v);
        e.template store<ONCE>(p);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) store1(p + k, v[k]);
}

// ---- sums over lanes -------------------------------------------------------------

template <int CONTROL>
__device__ __forceinline__ float lanes_of(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CONTROL, 0xf, 0xf, true));
}

// The sum over each aligned run of `lanes` lanes (8, 16, 32 or 64), in every one of
// them: neighbours by data-parallel moves, which need no trip through LDS.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
    v += lanes_of<0xb1>(v);   // the other one of each pair
    v += lanes_of<0x4e>(v);   // the other pair of each four
    v += lanes_of<0x141>(v);  // eight lanes mirrored
    if (lanes > 8) v += lanes_of<0x140>(v);  // 16 lanes mirrored
    if (lanes > 16) v += __shfl_xor(v, 16);
    if (lanes > 32) v += __shfl_xor(v, 32);
    return v;
}

// The largest value of such a run.
__device__ __forceinline__ float lanes_max(float v, int lanes) {
    v = fmaxf(v, lanes_of<0xb1>(v));
    v = fmaxf(v, lanes_of<0x4e>(v));
    v = fmaxf(v, lanes_of<0x141>(v));
    if (lanes > 8) v = fmaxf(v, lanes_of<0x140>(v));
    if (lanes > 16) v = fmaxf(v, __shfl_xor(v, 16));
    if (lanes > 32) v = fmaxf(v, __shfl_xor(v, 32));
    return v;
}

}  // namespace sdpops
