// Device helpers of the training operators around the experts' products: 16
// bytes of a row at a time, wherever the row starts.
#pragma once

#include "sdp_ops_device.h"

namespace sdpops {

// A row starts wherever its stride puts it, so 16-byte accesses are only aligned
// to an element.
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

// Eight elements of a row as they are stored.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    u32x4 raw;
    __device__ __forceinline__ void load(const uint16_t *p) { raw = *(const u32x4_any *)p; }
    __device__ __forceinline__ void floats(float *v) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[2 * k] = bf16_lo(raw[k]), v[2 * k + 1] = bf16_hi(raw[k]);
    }
    __device__ __forceinline__ void set(const float *v) {
#pragma unroll
        for (int k = 0; k < 4; ++k) raw[k] = pack2(v[2 * k], v[2 * k + 1]);
    }
    __device__ __forceinline__ void store(uint16_t *p) const { *(u32x4_any *)p = raw; }
};
template <>
struct Eight<float> {
    u32x4 a, b;
    __device__ __forceinline__ void load(const float *p) { a = *(const u32x4_any *)p, b = *(const u32x4_any *)(p + 4); }
    __device__ __forceinline__ void floats(float *v) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(a[k]), v[4 + k] = __uint_as_float(b[k]);
    }
    __device__ __forceinline__ void set(const float *v) {
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = __float_as_uint(v[k]), b[k] = __float_as_uint(v[4 + k]);
    }
    __device__ __forceinline__ void store(float *p) const { *(u32x4_any *)p = a, *(u32x4_any *)(p + 4) = b; }
};

// n (at most 8) elements from p on as floats, zeros behind them; and back.
template <typename T>
__device__ __forceinline__ void load_floats(const T *p, int n, float *v) {
    if (n >= 8) {
        Eight<T> e;
        e.load(p);
        e.floats(v);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < n ? load1(p + k) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_floats(T *p, int n, const float *v) {
    if (n >= 8) {
        Eight<T> e;
        e.set(v);
        e.store(p);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) store1(p + k, v[k]);
}

}  // namespace sdpops
