// Device helpers shared by the training operators' kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace sdpops {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// Two floats rounded to BF16, nearest even: one conversion instruction on gfx950.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

template <typename T>
__device__ __forceinline__ float load1(const T *p);
template <>
__device__ __forceinline__ float load1<float>(const float *p) { return *p; }
template <>
__device__ __forceinline__ float load1<uint16_t>(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }

__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t *p, float v) { *p = (uint16_t)pack2(v, 0.0f); }

// Element i of an FP32 or BF16 array.
__device__ __forceinline__ float load_either(const void *p, int64_t i, int bf16) {
    return bf16 ? load1((const uint16_t *)p + i) : ((const float *)p)[i];
}

// Element i of an array of 32- or 64-bit integers.
__device__ __forceinline__ int64_t load_int(const void *p, int64_t i, int is64) {
    return is64 ? ((const int64_t *)p)[i] : (int64_t)((const int32_t *)p)[i];
}

__device__ __forceinline__ float wave_sum(float v) {
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

__device__ __forceinline__ float wave_max(float v) {
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

}  // namespace sdpops
