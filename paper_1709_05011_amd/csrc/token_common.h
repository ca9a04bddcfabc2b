// Shared by the kernels of a token model's output side (rmsnorm.hip, token_logprob.hip, adamw.hip): accesses of eight elements at any
// element's alignment, sums and maxima over a wave and a block.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace {

// Global accesses of 16 bytes need no alignment beyond the element's on gfx950 (the unaligned access mode that HSA code objects run in).
template <typename T>
struct Packed;      // eight elements as loaded
template <>
struct Packed<float> {
    lc_u32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        __builtin_memcpy(&a, p, 16);
        __builtin_memcpy(&b, p + 4, 16);
    }
    __device__ __forceinline__ void load_some(const float* p, int n, uint32_t fill = 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = j < n ? __float_as_uint(p[j]) : fill;
            b[j] = j + 4 < n ? __float_as_uint(p[j + 4]) : fill;
        }
    }
    __device__ __forceinline__ float get(int j) const { return __uint_as_float(j < 4 ? a[j] : b[j - 4]); }
};
template <>
struct Packed<uint16_t> {
    lc_u32x4 a;
    __device__ __forceinline__ void load(const uint16_t* p) { __builtin_memcpy(&a, p, 16); }
    __device__ __forceinline__ void load_some(const uint16_t* p, int n, uint32_t fill = 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            a[j] = (2 * j < n ? (uint32_t)p[2 * j] : fill) | (2 * j + 1 < n ? (uint32_t)p[2 * j + 1] : fill) << 16;
    }
    __device__ __forceinline__ float get(int j) const { return __uint_as_float(j & 1 ? a[j >> 1] & 0xffff0000u : a[j >> 1] << 16); }
};

// Columns col .. col + 7 of a row of c; what lies past its end is `fill` (the type's own bit pattern).
template <typename T>
__device__ __forceinline__ void lc_load8(Packed<T>& to, const T* row, int col, int c, uint32_t fill = 0) {
    if (col + 8 <= c) to.load(row + col);
    else to.load_some(row + col, c - col, fill);
}

// Eight results, rounded once.
__device__ __forceinline__ void lc_store8(float* p, const float* v, int n) {
    if (n >= 8) {
        const lc_u32x4 a = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        const lc_u32x4 b = {__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
        __builtin_memcpy(p, &a, 16);
        __builtin_memcpy(p + 4, &b, 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = v[j];
    }
}
__device__ __forceinline__ void lc_store8(uint16_t* p, const float* v, int n) {
    if (n >= 8) {
        const lc_u32x4 a = {lc_bf16x2_rne(v[0], v[1]), lc_bf16x2_rne(v[2], v[3]), lc_bf16x2_rne(v[4], v[5]), lc_bf16x2_rne(v[6], v[7])};
        __builtin_memcpy(p, &a, 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = lc_bf16_rne(v[j]);
    }
}

// What a value is after it has been stored as T.
template <typename T>
__device__ __forceinline__ float lc_as_stored(float x) {
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)lc_bf16_rne(x) << 16);
    else return x;
}

__device__ __forceinline__ float lc_wave_sum(float x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}
__device__ __forceinline__ float lc_wave_max(float x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
    return x;
}
// Over a block of WAVES waves, every thread with the result; `red` (WAVES floats) must not be in use by an earlier call that a slower wave may still read.
template <int WAVES>
__device__ __forceinline__ float lc_block_sum(float x, float* red) {
    x = lc_wave_sum(x);
    if constexpr (WAVES == 1) return x;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = red[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += red[w];
    return s;
}
template <int WAVES>
__device__ __forceinline__ float lc_block_max(float x, float* red) {
    x = lc_wave_max(x);
    if constexpr (WAVES == 1) return x;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = red[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s = fmaxf(s, red[w]);
    return s;
}

inline bool lc_off_element(const void* p, size_t element) { return (reinterpret_cast<uintptr_t>(p) & (element - 1)) != 0; }

}  // namespace
