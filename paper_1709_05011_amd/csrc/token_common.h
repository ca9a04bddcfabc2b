// Shared by the kernels of a token model (embedding.hip, rmsnorm.hip, layernorm.hip, token_logprob.hip, adamw.hip, newton_schulz.hip): accesses of eight elements at any
// element's alignment, sums and maxima over a wave and a block.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "internal.h"

namespace {

// 16 bytes at any element's alignment, past the caches' usual keeping with NT.
typedef lc_u32x4 lc_u32x4_any __attribute__((aligned(2)));
template <bool NT = false>
__device__ __forceinline__ lc_u32x4 lc_load16(const void* p) {
    if constexpr (NT) return __builtin_nontemporal_load(static_cast<const lc_u32x4_any*>(p));
    else return *static_cast<const lc_u32x4_any*>(p);
}
template <bool NT = false>
__device__ __forceinline__ void lc_store16(void* p, const lc_u32x4& v) {
    if constexpr (NT) __builtin_nontemporal_store(v, static_cast<lc_u32x4_any*>(p));
    else *static_cast<lc_u32x4_any*>(p) = v;
}

// Eight elements of a row as loaded.  Global accesses of 16 bytes need no alignment beyond the element's on gfx950 (the unaligned access mode that HSA code objects
// run in).  load_some(): the first n one by one, in a loop of few instructions (a short call's time goes by the code it has to fetch, too); shift(): drops the
// first k elements and fills up at the end.
template <typename T>
struct Packed;
template <>
struct Packed<float> {
    lc_u32x4 a, b;
    template <bool NT = false>
    __device__ __forceinline__ void load(const float* p) {
        a = lc_load16<NT>(p);
        b = lc_load16<NT>(p + 4);
    }
    __device__ __forceinline__ void load_some(const float* p, int n, uint32_t fill) {
        a = b = lc_u32x4{fill, fill, fill, fill};
#pragma unroll 1
        for (int j = min(n, 8) - 1; j >= 0; --j) {
            b = lc_u32x4{a[3], b[0], b[1], b[2]};
            a = lc_u32x4{__float_as_uint(p[j]), a[0], a[1], a[2]};
        }
    }
    __device__ __forceinline__ void shift(int k, uint32_t fill) {
        const lc_u32x4 f = {fill, fill, fill, fill};
        if (k >= 8) a = b = f;
        if (k & 4) {
            a = b;
            b = f;
        }
        if (k & 2) {
            a = lc_u32x4{a[2], a[3], b[0], b[1]};
            b = lc_u32x4{b[2], b[3], fill, fill};
        }
        if (k & 1) {
            a = lc_u32x4{a[1], a[2], a[3], b[0]};
            b = lc_u32x4{b[1], b[2], b[3], fill};
        }
    }
    __device__ __forceinline__ float get(int j) const { return __uint_as_float(j < 4 ? a[j] : b[j - 4]); }
};
template <>
struct Packed<uint16_t> {
    lc_u32x4 a;
    template <bool NT = false>
    __device__ __forceinline__ void load(const uint16_t* p) { a = lc_load16<NT>(p); }
    __device__ __forceinline__ void load_some(const uint16_t* p, int n, uint32_t fill) {
        const uint32_t f = fill | fill << 16;
        a = lc_u32x4{f, f, f, f};
#pragma unroll 1
        for (int j = min(n, 8) - 1; j >= 0; --j)
            a = lc_u32x4{a[0] << 16 | p[j], __builtin_amdgcn_alignbit(a[1], a[0], 16), __builtin_amdgcn_alignbit(a[2], a[1], 16),
                         __builtin_amdgcn_alignbit(a[3], a[2], 16)};
    }
    __device__ __forceinline__ void shift(int k, uint32_t fill) {
        const uint32_t f = fill | fill << 16;
        if (k >= 8) a = lc_u32x4{f, f, f, f};
        if (k & 4) a = lc_u32x4{a[2], a[3], f, f};
        if (k & 2) a = lc_u32x4{a[1], a[2], a[3], f};
        if (k & 1)
            a = lc_u32x4{__builtin_amdgcn_alignbit(a[1], a[0], 16), __builtin_amdgcn_alignbit(a[2], a[1], 16), __builtin_amdgcn_alignbit(a[3], a[2], 16),
                         __builtin_amdgcn_alignbit(f, a[3], 16)};
    }
    __device__ __forceinline__ float get(int j) const { return __uint_as_float(j & 1 ? a[j >> 1] & 0xffff0000u : a[j >> 1] << 16); }
};

// How a row's columns meet the threads that own eight of them each: kWhole: every thread's lie in the row; kEights: a thread's lie in it or past it, all of them; kAny.
enum Ends { kWhole, kEights, kAny };

// Columns col(i) .. col(i) + 7 of a row of c >= 8 for i < CH in two steps, so that all of a thread's loads are under way before the first is looked at:
// lc_issue8() loads the row's last eight columns in place of what would pass its end (no branch, nothing outside the row), lc_settle8() moves those to
// their places and puts `fill` (the type's own bits) where a column lies at `end` or past it; end is c, or a multiple of 8 before it.
template <Ends ENDS, bool NT = false, int CH, typename T, typename F>
__device__ __forceinline__ void lc_issue8(Packed<T> (&to)[CH], const T* row, F&& col, int c) {
#pragma unroll
    for (int i = 0; i < CH; ++i) to[i].template load<NT>(row + (ENDS == kWhole ? col(i) : min(col(i), c - 8)));
}
template <Ends ENDS, int CH, typename T, typename F>
__device__ __forceinline__ void lc_settle8(Packed<T> (&to)[CH], F&& col, int end, uint32_t fill = 0) {
    if constexpr (ENDS == kWhole) return;
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (end - col(i) < 8) to[i].shift(ENDS == kEights ? 8 : min(8 - (end - col(i)), 8), fill);
}
// The same where it depends on the place (full: the same for a wave; every column asked for lies before `end`), and for rows under eight columns, one thread's at
// most, which are read one by one.
template <bool NT = false, int CH, typename T, typename F>
__device__ __forceinline__ void lc_issue8(Packed<T> (&to)[CH], const T* row, F&& col, int c, bool full, uint32_t fill = 0) {
    if (full) {
        lc_issue8<kWhole, NT>(to, row, col, c);
    } else if (c >= 8) {
        lc_issue8<kAny, NT>(to, row, col, c);
    } else {
        to[0].load_some(row + col(0), c - col(0), fill);
#pragma unroll
        for (int i = 1; i < CH; ++i) to[i].shift(8, fill);
    }
}
template <int CH, typename T, typename F>
__device__ __forceinline__ void lc_settle8(Packed<T> (&to)[CH], F&& col, int c, int end, bool full, uint32_t fill = 0) {
    if (!full && c >= 8) lc_settle8<kAny>(to, col, end, fill);
}
template <bool NT = false, typename T>
__device__ __forceinline__ void lc_load8(Packed<T>& to, const T* row, int col, int c) {
    Packed<T> one[1];
    const auto column = [&](int) { return col; };
    lc_issue8<NT>(one, row, column, c, false);
    lc_settle8(one, column, c, c, false);
    to = one[0];
}

// The first n of eight results (none for n <= 0), rounded once.
template <bool NT = false>
__device__ __forceinline__ void lc_store8(float* p, const float* v, int n) {
    lc_u32x4 a = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    lc_u32x4 b = {__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
    if (n >= 8) {
        lc_store16<NT>(p, a);
        lc_store16<NT>(p + 4, b);
    } else {
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            p[j] = __uint_as_float(a[0]);
            a = lc_u32x4{a[1], a[2], a[3], b[0]};
            b = lc_u32x4{b[1], b[2], b[3], 0u};
        }
    }
}
template <bool NT = false>
__device__ __forceinline__ void lc_store8(uint16_t* p, const float* v, int n) {
    lc_u32x4 a = {lc_bf16x2_rne(v[0], v[1]), lc_bf16x2_rne(v[2], v[3]), lc_bf16x2_rne(v[4], v[5]), lc_bf16x2_rne(v[6], v[7])};
    if (n >= 8) {
        lc_store16<NT>(p, a);
    } else {
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            p[j] = (uint16_t)a[0];
            a = lc_u32x4{__builtin_amdgcn_alignbit(a[1], a[0], 16), __builtin_amdgcn_alignbit(a[2], a[1], 16), __builtin_amdgcn_alignbit(a[3], a[2], 16),
                         a[3] >> 16};
        }
    }
}

// What a value is after it has been stored as T.
template <typename T>
__device__ __forceinline__ float lc_as_stored(float x) {
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)lc_bf16_rne(x) << 16);
    else return x;
}

// Sum and maximum over a wave, every lane with the result: five exchanges inside the vector unit (neighbours, pairs, halves of 8 and of 16 lanes, a row's last lane to the
// next row, the first two rows' to the last two) and one lane read back as a scalar, where a shuffle through LDS takes some 100 cycles for each of six.  What a lane
// outside an exchange meets is the operation's neutral element: 0, or its own value.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t lc_dpp(uint32_t other, uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)other, (int)x, CTRL, ROWS, 0xf, false);
}
template <typename F>
__device__ __forceinline__ uint32_t lc_wave_join(uint32_t x, F&& step) {
    x = step(x, std::integral_constant<int, 0xB1>{}, std::integral_constant<int, 0xf>{});        // quad_perm 1 0 3 2
    x = step(x, std::integral_constant<int, 0x4E>{}, std::integral_constant<int, 0xf>{});        // quad_perm 2 3 0 1
    x = step(x, std::integral_constant<int, 0x141>{}, std::integral_constant<int, 0xf>{});       // row_half_mirror
    x = step(x, std::integral_constant<int, 0x140>{}, std::integral_constant<int, 0xf>{});       // row_mirror
    x = step(x, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});       // row_bcast:15 into rows 1 and 3
    x = step(x, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});       // row_bcast:31 into rows 2 and 3
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ float lc_wave_sum(float x) {
    return __uint_as_float(lc_wave_join(__float_as_uint(x), [](uint32_t a, auto ctrl, auto rows) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(lc_dpp<decltype(ctrl)::value, decltype(rows)::value>(0u, a)));
    }));
}
__device__ __forceinline__ float lc_wave_max(float x) {
    return __uint_as_float(lc_wave_join(__float_as_uint(x), [](uint32_t a, auto ctrl, auto rows) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(lc_dpp<decltype(ctrl)::value, decltype(rows)::value>(a, a))));
    }));
}
__device__ __forceinline__ uint32_t lc_wave_umax(uint32_t x) {
    return lc_wave_join(x, [](uint32_t a, auto ctrl, auto rows) {
        const uint32_t b = lc_dpp<decltype(ctrl)::value, decltype(rows)::value>(0u, a);
        return a > b ? a : b;
    });
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
