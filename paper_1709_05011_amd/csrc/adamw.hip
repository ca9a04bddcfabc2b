// AdamW over a list of tensors for gfx950: one streaming pass, states in fp32 or in 8 bits with a scale per 256 elements.
//
// m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  w <- w - lr decay w - lr (m / c1) / (sqrt(v) / sqrt(c2) + eps).  Bound by memory: 28 bytes a
// parameter with fp32 states and gradients (2 more with a bf16 copy of w, 2 fewer with bf16 gradients), 16.06 with 8-bit states, fp32 gradients and no copy.
// The list is cut into chunks of one tensor each; descriptors travel as launch arguments, and a wave finds the tensor of its chunk with
// one probe of their first chunks.  A wave owns 256 consecutive elements, four a lane: one block of the 8-bit states, whose new
// values, largest magnitudes and codes are made in registers between the loads and the stores.  25.6 million parameters in 161 tensors 118 us with the bf16 copies, 6.5 TB/s; 201 million
// with 8-bit states, bf16 gradients and copies 514 us, 6.3 TB/s; 19 million 8-bit ones with fp32 gradients 4 bytes off alignment 51 us, 6 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "token_common.h"

namespace {

constexpr int kPart = 256;                                       // elements of a wave, four a lane
constexpr int kTable = 176, kSmallTable = 24;                    // descriptors per launch: 13.4 KB of launch arguments, which a short list's call need not copy (4.4 us a call, so 3.3)
static_assert(kPart == ADAMW_Q8_BLOCK, "a wave makes a block's scale by itself");

struct AdamTensor {
    float* w;
    const void* g;
    void* m;
    void* v;
    float* m_scale;        // 8-bit states only
    float* v_scale;
    uint16_t* w_lowp;      // or null
    long long numel;
    float lr_decay;
};

struct AdamScalars {
    int chunks;
    const float* grad_scale;
    float b1, one_b1, b2, one_b2, step_size, inv_root_c2, eps;
    bool small_eps;
    uint32_t dither;
};

template <int TABLE>
struct AdamArgs {
    static constexpr int kStarts = (TABLE + 63) / 64 * 64;
    AdamTensor t[TABLE];
    int start[kStarts];    // first chunk of each, ascending; past the last the largest int
    AdamScalars s;
};

// 21 bits from an element's number: two rounds of shift and odd product (the golden ratio's and root two's bits) modulo 2^32.
__device__ __forceinline__ uint32_t dither21(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x9E3779B1u;
    x = (x ^ (x >> 15)) * 0x6A09E667u;
    return x >> 11;
}

// The exponent of the smallest power of two >= 2^-126 that brings the magnitude with these bits to 1.75 * 2^top at most (0 for zero).
__device__ __forceinline__ int scale_exponent(uint32_t bits, int top) {
    const int k = (int)(bits >> 23) - 127 - top + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return bits == 0 ? 0 : max(k, -126);
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// e5m2 of x in [0, 57344] rounded up with the probability that keeps the mean: the dither is added below the last place.  Above zero at least code 1.
__device__ __forceinline__ uint32_t e5m2_dithered(float x, uint32_t r) {
    const uint32_t b = __float_as_uint(x);
    const uint32_t code = x < 0x1p-14f ? ((uint32_t)(x * 0x1p37f) + r) >> 21 : ((b + r) >> 21) - (112u << 2);
    return x > 0.f ? max(code, 1u) : 0u;
}

__device__ __forceinline__ uint32_t finite_size(float x) { return fabsf(x) < INFINITY ? __float_as_uint(fabsf(x)) : 0u; }

// Four neighbouring elements at any element's alignment; n of them where FULL is not set (none for n <= 0; what is not read is 0).
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <bool NT, bool FULL>
__device__ __forceinline__ void load4(float* to, const float* p, int n) {
    lc_u32x4 x = {};
    if (FULL || n >= 4) x = lc_load16<NT>(p);
    else
        for (int j = 0; j < 4; ++j)
            if (j < n) x[j] = __float_as_uint(p[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) to[j] = __uint_as_float(x[j]);
}
template <bool NT, bool FULL>
__device__ __forceinline__ void load4(float* to, const uint16_t* p, int n) {
    u32x2 x = {};
    if (FULL || n >= 4) {
        if constexpr (NT) x = __builtin_nontemporal_load(reinterpret_cast<const u32x2_any*>(p));
        else x = *reinterpret_cast<const u32x2_any*>(p);
    } else {
        for (int j = 0; j < 4; ++j)
            if (j < n) x[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) to[j] = __uint_as_float(j & 1 ? x[j >> 1] & 0xffff0000u : x[j >> 1] << 16);
}
template <bool NT, bool FULL>
__device__ __forceinline__ uint32_t load4(const uint8_t* p, int n) {
    if (FULL || n >= 4) {
        if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const u32_any*>(p));
        else return *reinterpret_cast<const u32_any*>(p);
    }
    uint32_t x = 0;
    for (int j = 0; j < 4; ++j)
        if (j < n) x |= (uint32_t)p[j] << (8 * j);
    return x;
}
template <bool NT, bool FULL>
__device__ __forceinline__ void store4(float* p, const float* v, int n) {
    const lc_u32x4 x = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    if (FULL || n >= 4) lc_store16<NT>(p, x);
    else
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = v[j];
}
template <bool NT, bool FULL>
__device__ __forceinline__ void store4(uint16_t* p, const float* v, int n) {
    const u32x2 x = {lc_bf16x2_rne(v[0], v[1]), lc_bf16x2_rne(v[2], v[3])};
    if (FULL || n >= 4) {
        if constexpr (NT) __builtin_nontemporal_store(x, reinterpret_cast<u32x2_any*>(p));
        else *reinterpret_cast<u32x2_any*>(p) = x;
    } else {
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = (uint16_t)(x[j >> 1] >> (16 * (j & 1)));
    }
}
template <bool NT, bool FULL>
__device__ __forceinline__ void store4(uint8_t* p, uint32_t x, int n) {
    if (FULL || n >= 4) {
        if constexpr (NT) __builtin_nontemporal_store(x, reinterpret_cast<u32_any*>(p));
        else *reinterpret_cast<u32_any*>(p) = x;
    } else {
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = (uint8_t)(x >> (8 * j));
    }
}

// m / (sqrt(v) / root c2 + eps) by the instructions for roots and reciprocals, one unit in the last place each.  They take a number under 2^-126 for zero, which a root of 2^-63 beside an eps
// shows where eps is less than 2^25 of them (SMALL): scaled by powers of two then.
template <bool SMALL>
__device__ __forceinline__ float update_of(const AdamScalars& p, float m, float v) {
    if constexpr (!SMALL) return m * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v), p.inv_root_c2, p.eps));
    const bool low = v < 0x1p-96f;
    const float root = fmaf(__builtin_amdgcn_sqrtf(low ? v * 0x1p64f : v) * (low ? 0x1p-32f : 1.f), p.inv_root_c2, p.eps);
    return root < 0x1p-64f ? m * __builtin_amdgcn_rcpf(root * 0x1p64f) * 0x1p64f : m * __builtin_amdgcn_rcpf(root);
}

// What a wave does to its 256 elements, number `block` of the tensor; FULL: all of them lie within it (left: how many do).
template <typename G, bool Q8, int PAST, bool FULL>
__device__ __forceinline__ void adamw_part(const AdamScalars& p, const AdamTensor& t, long long block, long long left_in_block) {
#pragma clang fp contract(off)
    constexpr bool NT = PAST > 0;
    const int lane = threadIdx.x & 63, own = lane * 4;
    const int n = FULL ? 4 : (int)left_in_block - own;                // this lane's elements; none or fewer than none past the end
    const long long first = block * kPart;
    const float gs = p.grad_scale ? *p.grad_scale : 1.f;
    float w[4], g[4], m[4], v[4];
    load4<NT, FULL>(w, t.w + first + own, n);
    load4<NT, FULL>(g, static_cast<const G*>(t.g) + first + own, n);
    if constexpr (Q8) {
        const uint32_t cm = load4<NT, FULL>(static_cast<const uint8_t*>(t.m) + first + own, n);
        const uint32_t cv = load4<NT, FULL>(static_cast<const uint8_t*>(t.v) + first + own, n);
        const float ms = t.m_scale[block], vs = t.v_scale[block];
        const f32x2 m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm, false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm, true);
        const f32x2 v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)cv, false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)cv, true);
        m[0] = m0[0] * ms;
        m[1] = m0[1] * ms;
        m[2] = m1[0] * ms;
        m[3] = m1[1] * ms;
        v[0] = v0[0] * vs;
        v[1] = v0[1] * vs;
        v[2] = v1[0] * vs;
        v[3] = v1[1] * vs;
    } else {
        load4<NT, FULL>(m, static_cast<const float*>(t.m) + first + own, n);
        load4<NT, FULL>(v, static_cast<const float*>(t.v) + first + own, n);
    }
    // m and v by separately rounded products and sums (their bits are defined so)
    float update[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float x = g[j] * gs;
        m[j] = p.b1 * m[j] + p.one_b1 * x;
        v[j] = p.b2 * v[j] + p.one_b2 * (x * x);
        update[j] = update_of<false>(p, m[j], v[j]);
    }
    if (p.small_eps) {
#pragma unroll
        for (int j = 0; j < 4; ++j) update[j] = update_of<true>(p, m[j], v[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = fmaf(-p.step_size, update[j], fmaf(-t.lr_decay, w[j], w[j]));
    store4<NT, FULL>(t.w + first + own, w, n);
    if (t.w_lowp) store4<(PAST > 1), FULL>(t.w_lowp + first + own, w, n);
    if constexpr (!Q8) {
        store4<NT, FULL>(static_cast<float*>(t.m) + first + own, m, n);
        store4<NT, FULL>(static_cast<float*>(t.v) + first + own, v, n);
    } else {
        // the largest magnitudes as the unsigned numbers that their bits are: what is infinite or no number is above every other
        uint32_t am = 0, av = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            am = max(am, __float_as_uint(m[j]) & 0x7fffffffu);
            av = max(av, __float_as_uint(v[j]));
        }
        am = lc_wave_umax(am);
        av = lc_wave_umax(av);
        const bool odd = max(am, av) >= 0x7f800000u;                 // (the same for the wave)
        if (odd) {
            am = av = 0;
            for (int j = 0; j < 4; ++j) {
                am = max(am, finite_size(m[j]));
                av = max(av, finite_size(v[j]));
            }
            am = lc_wave_umax(am);
            av = lc_wave_umax(av);
        }
        const int km = scale_exponent(am, 8), kv = scale_exponent(av, 15);
        if (lane == 0) {
            t.m_scale[block] = power_of_two(km);
            t.v_scale[block] = power_of_two(kv);
        }
        const float im = power_of_two(-km), iv = power_of_two(-kv);
        int cm = 0;
        cm = __builtin_amdgcn_cvt_pk_fp8_f32(m[0] * im, m[1] * im, cm, false);
        cm = __builtin_amdgcn_cvt_pk_fp8_f32(m[2] * im, m[3] * im, cm, true);
        const uint32_t number = (uint32_t)first + (uint32_t)((unsigned long long)first >> 32) * 0x6A09E667u + p.dither + own;
        uint32_t code[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            code[j] = e5m2_dithered(v[j] * iv, dither21(number + j));
        }
        if (odd) {
#pragma unroll
            for (int j = 0; j < 4; ++j) code[j] = v[j] < INFINITY ? code[j] : 0x7fu;
        }
        store4<NT, FULL>(static_cast<uint8_t*>(t.m) + first + own, (uint32_t)cm, n);
        store4<NT, FULL>(static_cast<uint8_t*>(t.v) + first + own, code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24, n);
    }
}

// One vector a thread, so that the chip works on one narrow stretch of each array at a time.  PAST: accesses past the caches' usual keeping, for lists that the
// caches do not hold; 1: but for the bf16 copies, 2: all.  Blocks of one wave; of four where a tensor's arrays do not start on whole lines of 128 bytes: a line that two waves fill is then
// mostly filled within one unit's cache and not by two dies' (201 million parameters with 8-bit states 4 bytes off a line, us: waves by themselves 737, four 617; on it 540 and 580).
template <typename G, bool Q8, int PAST, int WAVES, int TABLE>
__global__ void __launch_bounds__(WAVES * 64) adamw_kernel(const AdamArgs<TABLE> args) {
    constexpr int kStarts = AdamArgs<TABLE>::kStarts;
    const AdamScalars& p = args.s;
    const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x) {
        int first[kStarts / 64], owner = -1;
#pragma unroll
        for (int i = 0; i < kStarts / 64; ++i) first[i] = args.start[64 * i + lane];
#pragma unroll
        for (int i = 0; i < kStarts / 64; ++i) owner += __popcll(__ballot(first[i] <= chunk));
        owner = __builtin_amdgcn_readfirstlane(owner);
        const AdamTensor t = args.t[owner];
        const long long block = (long long)(chunk - args.start[owner]) * WAVES + wave, left = t.numel - block * kPart;
        if (left >= kPart) adamw_part<G, Q8, PAST, true>(p, t, block, kPart);
        else if (left > 0) adamw_part<G, Q8, PAST, false>(p, t, block, left);
    }
}

constexpr int kMostWaves = 1 << 24;       // of a launch, which holds fewer than 2^32 threads; chunks beyond are dealt round

struct AdamList {                          // what both entry points take
    int n;
    float* const* w;
    const void* const* g;
    lc_dtype g_dtype;
    void* const* m;
    void* const* v;
    float* const* m_scale;                 // null: fp32 states
    float* const* v_scale;
    const int64_t* numel;
    float lr, weight_decay;
    double beta1, beta2;
    float eps;
    int64_t step;
    uint32_t seed;
    const float* weight_decay_per_tensor;
    const float* grad_scale;
    void* const* w_lowp;
};

long long chunks_of(int64_t numel, int waves) { return numel / (kPart * waves) + (numel % (kPart * waves) != 0); }

lc_status check_list(const AdamList& a, bool q8) {
    if (a.n < 0) return LC_ERR_SHAPE;
    if (a.g_dtype != LC_F32 && a.g_dtype != LC_BF16) return LC_ERR_UNSUPPORTED;
    if (!(a.beta1 >= 0.0 && a.beta1 < 1.0) || !(a.beta2 >= 0.0 && a.beta2 < 1.0) || !(a.eps > 0.f) || a.step < 1) return LC_ERR_UNSUPPORTED;
    if (a.n == 0) return LC_OK;
    if (!a.w || !a.g || !a.m || !a.v || !a.numel || (q8 && (!a.m_scale || !a.v_scale))) return LC_ERR_NULL;
    if (lc_off_element(a.grad_scale, 4)) return LC_ERR_ALIGN;
    for (int l = 0; l < a.n; ++l) {
        if (a.numel[l] < 0 || a.numel[l] > (int64_t)1 << 38) return LC_ERR_SHAPE;
        if (a.numel[l] == 0) continue;
        if (!a.w[l] || !a.g[l] || !a.m[l] || !a.v[l] || (q8 && (!a.m_scale[l] || !a.v_scale[l]))) return LC_ERR_NULL;
        if (lc_off_element(a.w[l], 4) || lc_off_element(a.g[l], a.g_dtype == LC_BF16 ? 2 : 4) || (a.w_lowp && lc_off_element(a.w_lowp[l], 2))) return LC_ERR_ALIGN;
        if (q8 ? lc_off_element(a.m_scale[l], 4) || lc_off_element(a.v_scale[l], 4) : lc_off_element(a.m[l], 4) || lc_off_element(a.v[l], 4)) return LC_ERR_ALIGN;
    }
    return LC_OK;
}

template <typename G, bool Q8, int PAST, int TABLE>
void launch(const AdamArgs<TABLE>& args, int waves, hipStream_t stream) {
    const dim3 grid((unsigned)std::min(args.s.chunks, kMostWaves / waves));
    if (waves == 1) hipLaunchKernelGGL((adamw_kernel<G, Q8, PAST, 1, TABLE>), grid, dim3(64), 0, stream, args);
    else hipLaunchKernelGGL((adamw_kernel<G, Q8, PAST, 4, TABLE>), grid, dim3(256), 0, stream, args);
}
template <typename G, bool Q8>
void launch(const AdamArgs<kTable>& args, int count, int waves, int past, hipStream_t stream) {
    if (past == 0 && count <= kSmallTable) {
        AdamArgs<kSmallTable> few;
        std::copy(args.t, args.t + kSmallTable, few.t);
        std::copy(args.start, args.start + few.kStarts, few.start);
        few.s = args.s;
        launch<G, Q8, 0>(few, waves, stream);
    } else if (past == 0) {
        launch<G, Q8, 0>(args, waves, stream);
    } else if (past == 1) {
        launch<G, Q8, 1>(args, waves, stream);
    } else {
        launch<G, Q8, 2>(args, waves, stream);
    }
}

// What a step reads and writes from which it goes past the caches.  Three lists in turn, us, ordinary / past: fp32 states, 5.9 million parameters (166 MB) 28.9 / 29.4, 7.1 (198 MB)
// 35.1 / 34.5, 9.6 (270 MB) 52.4 / 45.9; 8 bits, 6.3 million (101 MB) 20.1 / 20.7, 9.8 (157 MB) 30.3 / 29.6, 14.2 (226 MB) 44.6 / 41.2.
constexpr long long kStreamBytes = 160 << 20;

lc_status run_list(const AdamList& a, bool q8, void* hip_stream) {
    const lc_status st = check_list(a, q8);
    if (st != LC_OK || a.n == 0 || std::all_of(a.numel, a.numel + a.n, [](int64_t n) { return n == 0; })) return st;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    AdamArgs<kTable> args;
    AdamScalars& p = args.s;
    p.grad_scale = a.grad_scale;
    p.b1 = (float)a.beta1;
    p.one_b1 = (float)(1.0 - a.beta1);
    p.b2 = (float)a.beta2;
    p.one_b2 = (float)(1.0 - a.beta2);
    p.step_size = (float)((double)a.lr / (1.0 - std::pow(a.beta1, (double)a.step)));
    p.inv_root_c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(a.beta2, (double)a.step)));
    p.eps = a.eps;
    p.small_eps = a.eps < 0x1p-38f * p.inv_root_c2;
    p.dither = a.seed * 0x9E3779B1u + 0x7F4A7C15u;
    double all = 0.0;
    uintptr_t starts = 0;
    for (int l = 0; l < a.n; ++l) {
        if (a.numel[l] == 0) continue;
        all += (double)a.numel[l];
        starts |= (uintptr_t)a.w[l] | (uintptr_t)a.m[l] | (uintptr_t)a.v[l];
    }
    // (copies of 51 MB are worth more in the caches, to this call too: 120 us, past them 125; 170 MB 237 / 235, 402 MB 543 / 522)
    const int past = all * ((q8 ? 12 : 24) + (a.g_dtype == LC_BF16 ? 2 : 4)) < (double)kStreamBytes ? 0 : all * 2 < (double)kStreamBytes ? 1 : 2;
    const int waves = (starts & 127) == 0 ? 1 : 4;
    lc_begin_call();
    for (int l = 0; l < a.n;) {
        long long chunks = 0;
        int count = 0;
        for (; l < a.n && count < kTable; ++l) {
            if (a.numel[l] == 0) continue;
            const long long more = chunks_of(a.numel[l], waves);
            if (chunks + more > 0x7f000000ll) break;                   // a chunk's number and the grid beyond it stay in 31 bits (one tensor has 2^30 at most)
            AdamTensor& t = args.t[count];
            t.w = a.w[l];
            t.g = a.g[l];
            t.m = a.m[l];
            t.v = a.v[l];
            t.m_scale = q8 ? a.m_scale[l] : nullptr;
            t.v_scale = q8 ? a.v_scale[l] : nullptr;
            t.w_lowp = a.w_lowp ? static_cast<uint16_t*>(a.w_lowp[l]) : nullptr;
            t.numel = a.numel[l];
            t.lr_decay = (float)((double)a.lr * (a.weight_decay_per_tensor ? a.weight_decay_per_tensor[l] : a.weight_decay));
            args.start[count++] = (int)chunks;
            chunks += more;
        }
        if (count == 0) break;                                         // only empty tensors were left
        std::fill(args.start + count, args.start + args.kStarts, 0x7fffffff);
        p.chunks = (int)chunks;
        if (a.g_dtype == LC_BF16) q8 ? launch<uint16_t, true>(args, count, waves, past, stream) : launch<uint16_t, false>(args, count, waves, past, stream);
        else q8 ? launch<float, true>(args, count, waves, past, stream) : launch<float, false>(args, count, waves, past, stream);
    }
    return lc_end_call();
}

}  // namespace

extern "C" lc_status adamw_step(int n_tensors, float* const* w, const void* const* g, lc_dtype g_dtype, float* const* m, float* const* v,
                                const int64_t* numel, float lr, double beta1, double beta2, float eps, float weight_decay, int64_t step,
                                const float* weight_decay_per_tensor, const float* grad_scale, void* const* w_lowp_out, void* hip_stream) {
    const AdamList a{n_tensors, w, g, g_dtype, reinterpret_cast<void* const*>(m), reinterpret_cast<void* const*>(v), nullptr, nullptr, numel, lr,
                     weight_decay, beta1, beta2, eps, step, 0, weight_decay_per_tensor, grad_scale, w_lowp_out};
    return run_list(a, false, hip_stream);
}

extern "C" lc_status adamw_step_q8(int n_tensors, float* const* w, const void* const* g, lc_dtype g_dtype, uint8_t* const* m,
                                   float* const* m_scale, uint8_t* const* v, float* const* v_scale, const int64_t* numel, float lr, double beta1,
                                   double beta2, float eps, float weight_decay, int64_t step, uint32_t seed,
                                   const float* weight_decay_per_tensor, const float* grad_scale, void* const* w_lowp_out, void* hip_stream) {
    const AdamList a{n_tensors, w, g, g_dtype, reinterpret_cast<void* const*>(m), reinterpret_cast<void* const*>(v), m_scale, v_scale, numel, lr,
                     weight_decay, beta1, beta2, eps, step, seed, weight_decay_per_tensor, grad_scale, w_lowp_out};
    return run_list(a, true, hip_stream);
}
