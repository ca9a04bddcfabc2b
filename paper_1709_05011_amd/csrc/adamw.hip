// AdamW over a list of tensors for gfx950: one streaming pass, states in fp32 or in 8 bits with a scale per 256 elements.
//
// m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  w <- w - lr decay w - lr (m / c1) / (sqrt(v) / sqrt(c2) + eps).  Bound by memory: 28 bytes a
// parameter with fp32 states and gradients (2 more with a bf16 copy of w, 2 fewer with bf16 gradients), 16.06 with 8-bit states, fp32 gradients and no copy.
// The list is cut into chunks of one tensor each; descriptors travel as launch arguments, and a wave finds the tensor of its chunk with
// one probe of their first chunks.  A wave owns 256 consecutive elements, four a lane: one block of the 8-bit states, whose new
// values, largest magnitudes and codes are made in registers between the loads and the stores.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "token_common.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWavePart = 256;                                   // elements of a wave
constexpr int kChunk = kWavePart * (kThreads / 64);
constexpr int kTable = 176;                                      // descriptors per launch (13.4 KB of launch arguments)
static_assert(kWavePart == ADAMW_Q8_BLOCK, "a wave makes a block's scale by itself");

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

struct AdamArgs {
    AdamTensor t[kTable];
    int start[kTable];     // first chunk of each, ascending
    int count, chunks;
    const float* grad_scale;
    float b1, one_b1, b2, one_b2, step_size, inv_root_c2, eps;
    uint32_t dither;
};

// 21 bits from an element's number: two rounds of shift and odd product (the golden ratio's and root two's bits) modulo 2^32.
__device__ __forceinline__ uint32_t dither21(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x9E3779B1u;
    x = (x ^ (x >> 15)) * 0x6A09E667u;
    return x >> 11;
}

// The exponent of the smallest power of two >= 2^-126 that brings amax to 1.75 * 2^top at most (0 for amax = 0).
__device__ __forceinline__ int scale_exponent(float amax, int top) {
    const uint32_t b = __float_as_uint(amax);
    const int k = (int)(b >> 23) - 127 - top + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return b == 0 ? 0 : max(k, -126);
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// e5m2 of x in [0, 57344] rounded up with the probability that keeps the mean: the dither is added below the last place.  Above zero at least code 1.
__device__ __forceinline__ uint32_t e5m2_dithered(float x, uint32_t r) {
    const uint32_t b = __float_as_uint(x);
    const uint32_t code = x < 0x1p-14f ? ((uint32_t)(x * 0x1p37f) + r) >> 21 : ((b + r) >> 21) - (112u << 2);
    return x > 0.f ? max(code, 1u) : 0u;
}

__device__ __forceinline__ float finite_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }

template <typename G, bool Q8>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const AdamArgs p) {
#pragma clang fp contract(off)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float gs = p.grad_scale ? *p.grad_scale : 1.f;
    for (int chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x) {
        int owner = -1;
#pragma unroll
        for (int i = 0; i < kTable; i += 64) {
            const int at = i + lane;
            owner += __popcll(__ballot(at < p.count && p.start[at < kTable ? at : 0] <= chunk));
        }
        const AdamTensor& t = p.t[__builtin_amdgcn_readfirstlane(owner)];
        const long long block = (long long)(chunk - p.start[__builtin_amdgcn_readfirstlane(owner)]) * (kThreads / 64) + wave;
        const long long first = block * kWavePart, at = first + lane * 4;
        if (first >= t.numel) continue;
        const long long left = t.numel - at;
        const int n = left < 4 ? (int)left : 4;                       // this lane's elements; none or fewer than none past the end
        float w[4], g[4], m[4], v[4];
        const float* tw = t.w + at;
        const G* tg = static_cast<const G*>(t.g) + at;
        if (n == 4) {
            lc_u32x4 x;
            __builtin_memcpy(&x, tw, 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = __uint_as_float(x[j]);
            if constexpr (sizeof(G) == 2) {
                uint32_t h[2];
                __builtin_memcpy(h, tg, 8);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] = __uint_as_float(j & 1 ? h[j >> 1] & 0xffff0000u : h[j >> 1] << 16);
            } else {
                __builtin_memcpy(&x, tg, 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] = __uint_as_float(x[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = j < n ? tw[j] : 0.f;
                if constexpr (sizeof(G) == 2) g[j] = j < n ? __uint_as_float((uint32_t)tg[j] << 16) : 0.f;
                else g[j] = j < n ? tg[j] : 0.f;
            }
        }
        if constexpr (Q8) {
            const uint8_t* tm = static_cast<const uint8_t*>(t.m) + at;
            const uint8_t* tv = static_cast<const uint8_t*>(t.v) + at;
            uint32_t cm = 0, cv = 0;
            if (n == 4) {
                __builtin_memcpy(&cm, tm, 4);
                __builtin_memcpy(&cv, tv, 4);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < n) {
                        cm |= (uint32_t)tm[j] << (8 * j);
                        cv |= (uint32_t)tv[j] << (8 * j);
                    }
            }
            const float ms = t.m_scale[block], vs = t.v_scale[block];
            m[0] = __builtin_amdgcn_cvt_f32_fp8((int)cm, 0) * ms;
            m[1] = __builtin_amdgcn_cvt_f32_fp8((int)cm, 1) * ms;
            m[2] = __builtin_amdgcn_cvt_f32_fp8((int)cm, 2) * ms;
            m[3] = __builtin_amdgcn_cvt_f32_fp8((int)cm, 3) * ms;
            v[0] = __builtin_amdgcn_cvt_f32_bf8((int)cv, 0) * vs;
            v[1] = __builtin_amdgcn_cvt_f32_bf8((int)cv, 1) * vs;
            v[2] = __builtin_amdgcn_cvt_f32_bf8((int)cv, 2) * vs;
            v[3] = __builtin_amdgcn_cvt_f32_bf8((int)cv, 3) * vs;
        } else {
            const float* tm = static_cast<const float*>(t.m) + at;
            const float* tv = static_cast<const float*>(t.v) + at;
            if (n == 4) {
                lc_u32x4 x, y;
                __builtin_memcpy(&x, tm, 16);
                __builtin_memcpy(&y, tv, 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    m[j] = __uint_as_float(x[j]);
                    v[j] = __uint_as_float(y[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    m[j] = j < n ? tm[j] : 0.f;
                    v[j] = j < n ? tv[j] : 0.f;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = g[j] * gs;
            m[j] = p.b1 * m[j] + p.one_b1 * x;
            v[j] = p.b2 * v[j] + p.one_b2 * (x * x);
            const float root = sqrtf(v[j]) * p.inv_root_c2 + p.eps;
            w[j] = w[j] - t.lr_decay * w[j] - p.step_size * (m[j] / root);
        }
        float* ow = t.w + at;
        uint16_t* ol = t.w_lowp ? t.w_lowp + at : nullptr;
        if (n == 4) {
            const lc_u32x4 x = {__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3])};
            __builtin_memcpy(ow, &x, 16);
            if (ol) {
                const uint32_t h[2] = {lc_bf16x2_rne(w[0], w[1]), lc_bf16x2_rne(w[2], w[3])};
                __builtin_memcpy(ol, h, 8);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < n) {
                    ow[j] = w[j];
                    if (ol) ol[j] = lc_bf16_rne(w[j]);
                }
        }
        if constexpr (Q8) {
            float am = 0.f, av = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                am = fmaxf(am, finite_size(m[j]));
                av = fmaxf(av, finite_size(v[j]));
            }
            const int km = scale_exponent(lc_wave_max(am), 8), kv = scale_exponent(lc_wave_max(av), 15);
            if (lane == 0) {
                t.m_scale[block] = power_of_two(km);
                t.v_scale[block] = power_of_two(kv);
            }
            const float im = power_of_two(-km), iv = power_of_two(-kv);
            int cm = 0;
            cm = __builtin_amdgcn_cvt_pk_fp8_f32(m[0] * im, m[1] * im, cm, false);
            cm = __builtin_amdgcn_cvt_pk_fp8_f32(m[2] * im, m[3] * im, cm, true);
            uint32_t cv = 0;
            const uint32_t number = (uint32_t)at + (uint32_t)((unsigned long long)at >> 32) * 0x6A09E667u + p.dither;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = v[j] * iv;
                const uint32_t code = x < INFINITY ? e5m2_dithered(x, dither21(number + j)) : 0x7fu;
                cv |= code << (8 * j);
            }
            uint8_t* om = static_cast<uint8_t*>(t.m) + at;
            uint8_t* ov = static_cast<uint8_t*>(t.v) + at;
            if (n == 4) {
                __builtin_memcpy(om, &cm, 4);
                __builtin_memcpy(ov, &cv, 4);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < n) {
                        om[j] = (uint8_t)((uint32_t)cm >> (8 * j));
                        ov[j] = (uint8_t)(cv >> (8 * j));
                    }
            }
        } else {
            float* om = static_cast<float*>(t.m) + at;
            float* ov = static_cast<float*>(t.v) + at;
            if (n == 4) {
                const lc_u32x4 x = {__float_as_uint(m[0]), __float_as_uint(m[1]), __float_as_uint(m[2]), __float_as_uint(m[3])};
                const lc_u32x4 y = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                __builtin_memcpy(om, &x, 16);
                __builtin_memcpy(ov, &y, 16);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < n) {
                        om[j] = m[j];
                        ov[j] = v[j];
                    }
            }
        }
    }
}

constexpr int kMostBlocks = 1 << 23;      // of 256 threads: a launch holds fewer than 2^32

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

long long chunks_of(int64_t numel) { return numel / kChunk + (numel % kChunk != 0); }

lc_status check_list(const AdamList& a, bool q8) {
    if (a.n < 0) return LC_ERR_SHAPE;
    if (a.g_dtype != LC_F32 && a.g_dtype != LC_BF16) return LC_ERR_UNSUPPORTED;
    if (!(a.beta1 >= 0.0 && a.beta1 < 1.0) || !(a.beta2 >= 0.0 && a.beta2 < 1.0) || !(a.eps > 0.f) || a.step < 1) return LC_ERR_UNSUPPORTED;
    if (a.n == 0) return LC_OK;
    if (!a.w || !a.g || !a.m || !a.v || !a.numel || (q8 && (!a.m_scale || !a.v_scale))) return LC_ERR_NULL;
    if (lc_off_element(a.grad_scale, 4)) return LC_ERR_ALIGN;
    for (int l = 0; l < a.n; ++l) {
        if (a.numel[l] < 0 || a.numel[l] > (int64_t)1 << 40) return LC_ERR_SHAPE;
        if (a.numel[l] == 0) continue;
        if (!a.w[l] || !a.g[l] || !a.m[l] || !a.v[l] || (q8 && (!a.m_scale[l] || !a.v_scale[l]))) return LC_ERR_NULL;
        if (lc_off_element(a.w[l], 4) || lc_off_element(a.g[l], a.g_dtype == LC_BF16 ? 2 : 4) || (a.w_lowp && lc_off_element(a.w_lowp[l], 2))) return LC_ERR_ALIGN;
        if (q8 ? lc_off_element(a.m_scale[l], 4) || lc_off_element(a.v_scale[l], 4) : lc_off_element(a.m[l], 4) || lc_off_element(a.v[l], 4)) return LC_ERR_ALIGN;
    }
    return LC_OK;
}

lc_status run_list(const AdamList& a, bool q8, void* hip_stream) {
    const lc_status st = check_list(a, q8);
    if (st != LC_OK || a.n == 0 || std::all_of(a.numel, a.numel + a.n, [](int64_t n) { return n == 0; })) return st;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    AdamArgs args;
    args.grad_scale = a.grad_scale;
    args.b1 = (float)a.beta1;
    args.one_b1 = (float)(1.0 - a.beta1);
    args.b2 = (float)a.beta2;
    args.one_b2 = (float)(1.0 - a.beta2);
    args.step_size = (float)((double)a.lr / (1.0 - std::pow(a.beta1, (double)a.step)));
    args.inv_root_c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(a.beta2, (double)a.step)));
    args.eps = a.eps;
    args.dither = a.seed * 0x9E3779B1u + 0x7F4A7C15u;
    lc_begin_call();
    for (int l = 0; l < a.n;) {
        long long chunks = 0;
        int count = 0;
        for (; l < a.n && count < kTable; ++l) {
            if (a.numel[l] == 0) continue;
            const long long more = chunks_of(a.numel[l]);
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
        args.count = count;
        args.chunks = (int)chunks;
        const dim3 grid((unsigned)std::min<long long>(chunks, kMostBlocks));
        if (a.g_dtype == LC_BF16) {
            if (q8) hipLaunchKernelGGL((adamw_kernel<uint16_t, true>), grid, dim3(kThreads), 0, stream, args);
            else hipLaunchKernelGGL((adamw_kernel<uint16_t, false>), grid, dim3(kThreads), 0, stream, args);
        } else {
            if (q8) hipLaunchKernelGGL((adamw_kernel<float, true>), grid, dim3(kThreads), 0, stream, args);
            else hipLaunchKernelGGL((adamw_kernel<float, false>), grid, dim3(kThreads), 0, stream, args);
        }
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
