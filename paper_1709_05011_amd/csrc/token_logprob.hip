// Log probabilities of given tokens over a vocabulary, with entropy and the likeliest alternatives, and the gradient, for gfx950.
//
// Per row of logits z: m = max z, S = sum e^(z-m), T = sum e^(z-m) (z-m); lse = m + log S, log p = z - m - log S, entropy = log S - T/S.
// Bound by memory: the logits are read once.  A row is cut into slices of up to 8192 values that a block holds in registers, so that the
// maximum is known before the first exponential and nothing is rescaled on the way; slices leave (m, S, T) and their own list of
// alternatives, and a second launch joins them (rows of one slice finish where they are).
//
// Alternatives: a value and its place make one 64-bit key (the value's order in the upper half, the complement of its place in the
// lower: equal values by rising place), all different.  A lower bound on the N-th largest of a slice comes from the lanes' own maxima -- N lanes
// have one at least as large -- found by halving over their order with a ballot a step; what reaches it, a few more than N as a
// rule, is gathered in LDS and ranked by one wave.  More than LDS has room for (many equal values): the bound is raised by
// halving over the keys themselves, which ends, as no two are equal.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "token_common.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMostTop = 32;
constexpr int kCandidates = 512;            // keys that LDS has room for
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFar = -150.f;              // e^-150 is 0 in fp32: distances are no longer than this where 0 * infinity would be formed

typedef unsigned long long Key;

struct TokenArgs {
    const void* z;
    const int32_t* tokens;
    float* logprob;
    float* entropy;          // or null
    float* lse;              // or null
    int32_t* top_tokens;
    float* top_logprobs;
    float* stats;            // [rows][slices][4]: m, S, T
    Key* keys;               // [rows][slices][top]
    long long rows, ld;
    int vocab, top, slices, slice;      // slice: values of one, a multiple of 8
};

// order-preserving map of floats to unsigned; both zeros alike
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o ^ ((uint32_t)((int32_t)~o >> 31) | 0x80000000u)); }
__device__ __forceinline__ Key key_of(float z, int at) { return (Key)order_of(z) << 32 | (uint32_t)~(uint32_t)at; }
__device__ __forceinline__ bool listable(float z) { return z > -INFINITY; }         // (false for NaN)

template <typename T>
__device__ __forceinline__ float as_float(T v) {
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)v << 16);
    else return v;
}

struct Row {
    float m, log_s;          // maximum (0 where there is none) and log S
    bool empty;              // every logit is masked
};

// What a row gives but for its alternatives, from its m, S and T (one thread).
template <typename T>
__device__ __forceinline__ Row finish_row(const TokenArgs& p, long long row, float m, double s, double t) {
    Row r;
    r.empty = s == 0.0;
    r.m = m == -INFINITY ? 0.f : m;
    const double log_s = log(s);
    r.log_s = (float)log_s;
    const int token = p.tokens[row];
    float lp = 0.f;
    if (token >= 0 && token < p.vocab) {
        const float z = as_float<T>(static_cast<const T*>(p.z)[row * p.ld + token]);
        lp = r.empty ? -INFINITY : (float)((double)(z - r.m) - log_s);
    }
    p.logprob[row] = lp;
    if (p.entropy) p.entropy[row] = r.empty ? 0.f : (float)(log_s - t / s);
    if (p.lse) p.lse[row] = r.empty ? -INFINITY : (float)((double)r.m + log_s);
    return r;
}

__device__ __forceinline__ void put_alternative(const TokenArgs& p, long long row, int place, Key key, const Row& r) {
    p.top_tokens[row * p.top + place] = key ? (int)~(uint32_t)key : -1;
    p.top_logprobs[row * p.top + place] = key ? (value_of((uint32_t)(key >> 32)) - r.m) - r.log_s : -INFINITY;
}

// Ranks `count` different keys in LDS with one wave; emit(place, key) for the first `top` places, key 0 where there are fewer.
template <typename F>
__device__ __forceinline__ void rank_keys(const Key* keys, int count, int top, F&& emit) {
    const int lane = threadIdx.x & 63;
    for (int i = lane; i < count; i += 64) {
        const Key mine = keys[i];
        int place = 0;
        for (int j = 0; j < count; ++j) place += keys[j] > mine;
        if (place < top) emit(place, mine);
    }
    for (int i = count + lane; i < top; i += 64) emit(i, (Key)0);
}

template <typename T, int CH, bool TOP>
__global__ void __launch_bounds__(kThreads) token_slice_kernel(const TokenArgs p) {
    __shared__ float sums[kWaves][3];
    __shared__ Row joined;
    __shared__ uint32_t bound[kWaves];
    __shared__ int counts[2];
    __shared__ Key keys[TOP ? kCandidates : 1];
    constexpr uint32_t kMaskedBits = sizeof(T) == 2 ? 0xff80u : 0xff800000u;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long units = p.rows * p.slices;
    for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const long long row = p.slices == 1 ? unit : unit / p.slices;
        const int part = (int)(unit - row * p.slices);
        const int first = part * p.slice, end = min(p.vocab - first, p.slice) + first;
        const T* z = static_cast<const T*>(p.z) + row * p.ld;
        Packed<T> v[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) lc_load8(v[i], z, first + (i * kThreads + tid) * 8, end, kMaskedBits);

        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) most = fmaxf(most, v[i].get(j));
        const float m = lc_wave_max(most), from = m == -INFINITY ? 0.f : m;
        float s = 0.f, t = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = v[i].get(j) - from;
                const float e = __builtin_amdgcn_exp2f(d * kLog2e);
                s += e;
                t = fmaf(e, fmaxf(d, kFar), t);
            }
        s = lc_wave_sum(s);
        t = lc_wave_sum(t);
        if (lane == 0) {
            sums[wave][0] = m;
            sums[wave][1] = s;
            sums[wave][2] = t;
        }
        if constexpr (TOP) {
            // the largest order lo that `top` lanes of the wave reach, nearly; without so many lanes that hold a value, the least order
            const uint32_t mine = order_of(most);
            uint32_t lo = order_of(-3.402823466e38f), hi = order_of(m) + 1;
            if (__popcll(__ballot(listable(most))) >= p.top) {
                while (hi - lo > 1) {
                    const uint32_t mid = lo + ((hi - lo) >> 1);
                    const int n = __popcll(__ballot(listable(most) && mine >= mid));
                    if (n >= p.top) {
                        lo = mid;
                        if (n <= p.top + 4) break;
                    } else {
                        hi = mid;
                    }
                }
            }
            if (lane == 0) bound[wave] = lo;
            if (tid == 0) counts[0] = 0;
        }
        __syncthreads();
        if (tid == 0) {
            float bm = sums[0][0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) bm = fmaxf(bm, sums[w][0]);
            double bs = 0.0, bt = 0.0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                // (a wave without a value keeps its sums: 0, or NaN)
                const double shift = sums[w][0] == -INFINITY ? 0.0 : (double)sums[w][0] - (double)bm;
                const double f = exp(shift);
                bs += f * sums[w][1];
                bt += f * (sums[w][2] + shift * sums[w][1]);
            }
            if (p.slices == 1) {
                joined = finish_row<T>(p, row, bm, bs, bt);
            } else {
                float* out = p.stats + unit * 4;
                out[0] = bm;
                out[1] = (float)bs;
                out[2] = (float)bt;
            }
        }
        if constexpr (TOP) {
            Key least = (Key)max(max(bound[0], bound[1]), max(bound[2], bound[3])) << 32;
            auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float x = v[i].get(j);
                        if (listable(x)) f(key_of(x, first + (i * kThreads + tid) * 8 + j));
                    }
            };
            auto gather = [&]() __attribute__((always_inline)) {
                each([&](Key k) {
                    if (k >= least) {
                        const int at = atomicAdd(&counts[0], 1);
                        if (at < kCandidates) keys[at] = k;
                    }
                });
            };
            gather();
            __syncthreads();
            if (counts[0] > kCandidates) {          // the same for every thread
                Key hi = ~(Key)0;                   // fewer than `top` keys reach hi, more than there is room for reach least
                while (true) {
                    const Key mid = least + ((hi - least) >> 1);
                    __syncthreads();
                    if (tid == 0) counts[1] = 0;
                    __syncthreads();
                    int n = 0;
                    each([&](Key k) { n += k >= mid; });
                    if (n) atomicAdd(&counts[1], n);
                    __syncthreads();
                    n = counts[1];
                    if (n >= p.top) least = mid;
                    else hi = mid;
                    if ((n >= p.top && n <= kCandidates) || hi - least <= 1) break;
                }
                __syncthreads();
                if (tid == 0) counts[0] = 0;
                __syncthreads();
                gather();
                __syncthreads();
            }
            if (wave == 0) {
                const int count = min(counts[0], kCandidates);
                if (p.slices == 1) rank_keys(keys, count, p.top, [&](int place, Key k) { put_alternative(p, row, place, k, joined); });
                else rank_keys(keys, count, p.top, [&](int place, Key k) { p.keys[unit * p.top + place] = k; });
            }
        }
        __syncthreads();
    }
}

// Joins a row's slices: one wave a row.
template <typename T>
__global__ void __launch_bounds__(64) token_join_kernel(const TokenArgs p) {
    __shared__ Key keys[kCandidates];
    __shared__ int held;
    const int lane = threadIdx.x;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const float* stats = p.stats + row * p.slices * 4;
        float m = -INFINITY;
        for (int i = lane; i < p.slices; i += 64) m = fmaxf(m, stats[4 * i]);
        m = lc_wave_max(m);
        double s = 0.0, t = 0.0;
        for (int i = lane; i < p.slices; i += 64) {
            const double shift = stats[4 * i] == -INFINITY ? 0.0 : (double)stats[4 * i] - (double)m;
            const double f = exp(shift);
            s += f * stats[4 * i + 1];
            t += f * (stats[4 * i + 2] + shift * stats[4 * i + 1]);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            s += __shfl_xor(s, off, 64);
            t += __shfl_xor(t, off, 64);
        }
        Row r;
        if (lane == 0) r = finish_row<T>(p, row, m, s, t);
        if (p.top) {
            r.m = __shfl(r.m, 0, 64);
            r.log_s = __shfl(r.log_s, 0, 64);
            const Key* lists = p.keys + row * p.slices * p.top;
            const long long all = (long long)p.slices * p.top;
            // slices * k keys are no smaller than the least of the lists' k-th ones
            const int k = (p.top + p.slices - 1) / p.slices;
            Key least = ~(Key)0;
            for (int i = lane; i < p.slices; i += 64) least = min(least, lists[(long long)i * p.top + k - 1]);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) least = min(least, (Key)__shfl_xor(least, off, 64));
            least = max(least, (Key)1);             // (0: a place left over)
            auto count = [&](Key bound) __attribute__((always_inline)) {
                int n = 0;
                for (long long i = lane; i < all; i += 64) n += lists[i] >= bound;
#pragma unroll
                for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, 64);
                return n;
            };
            int n = count(least);
            Key hi = ~(Key)0;
            while (n > kCandidates && hi - least > 1) {
                const Key mid = least + ((hi - least) >> 1);
                const int c = count(mid);
                if (c >= p.top) {
                    least = mid;
                    n = c;
                } else {
                    hi = mid;
                }
            }
            if (lane == 0) held = 0;
            __syncthreads();
            for (long long i = lane; i < all; i += 64) {
                const Key key = lists[i];
                if (key >= least) {
                    const int at = atomicAdd(&held, 1);
                    if (at < kCandidates) keys[at] = key;
                }
            }
            __syncthreads();
            rank_keys(keys, min(held, kCandidates), p.top, [&](int place, Key key) { put_alternative(p, row, place, key, r); });
            __syncthreads();
        }
    }
}

struct TokenBwdArgs {
    const void* z;
    const int32_t* tokens;
    const float* lse;
    const float* entropy;
    const float* dlogprob;
    const float* dentropy;
    void* dz;
    long long rows, ld, dld, units;
    int vocab, parts;        // parts of 512 columns a row has
};

// One wave a block, eight columns a lane.
template <typename T>
__global__ void __launch_bounds__(64) token_bwd_kernel(const TokenBwdArgs p) {
    for (long long unit = blockIdx.x; unit < p.units; unit += gridDim.x) {
        const long long row = p.parts == 1 ? unit : unit / p.parts;
        const int col = ((int)(unit - row * p.parts) * 64 + (int)threadIdx.x) * 8;
        if (col >= p.vocab) continue;
        Packed<T> v;
        lc_load8(v, static_cast<const T*>(p.z) + row * p.ld, col, p.vocab);
        const float lse = p.lse[row];
        const int token = p.tokens[row];
        const bool empty = lse == -INFINITY, counts = token >= 0 && token < p.vocab;
        const float a = p.dlogprob && counts && !empty ? p.dlogprob[row] : 0.f;
        const float b = p.dentropy && !empty ? p.dentropy[row] : 0.f;
        const float ent = p.dentropy ? p.entropy[row] : 0.f;
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = v.get(j) - lse;
            const float e = __builtin_amdgcn_exp2f(d * kLog2e);
            o[j] = empty ? 0.f : -e * (a + b * (fmaxf(d, kFar) + ent));
            if (col + j == token) o[j] += a;
        }
        lc_store8(static_cast<T*>(p.dz) + row * p.dld + col, o, p.vocab - col);
    }
}

constexpr int kMostWidth = 1 << 30;
constexpr long long kMostBlocks = 1 << 22;          // of 256 threads; more units are dealt round

lc_status check_desc(const lc_token_desc* d) {
    if (!d) return LC_ERR_NULL;
    if (d->dtype != LC_F32 && d->dtype != LC_BF16) return LC_ERR_UNSUPPORTED;
    if (d->rows < 0 || d->vocab <= 0 || d->vocab > kMostWidth || (d->ld && d->ld < d->vocab)) return LC_ERR_SHAPE;
    if (d->top < 0 || d->top > kMostTop) return LC_ERR_UNSUPPORTED;
    long long bytes;          // every offset in bytes, the workspace's (at most 260 for 512 logits) among them, fits 63 bits
    if (__builtin_mul_overflow((long long)d->rows, std::max<long long>({d->ld, d->vocab, 512}), &bytes) || __builtin_mul_overflow(bytes, 8ll, &bytes))
        return LC_ERR_SHAPE;
    return LC_OK;
}

struct TokenPlan {
    int chunks, slices, slice;
    size_t stats, keys, total;
};

// Even slices, so that no last one is short of values.
TokenPlan plan_of(const lc_token_desc* d) {
    TokenPlan p;
    p.chunks = d->vocab <= kThreads * 8 ? 1 : d->vocab <= kThreads * 16 ? 2 : 4;
    const int most = kThreads * 8 * p.chunks;
    p.slices = (d->vocab + most - 1) / most;
    p.slice = ((d->vocab + p.slices - 1) / p.slices + 7) & ~7;
    p.slices = (d->vocab + p.slice - 1) / p.slice;
    const size_t units = (size_t)d->rows * p.slices;
    p.stats = 0;
    p.keys = p.slices == 1 ? 0 : (units * 16 + 255) & ~(size_t)255;
    p.total = p.slices == 1 ? 0 : p.keys + ((units * d->top * sizeof(Key) + 255) & ~(size_t)255);
    return p;
}

template <typename T, bool TOP>
void launch_slices(const TokenArgs& a, int chunks, hipStream_t stream) {
    const dim3 grid((unsigned)std::min(a.rows * a.slices, kMostBlocks));
    if (chunks == 1) hipLaunchKernelGGL((token_slice_kernel<T, 1, TOP>), grid, dim3(kThreads), 0, stream, a);
    else if (chunks == 2) hipLaunchKernelGGL((token_slice_kernel<T, 2, TOP>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((token_slice_kernel<T, 4, TOP>), grid, dim3(kThreads), 0, stream, a);
}

template <typename T>
void launch_fwd(const TokenArgs& a, int chunks, hipStream_t stream) {
    a.top ? launch_slices<T, true>(a, chunks, stream) : launch_slices<T, false>(a, chunks, stream);
    if (a.slices > 1) hipLaunchKernelGGL((token_join_kernel<T>), dim3((unsigned)std::min(a.rows, kMostBlocks)), dim3(64), 0, stream, a);
}

}  // namespace

extern "C" size_t token_logprob_workspace_bytes(const lc_token_desc* desc) {
    if (check_desc(desc) != LC_OK) return 0;
    return plan_of(desc).total;
}

extern "C" lc_status token_logprob_fwd(const lc_token_desc* desc, const void* logits, const int32_t* tokens, float* logprob, float* entropy,
                                       float* lse, int32_t* top_tokens, float* top_logprobs, void* workspace, size_t workspace_bytes,
                                       void* hip_stream) {
    const lc_status st = check_desc(desc);
    if (st != LC_OK) return st;
    if (desc->rows == 0) return LC_OK;
    if (!logits || !tokens || !logprob) return LC_ERR_NULL;
    if (desc->top && (!top_tokens || !top_logprobs)) return LC_ERR_NULL;
    if (!desc->top && (top_tokens || top_logprobs)) return LC_ERR_UNSUPPORTED;
    if (lc_off_element(logits, desc->dtype == LC_BF16 ? 2 : 4) || lc_off_element(tokens, 4) || lc_off_element(logprob, 4) || lc_off_element(entropy, 4) ||
        lc_off_element(lse, 4) || lc_off_element(top_tokens, 4) || lc_off_element(top_logprobs, 4))
        return LC_ERR_ALIGN;
    const TokenPlan plan = plan_of(desc);
    if (plan.total && (!workspace || (((uintptr_t)workspace) & 255) || workspace_bytes < plan.total)) return LC_ERR_WORKSPACE;
    char* base = static_cast<char*>(workspace);
    TokenArgs a{logits, tokens, logprob, entropy, lse, top_tokens, top_logprobs, plan.total ? reinterpret_cast<float*>(base + plan.stats) : nullptr,
                plan.total ? reinterpret_cast<Key*>(base + plan.keys) : nullptr, desc->rows, desc->ld ? desc->ld : desc->vocab, desc->vocab, desc->top,
                plan.slices, plan.slice};
    lc_begin_call();
    if (desc->dtype == LC_BF16) launch_fwd<uint16_t>(a, plan.chunks, static_cast<hipStream_t>(hip_stream));
    else launch_fwd<float>(a, plan.chunks, static_cast<hipStream_t>(hip_stream));
    return lc_end_call();
}

extern "C" lc_status token_logprob_bwd(const lc_token_desc* desc, const void* logits, const int32_t* tokens, const float* lse,
                                       const float* entropy, const float* dlogprob, const float* dentropy, void* dlogits, int64_t dlogits_ld,
                                       void* hip_stream) {
    const lc_status st = check_desc(desc);
    if (st != LC_OK) return st;
    if (dlogits_ld && dlogits_ld < desc->vocab) return LC_ERR_SHAPE;
    long long span;
    if (__builtin_mul_overflow((long long)desc->rows, (long long)dlogits_ld, &span) || __builtin_mul_overflow(span, 4ll, &span)) return LC_ERR_SHAPE;
    if (desc->rows == 0) return LC_OK;
    if (!logits || !tokens || !lse || !dlogits || (!dlogprob && !dentropy) || (dentropy && !entropy)) return LC_ERR_NULL;
    const size_t e = desc->dtype == LC_BF16 ? 2 : 4;
    if (lc_off_element(logits, e) || lc_off_element(dlogits, e) || lc_off_element(tokens, 4) || lc_off_element(lse, 4) || lc_off_element(entropy, 4) ||
        lc_off_element(dlogprob, 4) || lc_off_element(dentropy, 4))
        return LC_ERR_ALIGN;
    TokenBwdArgs a{logits, tokens, lse, entropy, dlogprob, dentropy, dlogits, desc->rows, desc->ld ? desc->ld : desc->vocab,
                   dlogits_ld ? dlogits_ld : desc->vocab, 0, desc->vocab, (desc->vocab + 511) / 512};
    a.units = a.rows * a.parts;
    const dim3 grid((unsigned)std::min(a.units, 4 * kMostBlocks));
    lc_begin_call();
    if (desc->dtype == LC_BF16) hipLaunchKernelGGL((token_bwd_kernel<uint16_t>), grid, dim3(64), 0, static_cast<hipStream_t>(hip_stream), a);
    else hipLaunchKernelGGL((token_bwd_kernel<float>), grid, dim3(64), 0, static_cast<hipStream_t>(hip_stream), a);
    return lc_end_call();
}
