// Root-mean-square norm with the residual's addition, its output in the storage type or in 8 bits, and its gradient, for gfx950.
//
// total = x + residual, rstd = 1/sqrt(mean total^2 + eps), y = (total * rstd) * gamma; with a = dy * gamma and n = total * rstd,
// dx = rstd * (a - n * mean(a * n)) + dtotal and dgamma = sum over rows of dy * n.  Bound by memory: a row is read once into registers,
// summed, and written from there.  A thread owns eight neighbouring columns at a time for either type, so that a group of 32 to 512
// columns with a scale of its own is 4 to 64 neighbouring lanes of one wave.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "norm_common.h"
#include "token_common.h"

namespace {

struct NormArgs {
    const void* x;
    const void* r;           // residual or null
    const float* gamma;
    void* total;             // or null
    void* y;                 // T, or e4m3 codes
    float* scales;           // 8 bits only
    float* rstd;             // or null
    long long rows, x_ld, r_ld;
    int c, group;
    float eps;
    double inv_c;            // 1 / c
};

constexpr float kE4m3Max = 448.f, kLeastScale = 0x1p-126f;

// 1/sqrt(sum / c + eps) to more than fp32's places: the instruction's estimate and one step of Newton's method in double.
__device__ __forceinline__ double rstd_of(const NormArgs& p, float sum) {
    const double x = fma((double)sum, p.inv_c, (double)p.eps);
    const double r = (double)__builtin_amdgcn_rsqf((float)x);
    const double better = r * fma(-0.5 * x * r, r, 1.5);
    return fabs(better) < INFINITY ? better : r;         // (x = 0 or infinite: the estimate is the value)
}

// Whether squares summed as they are say enough: their sum is finite, and either eps hides what they lose under fp32's normal range or none does (2^30 of them lose 2^-120
// at most).  Other rows are summed again as totals / 2^e with 2^e above the largest.
__device__ __forceinline__ bool sum_serves(const NormArgs& p, float sum) { return sum < INFINITY && (p.eps >= 0x1p-120f || sum >= 0x1p-90f); }
__device__ __forceinline__ double rstd_of_scaled(const NormArgs& p, float sum, int e) {
    const double x = ldexp((double)sum * p.inv_c, 2 * e) + (double)p.eps;
    const int half = __builtin_amdgcn_frexp_exp(x) >> 1;
    const double near = ldexp(x, -2 * half), r = (double)__builtin_amdgcn_rsqf((float)near);
    const double better = r * fma(-0.5 * near * r, r, 1.5);
    return ldexp(fabs(better) < INFINITY ? better : r, -half);
}

// rstd as a power of two and the rest, in [0.5, 1): a total times the power is near its normalised value, so that its product with gamma leaves fp32's range only where the
// output does.  (The power is 1 for zero, infinity and NaN; it is exact otherwise, and so is a product with it.)
struct Split {
    float power;
    double rest;
};
__device__ __forceinline__ Split split_of(double rstd) {
    const int e = __builtin_amdgcn_frexp_exp(rstd);
    return {ldexpf(1.f, e), ldexp(rstd, -e)};
}

// A group's scale from its largest |g|, g = total * power * gamma, and the rest of rstd, and what takes g to codes: rest / scale as the sum of two floats.
struct Scale {
    float scale, hi, lo;
};
__device__ __forceinline__ Scale scale_of(float amax, double rest) {
    Scale s;
    s.scale = fmaxf((float)((double)amax * rest * (1.0 / kE4m3Max)), kLeastScale);
    const double r = (double)__builtin_amdgcn_rcpf(s.scale), k = rest * (r * fma(-(double)s.scale, r, 2.0));
    s.hi = s.scale < INFINITY ? (float)k : 0.f;
    s.lo = s.scale < INFINITY ? (float)(k - (double)s.hi) : 0.f;
    return s;
}

// Eight e4m3 codes of g[j] * rest / scale, to nearest even; `low` holds what the rounding of g[j] left.  The quotient is right to nearly all of fp32's places, so that a code is
// off the exact value's only next to a border; with y * (1 / scale) in fp32 more of them were (4099 rows of 5120 with groups of 128: 28.0 us, so 28.9).  NaN keeps the code of NaN.
__device__ __forceinline__ void store8_e4m3(uint8_t* p, const float* g, const float* low, const Scale& s, double rest, int n) {
    float q[8];
    if (s.scale > kLeastScale) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = g[j] * s.hi;
            q[j] = a + fmaf(g[j], s.lo, fmaf(low[j], s.hi, fmaf(g[j], s.hi, -a)));
        }
    } else {                                            // (rest / scale may be beyond fp32)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = (float)((double)g[j] * rest) * (1.f / kLeastScale);
    }
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int u = 0;
        u = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * k], q[4 * k + 1], u, false);
        u = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * k + 2], q[4 * k + 3], u, true);
        w[k] = (uint32_t)u;
    }
    if (n >= 8) {
        __builtin_memcpy(p, w, 8);
    } else {
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            p[j] = (uint8_t)w[0];
            w[0] = __builtin_amdgcn_alignbit(w[1], w[0], 8);
            w[1] >>= 8;
        }
    }
}

// A block per row (rows dealt round the grid), its waves as many as the row has 512 * CH columns: all of a row's loads are under way at once and it is read once.  What bounds it is
// memory: 8192 rows of 4096 bf16 with the residual, its sum and the output 45.5 us, 5.9 TB/s of the 268 MB that must move; 4099 rows of 5120 with residual and sum to 8 bits with a scale per 128
// 28.9 us, 5.1 TB/s; one row 2.8 us, a launch.  NT: past the caches.  ENDS: what may lie past a row's end, so that rows of whole waves carry no comparisons.  LANES: several narrow rows
// of a wave instead (2^18 rows of 128 bf16 26 us, 5.1 TB/s).
template <typename T, int CH, bool Q8, bool NT, Ends ENDS, int LANES = 0>
__global__ void __launch_bounds__(LANES ? kNarrowThreads : kMostWaves * 64) rmsnorm_fwd_kernel(const NormArgs p) {
    __shared__ float red[2][4][kMostWaves];
    using Of = Rows<LANES>;
    const int tid = Of::tid(), c = p.c, waves = blockDim.x >> 6, threads = LANES ? LANES : blockDim.x;
    const auto column = [=](int i) { return (i * threads + tid) * 8; };
    const auto inside = [&](int i) { return ENDS == kWhole ? 8 : ENDS == kEights ? (column(i) < c ? 8 : 0) : c - column(i); };
    int parity = 0;
    for (long long row = Of::first(); row < p.rows; row += Of::step(), parity ^= 1) {
        const T* x = static_cast<const T*>(p.x) + row * p.x_ld;
        Packed<T> px[CH], pr[CH];
        Packed<float> pg[CH];
        float h[CH][8];
        lc_issue8<ENDS, NT>(px, x, column, c);
        if (p.r) lc_issue8<ENDS, NT>(pr, static_cast<const T*>(p.r) + row * p.r_ld, column, c);
        lc_issue8<ENDS>(pg, p.gamma, column, c);
        float ss = 0.f;
        lc_settle8<ENDS>(px, column, c);
        if (p.r) {
            lc_settle8<ENDS>(pr, column, c);
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = lc_as_stored<T>(px[i].get(j) + pr[i].get(j));
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = px[i].get(j);
        }
        lc_settle8<ENDS>(pg, column, c);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) ss = fmaf(h[i][j], h[i][j], ss);
        if (p.total) {
            T* t = static_cast<T*>(p.total) + row * (long long)c;
#pragma unroll
            for (int i = 0; i < CH; ++i) lc_store8<NT>(t + column(i), h[i], inside(i));
        }
        ss = Of::join(ss, waves, red[parity][0], [](float a) { return lc_wave_sum(a); }, [](float a, float b) { return a + b; });
        double rstd;
        if (sum_serves(p, ss)) {
            rstd = rstd_of(p, ss);
        } else {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(h[i][j]));
            most = Of::join(most, waves, red[parity][2], [](float a) { return lc_wave_max(a); }, [](float a, float b) { return fmaxf(a, b); });
            const int e = __builtin_amdgcn_frexp_expf(most);         // (0 for zero and infinity)
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float n = ldexpf(h[i][j], -e);
                    s = fmaf(n, n, s);
                }
            rstd = rstd_of_scaled(p, Of::join(s, waves, red[parity][3], [](float a) { return lc_wave_sum(a); }, [](float a, float b) { return a + b; }), e);
        }
        if (p.rstd && tid == 0) p.rstd[row] = (float)rstd;
        if constexpr (!Q8) {
            const float r = (float)rstd;
            T* y = static_cast<T*>(p.y) + row * (long long)c;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = h[i][j] * r * pg[i].get(j);
                lc_store8<NT>(y + column(i), h[i], inside(i));
            }
        } else {
            uint8_t* y = static_cast<uint8_t*>(p.y) + row * (long long)c;
            const Split split = split_of(rstd);
            float low[CH][8], amax[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                amax[i] = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float n = h[i][j] * split.power, g = n * pg[i].get(j);
                    low[i][j] = fmaf(n, pg[i].get(j), -g);
                    h[i][j] = g;
                    amax[i] = fmaxf(amax[i], fabsf(g));
                }
            }
            if (p.group == 0) {
                float m = amax[0];
#pragma unroll
                for (int i = 1; i < CH; ++i) m = fmaxf(m, amax[i]);
                m = Of::join(m, waves, red[parity][1], [](float a) { return lc_wave_max(a); }, [](float a, float b) { return fmaxf(a, b); });
                const Scale scale = scale_of(m, split.rest);
                if (tid == 0) p.scales[row] = scale.scale;
#pragma unroll
                for (int i = 0; i < CH; ++i) store8_e4m3(y + column(i), h[i], low[i], scale, split.rest, inside(i));
            } else {
                const int lanes = LANES ? min(p.group >> 3, LANES) : p.group >> 3, shift = __builtin_ctz(p.group);
                const long long groups = (c + p.group - 1) >> shift;
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    float m = amax[i];
                    for (int off = 1; off < lanes; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
                    const Scale scale = scale_of(m, split.rest);
                    if (column(i) < c && (tid & (lanes - 1)) == 0) p.scales[row * groups + (column(i) >> shift)] = scale.scale;
                    store8_e4m3(y + column(i), h[i], low[i], scale, split.rest, inside(i));
                }
            }
        }
    }
}

// Rows too wide for the registers of a block, or under eight columns: the same in passes over the row, which the caches hold (2048 rows of 16384 bf16 68 us, in registers 47).
template <typename T, bool Q8>
__global__ void __launch_bounds__(1024) rmsnorm_fwd_wide_kernel(const NormArgs p) {
    constexpr int WAVES = 16, kSpan = WAVES * 64 * 8;
    __shared__ float red[2][4][WAVES];
    const int tid = threadIdx.x, c = p.c;
    int parity = 0;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x, parity ^= 1) {
        const T* x = static_cast<const T*>(p.x) + row * p.x_ld;
        const T* r = p.r ? static_cast<const T*>(p.r) + row * p.r_ld : nullptr;
        T* t = p.total ? static_cast<T*>(p.total) + row * (long long)c : nullptr;
        // the stored sum is what later passes read (total may be x's or the residual's own buffer)
        auto value = [&](int col, float* h, bool first) __attribute__((always_inline)) {
            Packed<T> a, b;
            if (!first && t) {
                lc_load8(a, const_cast<const T*>(t), col, c);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] = a.get(j);
                return;
            }
            lc_load8(a, x, col, c);
            if (r) lc_load8(b, r, col, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = r ? lc_as_stored<T>(a.get(j) + b.get(j)) : a.get(j);
        };
        float ss = 0.f, h[8];
        for (long long at = tid * 8; at < c; at += kSpan) {
            const int col = (int)at;
            value(col, h, true);
#pragma unroll
            for (int j = 0; j < 8; ++j) ss = fmaf(h[j], h[j], ss);
            if (t) lc_store8(t + col, h, c - col);
        }
        ss = lc_block_sum<WAVES>(ss, red[parity][0]);
        double rstd;
        if (sum_serves(p, ss)) {
            rstd = rstd_of(p, ss);
        } else {
            const auto over = [&](auto&& f) __attribute__((always_inline)) {
                for (long long at = tid * 8; at < c; at += kSpan) {
                    value((int)at, h, false);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f(h[j]);
                }
            };
            float most = 0.f, s = 0.f;
            over([&](float x) { most = fmaxf(most, fabsf(x)); });
            const int e = __builtin_amdgcn_frexp_expf(lc_block_max<WAVES>(most, red[parity][2]));
            over([&](float x) {
                const float n = ldexpf(x, -e);
                s = fmaf(n, n, s);
            });
            rstd = rstd_of_scaled(p, lc_block_sum<WAVES>(s, red[parity][3]), e);
        }
        if (p.rstd && tid == 0) p.rstd[row] = (float)rstd;
        if constexpr (!Q8) {
            const float r = (float)rstd;
            for (long long at = tid * 8; at < c; at += kSpan) {
                Packed<float> g;
                lc_load8(g, p.gamma, (int)at, c);
                value((int)at, h, false);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] = h[j] * r * g.get(j);
                lc_store8(static_cast<T*>(p.y) + row * (long long)c + at, h, c - (int)at);
            }
        } else {
            uint8_t* y = static_cast<uint8_t*>(p.y) + row * (long long)c;
            const int lanes = p.group >> 3;
            const long long groups = p.group ? (c + p.group - 1) / p.group : 1;
            const Split split = split_of(rstd);
            float low[8];
            const auto scaled = [&](int col) __attribute__((always_inline)) {        // g of the above; returns the largest magnitude
                Packed<float> g;
                lc_load8(g, p.gamma, col, c);
                value(col, h, false);
                float m = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float n = h[j] * split.power, a = n * g.get(j);
                    low[j] = fmaf(n, g.get(j), -a);
                    h[j] = a;
                    m = fmaxf(m, fabsf(a));
                }
                return m;
            };
            Scale scale;
            if (p.group == 0) {
                float m = 0.f;
                for (long long at = tid * 8; at < c; at += kSpan) m = fmaxf(m, scaled((int)at));
                scale = scale_of(lc_block_max<WAVES>(m, red[parity][1]), split.rest);
                if (tid == 0) p.scales[row] = scale.scale;
            }
            for (long long base = 0; base < c; base += kSpan) {     // every lane of a group takes part in its maximum
                const long long at = base + tid * 8;
                const int col = at < c ? (int)at : c;
                float m = scaled(col);
                if (p.group) {
                    for (int off = 1; off < lanes; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
                    scale = scale_of(m, split.rest);
                    if (col < c && (tid & (lanes - 1)) == 0) p.scales[row * groups + col / p.group] = scale.scale;
                }
                store8_e4m3(y + col, h, low, scale, split.rest, c - col);
            }
        }
    }
}

struct NormBwdArgs {
    const void* h;
    const void* dy;
    const void* dh;          // or null
    const float* gamma;
    const float* rstd;
    void* dx;
    float* part;             // [blocks][c]: each block's rows' share of dgamma
    long long rows, h_ld;
    int c;
};

// A block walks rows blockIdx, blockIdx + gridDim, ...; a thread's columns stay the same, so that its share of dgamma stays in registers and no atomics are needed, and the next row's loads
// are under way while one is summed.  Bound by memory: 8192 rows of 4096 bf16 with three inputs and dx 43 us, 6.2 TB/s; 1003 rows of 1537 fp32 7 to 8 us, of which the launch and the
// latency of four rows one after another are most.
template <typename T, int CH, bool NT, Ends ENDS, int LANES = 0>
__global__ void __launch_bounds__(LANES ? kNarrowThreads : kMostWaves * 64) rmsnorm_bwd_kernel(const NormBwdArgs p) {
    __shared__ float red[2][kMostWaves];
    using Of = Rows<LANES>;
    const int tid = Of::tid(), c = p.c, waves = blockDim.x >> 6, threads = LANES ? LANES : blockDim.x;
    const auto column = [=](int i) { return (i * threads + tid) * 8; };
    const auto inside = [&](int i) { return ENDS == kWhole ? 8 : ENDS == kEights ? (column(i) < c ? 8 : 0) : c - column(i); };
    Packed<float> pg[CH];
    float acc[CH][8] = {};
    lc_issue8<ENDS>(pg, p.gamma, column, c);
    lc_settle8<ENDS>(pg, column, c);
    // the next row's loads are under way while this one is summed and written
    Packed<T> ph[CH], pd[CH], pt[CH], nh[CH], nd[CH], nt[CH];
    float rstd = 0.f, next_rstd = 0.f;
    const auto issue = [&](long long row) __attribute__((always_inline)) {
        lc_issue8<ENDS, NT>(nh, static_cast<const T*>(p.h) + row * p.h_ld, column, c);
        lc_issue8<ENDS, NT>(nd, static_cast<const T*>(p.dy) + row * (long long)c, column, c);
        if (p.dh) lc_issue8<ENDS, NT>(nt, static_cast<const T*>(p.dh) + row * (long long)c, column, c);
        next_rstd = p.rstd[row];
    };
    int parity = 0;
    if (Of::first() < p.rows) issue(Of::first());
    for (long long row = Of::first(); row < p.rows; row += Of::step(), parity ^= 1) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            ph[i] = nh[i];
            pd[i] = nd[i];
            pt[i] = nt[i];
        }
        rstd = next_rstd;
        if (row + Of::step() < p.rows) issue(row + Of::step());
        float s = 0.f;
        lc_settle8<ENDS>(ph, column, c);
        lc_settle8<ENDS>(pd, column, c);
        if (p.dh) lc_settle8<ENDS>(pt, column, c);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = ph[i].get(j) * rstd, d = pd[i].get(j);
                s = fmaf(d * pg[i].get(j), n, s);
                acc[i][j] = fmaf(d, n, acc[i][j]);
            }
        const float mean = Of::join(s, waves, red[parity], [](float a) { return lc_wave_sum(a); }, [](float a, float b) { return a + b; }) / (float)c;
        T* dx = static_cast<T*>(p.dx) + row * (long long)c;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = ph[i].get(j) * rstd;
                o[j] = (pd[i].get(j) * pg[i].get(j) - n * mean) * rstd;
            }
            if (p.dh) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += pt[i].get(j);
            }
            lc_store8<NT>(dx + column(i), o, inside(i));
        }
    }
    float* part = p.part + (long long)blockIdx.x * c;
    if constexpr (LANES == 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) lc_store8(part + column(i), acc[i], inside(i));
    } else {                                    // the block's rows in a fixed order: those of a wave, then the waves
        __shared__ float share[kNarrowThreads / 64][LANES * 8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            for (int off = LANES; off < 64; off <<= 1) acc[0][j] += __shfl_xor(acc[0][j], off, 64);
            if ((threadIdx.x & 63) < LANES) share[threadIdx.x >> 6][tid * 8 + j] = acc[0][j];
        }
        __syncthreads();
        if (threadIdx.x < c) part[threadIdx.x] = (share[0][threadIdx.x] + share[1][threadIdx.x]) + (share[2][threadIdx.x] + share[3][threadIdx.x]);
    }
}

// Wide rows: dgamma's shares by column tiles and ranges of rows (blockIdx.y), and dx in two passes over a row.
template <typename T>
__global__ void __launch_bounds__(256) rmsnorm_dgamma_wide_kernel(const NormBwdArgs p) {
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= p.c) return;
    const int col = (int)at;
    float acc[8] = {};
    for (long long row = blockIdx.y; row < p.rows; row += gridDim.y) {
        Packed<T> h, d;
        lc_load8(h, static_cast<const T*>(p.h) + row * p.h_ld, col, p.c);
        lc_load8(d, static_cast<const T*>(p.dy) + row * (long long)p.c, col, p.c);
        const float rstd = p.rstd[row];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = fmaf(d.get(j), h.get(j) * rstd, acc[j]);
    }
    lc_store8(p.part + (long long)blockIdx.y * p.c + col, acc, p.c - col);
}

template <typename T>
__global__ void __launch_bounds__(1024) rmsnorm_bwd_wide_kernel(const NormBwdArgs p) {
    constexpr int WAVES = 16, kSpan = WAVES * 64 * 8;
    __shared__ float red[2][WAVES];
    const int tid = threadIdx.x, c = p.c;
    int parity = 0;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x, parity ^= 1) {
        const T* h = static_cast<const T*>(p.h) + row * p.h_ld;
        const T* dy = static_cast<const T*>(p.dy) + row * (long long)c;
        const T* dh = p.dh ? static_cast<const T*>(p.dh) + row * (long long)c : nullptr;
        T* dx = static_cast<T*>(p.dx) + row * (long long)c;
        const float rstd = p.rstd[row];
        Packed<T> a, b, t;
        Packed<float> g;
        float s = 0.f;
        for (long long at = tid * 8; at < c; at += kSpan) {
            lc_load8(a, h, (int)at, c);
            lc_load8(b, dy, (int)at, c);
            lc_load8(g, p.gamma, (int)at, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) s = fmaf(b.get(j) * g.get(j), a.get(j) * rstd, s);
        }
        const float mean = lc_block_sum<WAVES>(s, red[parity]) / (float)c;
        for (long long at = tid * 8; at < c; at += kSpan) {
            lc_load8(a, h, (int)at, c);
            lc_load8(b, dy, (int)at, c);
            lc_load8(g, p.gamma, (int)at, c);
            if (dh) lc_load8(t, dh, (int)at, c);
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[j] = (b.get(j) * g.get(j) - a.get(j) * rstd * mean) * rstd;
                if (dh) o[j] += t.get(j);
            }
            lc_store8(dx + at, o, c - (int)at);
        }
    }
}

lc_status check_desc(const lc_rmsnorm_desc* d) {
    if (!d) return LC_ERR_NULL;
    if (d->dtype != LC_F32 && d->dtype != LC_BF16) return LC_ERR_UNSUPPORTED;
    if (d->rows < 0 || d->c <= 0 || d->c > kMostWidth) return LC_ERR_SHAPE;
    if ((d->x_ld && d->x_ld < d->c) || (d->residual_ld && d->residual_ld < d->c)) return LC_ERR_SHAPE;
    const long long widest = std::max<long long>({d->c, d->x_ld, d->residual_ld});
    long long bytes;
    if (__builtin_mul_overflow((long long)d->rows, widest, &bytes) || __builtin_mul_overflow(bytes, 4ll, &bytes)) return LC_ERR_SHAPE;
    if (!(d->eps >= 0.f)) return LC_ERR_UNSUPPORTED;
    return LC_OK;
}

template <typename T, int CH, bool Q8, bool NT>
void launch_fwd(const NormArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)std::min(a.rows, kMostBlocks)), block((a.c + 512 * CH - 1) / (512 * CH) * 64);
    if (a.c % (512 * CH) == 0) hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, CH, Q8, NT, kWhole>), grid, block, 0, stream, a);
    else if (a.c % 8 == 0) hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, CH, Q8, NT, kEights>), grid, block, 0, stream, a);
    else if constexpr (CH * sizeof(T) < 8) hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, CH, Q8, NT, kAny>), grid, block, 0, stream, a);
}
template <typename T, bool Q8, bool NT, int LANES>
void launch_fwd_narrow(const NormArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)std::min((a.rows + Rows<LANES>::kEach - 1) / Rows<LANES>::kEach, kMostBlocks)), block(kNarrowThreads);
    if (a.c % 8 == 0) hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, 1, Q8, NT, kEights, LANES>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, 1, Q8, NT, kAny, LANES>), grid, block, 0, stream, a);
}
template <typename T, bool Q8, bool NT>
void launch_fwd_narrow(const NormArgs& a, hipStream_t stream) {
    const int lanes = lanes_of(a.c);
    lanes == 8 ? launch_fwd_narrow<T, Q8, NT, 8>(a, stream) : lanes == 16 ? launch_fwd_narrow<T, Q8, NT, 16>(a, stream) : launch_fwd_narrow<T, Q8, NT, 32>(a, stream);
}

template <typename T, bool Q8>
void launch_fwd(const NormArgs& a, hipStream_t stream) {
    if (in_passes(sizeof(T) == 2 ? LC_BF16 : LC_F32, a.c)) {
        hipLaunchKernelGGL((rmsnorm_fwd_wide_kernel<T, Q8>), dim3((unsigned)std::min(a.rows, kMostBlocks)), dim3(1024), 0, stream, a);
        return;
    }
    if constexpr (sizeof(T) == 2) {
        const long long bytes = a.rows * a.c * (2 + (a.r ? 2 : 0) + (a.total ? 2 : 0) + (Q8 ? 1 : 2));
        if (bytes >= kStreamBytes && narrow(a.rows, a.c)) return launch_fwd_narrow<T, Q8, true>(a, stream);
        if (bytes >= kStreamBytes) return chunks_of<T>(a.c) == 1 ? launch_fwd<T, 1, Q8, true>(a, stream) : launch_fwd<T, 2, Q8, true>(a, stream);
    }
    if (narrow(a.rows, a.c)) return launch_fwd_narrow<T, Q8, false>(a, stream);
    chunks_of<T>(a.c) == 1 ? launch_fwd<T, 1, Q8, false>(a, stream) : launch_fwd<T, 2, Q8, false>(a, stream);
}

lc_status run_fwd(const lc_rmsnorm_desc* d, const void* x, const void* residual, const float* gamma, void* total, void* y, float* scales,
                  int group, float* save_rstd, bool q8, void* hip_stream) {
    const lc_status st = check_desc(d);
    if (st != LC_OK) return st;
    if (q8 && group != 0 && (group < 32 || group > 512 || (group & (group - 1)))) return LC_ERR_UNSUPPORTED;
    if (!residual && total) return LC_ERR_UNSUPPORTED;
    if (d->rows == 0) return LC_OK;
    if (!x || !gamma || !y || (q8 && !scales)) return LC_ERR_NULL;
    const size_t e = d->dtype == LC_BF16 ? 2 : 4;
    if (lc_off_element(x, e) || lc_off_element(residual, e) || lc_off_element(total, e) || (!q8 && lc_off_element(y, e)) ||
        lc_off_element(gamma, 4) || lc_off_element(scales, 4) || lc_off_element(save_rstd, 4))
        return LC_ERR_ALIGN;
    NormArgs a{x, residual, gamma, total, y, scales, save_rstd, d->rows, d->x_ld ? d->x_ld : d->c, d->residual_ld ? d->residual_ld : d->c,
               d->c, group, d->eps, 1.0 / d->c};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    lc_begin_call();
    if (d->dtype == LC_BF16) q8 ? launch_fwd<uint16_t, true>(a, stream) : launch_fwd<uint16_t, false>(a, stream);
    else q8 ? launch_fwd<float, true>(a, stream) : launch_fwd<float, false>(a, stream);
    return lc_end_call();
}

template <typename T, int CH, bool NT>
void launch_bwd(const NormBwdArgs& a, int blocks, hipStream_t stream) {
    const dim3 grid((unsigned)blocks), block((a.c + 512 * CH - 1) / (512 * CH) * 64);
    if (a.c % (512 * CH) == 0) hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, CH, NT, kWhole>), grid, block, 0, stream, a);
    else if (a.c % 8 == 0) hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, CH, NT, kEights>), grid, block, 0, stream, a);
    else if constexpr (CH * sizeof(T) < 8) hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, CH, NT, kAny>), grid, block, 0, stream, a);
}
template <typename T, bool NT, int LANES>
void launch_bwd_narrow(const NormBwdArgs& a, int blocks, hipStream_t stream) {
    if (a.c % 8 == 0) hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, 1, NT, kEights, LANES>), dim3((unsigned)blocks), dim3(kNarrowThreads), 0, stream, a);
    else hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, 1, NT, kAny, LANES>), dim3((unsigned)blocks), dim3(kNarrowThreads), 0, stream, a);
}
template <typename T, bool NT>
void launch_bwd_narrow(const NormBwdArgs& a, int blocks, hipStream_t stream) {
    const int lanes = lanes_of(a.c);
    lanes == 8 ? launch_bwd_narrow<T, NT, 8>(a, blocks, stream) : lanes == 16 ? launch_bwd_narrow<T, NT, 16>(a, blocks, stream) : launch_bwd_narrow<T, NT, 32>(a, blocks, stream);
}
template <typename T>
void launch_bwd(const NormBwdArgs& a, int blocks, hipStream_t stream) {
    if (in_passes(sizeof(T) == 2 ? LC_BF16 : LC_F32, a.c)) {
        hipLaunchKernelGGL((rmsnorm_dgamma_wide_kernel<T>), dim3((unsigned)(((long long)a.c + 2047) / 2048), (unsigned)blocks), dim3(256), 0, stream, a);
        hipLaunchKernelGGL((rmsnorm_bwd_wide_kernel<T>), dim3((unsigned)std::min(a.rows, kMostBlocks)), dim3(1024), 0, stream, a);
        return;
    }
    if constexpr (sizeof(T) == 2) {
        if (a.rows * a.c * (a.dh ? 8 : 6) >= kStreamBytes && narrow(a.rows, a.c)) return launch_bwd_narrow<T, true>(a, blocks, stream);
        if (a.rows * a.c * (a.dh ? 8 : 6) >= kStreamBytes) return bwd_chunks(a.c) == 1 ? launch_bwd<T, 1, true>(a, blocks, stream) : launch_bwd<T, 2, true>(a, blocks, stream);
    }
    if (narrow(a.rows, a.c)) return launch_bwd_narrow<T, false>(a, blocks, stream);
    bwd_chunks(a.c) == 1 ? launch_bwd<T, 1, false>(a, blocks, stream) : launch_bwd<T, 2, false>(a, blocks, stream);
}

}  // namespace

extern "C" lc_status rmsnorm_fwd(const lc_rmsnorm_desc* desc, const void* x, const void* residual, const float* gamma, void* total, void* y,
                                 float* save_rstd, void* hip_stream) {
    return run_fwd(desc, x, residual, gamma, total, y, nullptr, 0, save_rstd, false, hip_stream);
}

extern "C" lc_status rmsnorm_fwd_q8(const lc_rmsnorm_desc* desc, const void* x, const void* residual, const float* gamma, void* total,
                                    uint8_t* y8, float* scales, int group, float* save_rstd, void* hip_stream) {
    return run_fwd(desc, x, residual, gamma, total, y8, scales, group, save_rstd, true, hip_stream);
}

extern "C" size_t rmsnorm_bwd_workspace_bytes(const lc_rmsnorm_desc* desc) {
    if (check_desc(desc) != LC_OK) return 0;
    return ((size_t)bwd_blocks(desc->dtype, desc->rows, desc->c) * desc->c * sizeof(float) + 255) & ~(size_t)255;
}

extern "C" lc_status rmsnorm_bwd(const lc_rmsnorm_desc* desc, const void* total, int64_t h_ld, const void* dy, const void* dtotal,
                                 const float* gamma, const float* save_rstd, void* dx, float* dgamma, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
    const lc_status st = check_desc(desc);
    if (st != LC_OK) return st;
    if (h_ld && h_ld < desc->c) return LC_ERR_SHAPE;
    long long span;
    if (__builtin_mul_overflow((long long)desc->rows, (long long)h_ld, &span) || __builtin_mul_overflow(span, 4ll, &span)) return LC_ERR_SHAPE;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (!dgamma) return LC_ERR_NULL;
    if (lc_off_element(dgamma, 4)) return LC_ERR_ALIGN;
    if (desc->rows == 0) {                   // a sum over no rows
        lc_begin_call();
        lc_fill_f32(dgamma, 0.f, (size_t)desc->c, stream);
        return lc_end_call();
    }
    if (!total || !dy || !gamma || !save_rstd || !dx) return LC_ERR_NULL;
    const size_t e = desc->dtype == LC_BF16 ? 2 : 4;
    if (lc_off_element(total, e) || lc_off_element(dy, e) || lc_off_element(dtotal, e) || lc_off_element(dx, e) || lc_off_element(gamma, 4) ||
        lc_off_element(save_rstd, 4))
        return LC_ERR_ALIGN;
    if (!workspace || (((uintptr_t)workspace) & 255) || workspace_bytes < rmsnorm_bwd_workspace_bytes(desc)) return LC_ERR_WORKSPACE;
    const int blocks = (int)bwd_blocks(desc->dtype, desc->rows, desc->c);
    NormBwdArgs a{total, dy, dtotal, gamma, save_rstd, dx, static_cast<float*>(workspace), desc->rows, h_ld ? h_ld : desc->c, desc->c};
    lc_begin_call();
    if (desc->dtype == LC_BF16) launch_bwd<uint16_t>(a, blocks, stream);
    else launch_bwd<float>(a, blocks, stream);
    sum_parts(a.part, dgamma, nullptr, blocks, desc->c, stream);
    return lc_end_call();
}
