// Layer norm with the residual's addition, and its gradient, for gfx950.
//
// total = x + residual, mean and variance over the row, rstd = 1/sqrt(variance + eps), n = (total - mean) * rstd, y = n * gamma + beta; with a = dy * gamma,
// dx = rstd * (a - mean(a) - n * mean(a * n)) + dtotal, dgamma = sum over rows of dy * n, dbeta = sum over rows of dy.  Bound by memory, as the RMS norm (rmsnorm.hip), whose
// division of rows over threads it has: a row is read once into registers.  A wave's sum gives a mean near its own; deviations from it are summed with their squares, and what their sum says
// that mean lacks is taken off both, so that a mean far from zero costs no places; waves are then joined by their means' differences, with one barrier a row.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "norm_common.h"
#include "token_common.h"

namespace {

struct LayerArgs {
    const void* x;
    const void* r;           // residual or null
    const float* gamma;
    const float* beta;       // or null
    void* total;             // or null
    void* y;
    float* mean;             // or null
    float* rstd;             // or null
    long long rows, x_ld, r_ld;
    int c;
    float eps;
    double inv_c;            // 1 / c
};

// 1/sqrt(x) to more than fp32's places over double's range: the instruction's estimate near one and one step of Newton's method in double.
__device__ __forceinline__ double inverse_root(double x) {
    const int half = __builtin_amdgcn_frexp_exp(x) >> 1;
    const double near = ldexp(x, -2 * half), r = (double)__builtin_amdgcn_rsqf((float)near);
    const double better = r * fma(-0.5 * near * r, r, 1.5);
    return ldexp(fabs(better) < INFINITY ? better : r, -half);         // (x = 0 or infinite: the estimate is the value)
}

// What deviations from a mean near the row's, `first`, say: `lack`, what the row's mean is above it, and the inverse deviation.  All in units of 2^e.
struct Moments {
    float first, lack, n_scale;      // n = (total / 2^e - first - lack) * n_scale
    double mean, rstd;
};
__device__ __forceinline__ Moments moments_of(const LayerArgs& p, float first, float lack, float squares, int e) {
    Moments m;
    const double var = fmax((double)squares * p.inv_c, (double)squares * 0.0);         // (rounding leaves nothing under zero; a NaN stays one)
    m.first = first;
    m.lack = lack;
    m.mean = ldexp((double)first + (double)lack, e);
    m.rstd = inverse_root(ldexp(var, 2 * e) + (double)p.eps);
    m.n_scale = (float)ldexp(m.rstd, e);
    return m;
}
// Whether deviations squared as they are say enough: their sum is finite, and either eps hides what they lose under fp32's normal range or none does.  Other rows are summed again
// as totals / 2^e with 2^e above the largest.
__device__ __forceinline__ bool squares_serve(const LayerArgs& p, float squares) { return squares < INFINITY && (p.eps >= 0x1p-120f || squares >= 0x1p-90f); }

// A sum, or two at once, over the threads of a row.
template <typename Of>
__device__ __forceinline__ float row_sum(float a, int waves, float* red) {
    return Of::join(a, waves, red, [](float v) { return lc_wave_sum(v); }, [](float u, float v) { return u + v; });
}
template <typename Of>
__device__ __forceinline__ float row_max(float a, int waves, float* red) {
    return Of::join(a, waves, red, [](float v) { return lc_wave_max(v); }, [](float u, float v) { return fmaxf(u, v); });
}
template <int LANES>
__device__ __forceinline__ void row_sums(float& a, float& b, int waves, float (*red)[kMostWaves]) {
    if constexpr (LANES == 0) {
        a = lc_wave_sum(a);
        b = lc_wave_sum(b);
        if (waves == 1) return;
        if ((threadIdx.x & 63) == 0) {
            red[0][threadIdx.x >> 6] = a;
            red[1][threadIdx.x >> 6] = b;
        }
        __syncthreads();
        a = red[0][0];
        b = red[1][0];
        for (int w = 1; w < waves; ++w) {
            a += red[0][w];
            b += red[1][w];
        }
    } else {
#pragma unroll
        for (int off = 1; off < LANES; off <<= 1) {
            a += __shfl_xor(a, off, 64);
            b += __shfl_xor(b, off, 64);
        }
    }
}

// A block walks rows blockIdx, blockIdx + gridDim, ... (LANES: narrow ones, several of a wave), with scale and shift in its registers and the next row's loads under way.  8192 x 4096 bf16 with the residual 48 us
// (268 MB, 5.6 TB/s), 65536 x 256 23 to 26, one row 2.5, a launch.  NT, ENDS: as the RMS norm's.
template <typename T, int CH, bool NT, Ends ENDS, int LANES = 0>
__global__ void __launch_bounds__(LANES ? kNarrowThreads : kMostWaves * 64) layernorm_fwd_kernel(const LayerArgs p) {
    __shared__ float red[2][7][kMostWaves];
    using Of = Rows<LANES>;
    const int tid = Of::tid(), c = p.c, waves = blockDim.x >> 6, threads = LANES ? LANES : blockDim.x;
    const auto column = [=](int i) { return (i * threads + tid) * 8; };
    const auto inside = [&](int i) { return ENDS == kWhole ? 8 : ENDS == kEights ? (column(i) < c ? 8 : 0) : c - column(i); };
    Packed<T> px[CH], pr[CH], nx[CH], nr[CH];
    Packed<float> pg[CH], pb[CH];
    const auto issue = [&](long long row) __attribute__((always_inline)) {
        lc_issue8<ENDS, NT>(nx, static_cast<const T*>(p.x) + row * p.x_ld, column, c);
        if (p.r) lc_issue8<ENDS, NT>(nr, static_cast<const T*>(p.r) + row * p.r_ld, column, c);
    };
    if (Of::first() < p.rows) issue(Of::first());
    lc_issue8<ENDS>(pg, p.gamma, column, c);
    if (p.beta) lc_issue8<ENDS>(pb, p.beta, column, c);
    lc_settle8<ENDS>(pg, column, c);
    if (p.beta) lc_settle8<ENDS>(pb, column, c);
    int parity = 0;
    for (long long row = Of::first(); row < p.rows; row += Of::step(), parity ^= 1) {
        float h[CH][8];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            px[i] = nx[i];
            pr[i] = nr[i];
        }
        if (row + Of::step() < p.rows) issue(row + Of::step());
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
        if (p.total) {
            T* t = static_cast<T*>(p.total) + row * (long long)c;
#pragma unroll
            for (int i = 0; i < CH; ++i) lc_store8<NT>(t + column(i), h[i], inside(i));
        }
        const auto sum_of = [&]() __attribute__((always_inline)) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) s += h[i][j];
            return s;
        };
        const auto deviations = [&](float from, float& sum, float& squares) __attribute__((always_inline)) {        // h becomes its deviation; what lies past the row stays 0
            sum = squares = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    h[i][j] = ENDS == kWhole || j < inside(i) ? h[i][j] - from : 0.f;
                    sum += h[i][j];
                    squares = fmaf(h[i][j], h[i][j], squares);
                }
        };
        float first, sum, squares;
        if constexpr (LANES == 0) {
            // deviations from the wave's own mean; a block's waves are joined as sums of squares around means are: by what each mean is off the first wave's
            const auto columns_of = [&](int w) __attribute__((always_inline)) {
                int n = 0;
#pragma unroll
                for (int i = 0; i < CH; ++i) n += ENDS == kWhole ? 512 : min(max(c - (i * threads + w * 64) * 8, 0), 512);
                return (float)n;
            };
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
            first = lc_wave_sum(sum_of()) * __builtin_amdgcn_rcpf(columns_of(wave));
            deviations(first, sum, squares);
            sum = lc_wave_sum(sum);
            squares = lc_wave_sum(squares);
            if (waves > 1) {
                if (lane == 0) {
                    red[parity][0][wave] = first;
                    red[parity][1][wave] = sum;
                    red[parity][2][wave] = squares;
                }
                __syncthreads();
                const bool in = lane < waves;
                const float n = columns_of(lane), inv_n = __builtin_amdgcn_rcpf(n), base = red[parity][0][0], s = in ? red[parity][1][lane] : 0.f;
                const float off = in ? fmaf(s, inv_n, red[parity][0][lane] - base) : 0.f, all = (float)((double)lc_wave_sum(in ? off * n : 0.f) * p.inv_c), d = off - all;
                squares = lc_wave_sum(in ? fmaf(n * d, d, fmaf(-s * s, inv_n, red[parity][2][lane])) : 0.f);
                sum = (base - first) + all;         // the row's mean less the wave's
            } else {
                sum *= (float)p.inv_c;
                squares = fmaf(-sum * sum, (float)c, squares);
            }
        } else {
            first = (float)((double)row_sum<Of>(sum_of(), waves, red[parity][0]) * p.inv_c);
            deviations(first, sum, squares);
            row_sums<LANES>(sum, squares, waves, red[parity] + 1);
            sum *= (float)p.inv_c;
            squares = fmaf(-sum * sum, (float)c, squares);
        }
        Moments m;
        if (squares_serve(p, squares)) {
            m = moments_of(p, first, sum, squares, 0);
        } else {                                          // the row again, divided by a power of two
            float most = 0.f, again = 0.f;
            if (p.r) {
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
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(h[i][j]));
            const int e = __builtin_amdgcn_frexp_expf(row_max<Of>(most, waves, red[parity][3]));         // (0 for zero and infinity)
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    h[i][j] = ldexpf(h[i][j], -e);
                    again += h[i][j];
                }
            const float from = (float)((double)row_sum<Of>(again, waves, red[parity][4]) * p.inv_c);
            deviations(from, sum, squares);
            row_sums<LANES>(sum, squares, waves, red[parity] + 5);
            sum *= (float)p.inv_c;
            m = moments_of(p, from, sum, fmaf(-sum * sum, (float)c, squares), e);
        }
        if (tid == 0) {
            if (p.mean) p.mean[row] = (float)m.mean;
            if (p.rstd) p.rstd[row] = (float)m.rstd;
        }
        T* y = static_cast<T*>(p.y) + row * (long long)c;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = (h[i][j] - m.lack) * m.n_scale;
                h[i][j] = p.beta ? fmaf(n, pg[i].get(j), pb[i].get(j)) : n * pg[i].get(j);
            }
            lc_store8<NT>(y + column(i), h[i], inside(i));
        }
    }
}

// Rows too wide for the registers of a block, or under eight columns: the same in passes over the row, which the caches hold.
template <typename T>
__global__ void __launch_bounds__(1024) layernorm_fwd_wide_kernel(const LayerArgs p) {
    constexpr int WAVES = 16, kSpan = WAVES * 64 * 8;
    __shared__ float red[2][7][WAVES];
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
        float s = 0.f, h[8];
        for (long long at = tid * 8; at < c; at += kSpan) {
            const int col = (int)at;
            value(col, h, true);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += h[j];
            if (t) lc_store8(t + col, h, c - col);
        }
        const auto over = [&](auto&& f) __attribute__((always_inline)) {
            for (long long at = tid * 8; at < c; at += kSpan) {
                value((int)at, h, false);
                const int n = min(8, c - (int)at);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) f(h[j]);
            }
        };
        float sum = 0.f, squares = 0.f;
        const auto deviations = [&](float from, int e) __attribute__((always_inline)) {
            sum = squares = 0.f;
            over([&](float v) __attribute__((always_inline)) {
                const float d = ldexpf(v, -e) - from;
                sum += d;
                squares = fmaf(d, d, squares);
            });
        };
        float first = (float)((double)lc_block_sum<WAVES>(s, red[parity][0]) * p.inv_c);
        int e = 0;
        deviations(first, 0);
        row_sums<0>(sum, squares, WAVES, red[parity] + 1);
        if (!squares_serve(p, squares)) {
            float most = 0.f, again = 0.f;
            over([&](float v) __attribute__((always_inline)) { most = fmaxf(most, fabsf(v)); });
            e = __builtin_amdgcn_frexp_expf(lc_block_max<WAVES>(most, red[parity][3]));
            over([&](float v) __attribute__((always_inline)) { again += ldexpf(v, -e); });
            first = (float)((double)lc_block_sum<WAVES>(again, red[parity][4]) * p.inv_c);
            deviations(first, e);
            row_sums<0>(sum, squares, WAVES, red[parity] + 5);
        }
        sum *= (float)p.inv_c;
        const Moments m = moments_of(p, first, sum, fmaf(-sum * sum, (float)c, squares), e);
        if (tid == 0) {
            if (p.mean) p.mean[row] = (float)m.mean;
            if (p.rstd) p.rstd[row] = (float)m.rstd;
        }
        for (long long at = tid * 8; at < c; at += kSpan) {
            Packed<float> g, b;
            lc_load8(g, p.gamma, (int)at, c);
            if (p.beta) lc_load8(b, p.beta, (int)at, c);
            value((int)at, h, false);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = ((ldexpf(h[j], -e) - m.first) - m.lack) * m.n_scale;
                h[j] = p.beta ? fmaf(n, g.get(j), b.get(j)) : n * g.get(j);
            }
            lc_store8(static_cast<T*>(p.y) + row * (long long)c + at, h, c - (int)at);
        }
    }
}

struct LayerBwdArgs {
    const void* h;
    const void* dy;
    const void* dh;          // or null
    const float* gamma;
    const float* mean;
    const float* rstd;
    void* dx;
    float* part;             // [blocks][width]: each block's rows' share of dgamma, behind it (width 2 c) of dbeta
    long long rows, h_ld, width;
    int c;
};

// n of a row's values from its saved statistics, (h - mean) * rstd.  Where deviations may leave fp32 (one over 2^127 in a row of up to 2^30 values takes rstd under 2^-112) h and mean are a quarter and rstd four times what they are;
// elsewhere the same bits as without (h times 1 is exact, and the operation as long as a subtraction).
template <bool SAME>                                                // the row is the same for a wave
struct Centred {
    float part, mean, n_scale;
    __device__ __forceinline__ Centred(float mean, float rstd) : part(rstd < 0x1p-100f ? 0.25f : 1.f), mean(mean * part), n_scale(rstd < 0x1p-100f ? 4.f * rstd : rstd) {
        if constexpr (SAME) part = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(part)));
    }
    __device__ __forceinline__ float operator()(float h) const { return fmaf(h, part, -mean) * n_scale; }
    __device__ __forceinline__ float rstd() const { return n_scale * part; }
};

// A block walks rows blockIdx, blockIdx + gridDim, ...; a thread's columns stay the same, so that its shares of dgamma and dbeta stay in registers and no atomics are needed, and the next
// row's loads are under way while one is summed.  8192 x 4096 bf16 46 us (268 MB, 5.8 TB/s), 65536 x 256 26, and 4.7 for the sum of the blocks' shares.
template <typename T, int CH, bool NT, Ends ENDS, int LANES = 0>
__global__ void __launch_bounds__(LANES ? kNarrowThreads : kMostWaves * 64) layernorm_bwd_kernel(const LayerBwdArgs p) {
    __shared__ float red[2][2][kMostWaves];
    using Of = Rows<LANES>;
    const int tid = Of::tid(), c = p.c, waves = blockDim.x >> 6, threads = LANES ? LANES : blockDim.x;
    const auto column = [=](int i) { return (i * threads + tid) * 8; };
    const auto inside = [&](int i) { return ENDS == kWhole ? 8 : ENDS == kEights ? (column(i) < c ? 8 : 0) : c - column(i); };
    const float inv_c = 1.f / (float)c;
    Packed<float> pg[CH];
    float acc[CH][8] = {}, shift[CH][8] = {};
    lc_issue8<ENDS>(pg, p.gamma, column, c);
    lc_settle8<ENDS>(pg, column, c);
    Packed<T> ph[CH], pd[CH], pt[CH], nh[CH], nd[CH], nt[CH];
    float next_rstd = 0.f, next_mean = 0.f;
    const auto issue = [&](long long row) __attribute__((always_inline)) {
        lc_issue8<ENDS, NT>(nh, static_cast<const T*>(p.h) + row * p.h_ld, column, c);
        lc_issue8<ENDS, NT>(nd, static_cast<const T*>(p.dy) + row * (long long)c, column, c);
        if (p.dh) lc_issue8<ENDS, NT>(nt, static_cast<const T*>(p.dh) + row * (long long)c, column, c);
        next_rstd = p.rstd[row];
        next_mean = p.mean[row];
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
        const Centred<LANES == 0> n_of(next_mean, next_rstd);
        if (row + Of::step() < p.rows) issue(row + Of::step());
        float s = 0.f, sn = 0.f;
        lc_settle8<ENDS>(ph, column, c);
        lc_settle8<ENDS>(pd, column, c);              // (dy past the row is 0: nothing there counts)
        if (p.dh) lc_settle8<ENDS>(pt, column, c);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = n_of(ph[i].get(j)), d = pd[i].get(j), a = d * pg[i].get(j);
                s += a;
                sn = fmaf(a, n, sn);
                acc[i][j] = fmaf(d, n, acc[i][j]);
                shift[i][j] += d;
            }
        row_sums<LANES>(s, sn, waves, red[parity]);
        s *= inv_c;
        sn *= inv_c;
        T* dx = static_cast<T*>(p.dx) + row * (long long)c;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = n_of(ph[i].get(j));
                o[j] = ((pd[i].get(j) * pg[i].get(j) - s) - n * sn) * n_of.rstd();
            }
            if (p.dh) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += pt[i].get(j);
            }
            lc_store8<NT>(dx + column(i), o, inside(i));
        }
    }
    float* part = p.part + (long long)blockIdx.x * p.width;
    const bool shifts = p.width > c;
    if constexpr (LANES == 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            lc_store8(part + column(i), acc[i], inside(i));
            if (shifts) lc_store8(part + c + column(i), shift[i], inside(i));
        }
    } else {                                    // the block's rows in a fixed order: those of a wave, then the waves
        __shared__ float share[2][kNarrowThreads / 64][LANES * 8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            for (int off = LANES; off < 64; off <<= 1) {
                acc[0][j] += __shfl_xor(acc[0][j], off, 64);
                shift[0][j] += __shfl_xor(shift[0][j], off, 64);
            }
            if ((threadIdx.x & 63) < LANES) {
                share[0][threadIdx.x >> 6][tid * 8 + j] = acc[0][j];
                share[1][threadIdx.x >> 6][tid * 8 + j] = shift[0][j];
            }
        }
        __syncthreads();
        if (threadIdx.x < c) {
            for (int k = 0; k < (shifts ? 2 : 1); ++k)
                part[k * c + threadIdx.x] = (share[k][0][threadIdx.x] + share[k][1][threadIdx.x]) + (share[k][2][threadIdx.x] + share[k][3][threadIdx.x]);
        }
    }
}

// Wide rows: the shares of dgamma and dbeta by column tiles and ranges of rows (blockIdx.y), and dx in two passes over a row.
template <typename T>
__global__ void __launch_bounds__(256) layernorm_parts_wide_kernel(const LayerBwdArgs p) {
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= p.c) return;
    const int col = (int)at;
    float acc[8] = {}, shift[8] = {};
    for (long long row = blockIdx.y; row < p.rows; row += gridDim.y) {
        Packed<T> h, d;
        lc_load8(h, static_cast<const T*>(p.h) + row * p.h_ld, col, p.c);
        lc_load8(d, static_cast<const T*>(p.dy) + row * (long long)p.c, col, p.c);
        const Centred<true> n_of(p.mean[row], p.rstd[row]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            acc[j] = fmaf(d.get(j), n_of(h.get(j)), acc[j]);
            shift[j] += d.get(j);
        }
    }
    float* part = p.part + (long long)blockIdx.y * p.width + col;
    lc_store8(part, acc, p.c - col);
    if (p.width > p.c) lc_store8(part + p.c, shift, p.c - col);
}

template <typename T>
__global__ void __launch_bounds__(1024) layernorm_bwd_wide_kernel(const LayerBwdArgs p) {
    constexpr int WAVES = 16, kSpan = WAVES * 64 * 8;
    __shared__ float red[2][2][WAVES];
    const int tid = threadIdx.x, c = p.c;
    int parity = 0;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x, parity ^= 1) {
        const T* h = static_cast<const T*>(p.h) + row * p.h_ld;
        const T* dy = static_cast<const T*>(p.dy) + row * (long long)c;
        const T* dh = p.dh ? static_cast<const T*>(p.dh) + row * (long long)c : nullptr;
        T* dx = static_cast<T*>(p.dx) + row * (long long)c;
        const Centred<true> n_of(p.mean[row], p.rstd[row]);
        Packed<T> a, b, t;
        Packed<float> g;
        float s = 0.f, sn = 0.f;
        for (long long at = tid * 8; at < c; at += kSpan) {
            lc_load8(a, h, (int)at, c);
            lc_load8(b, dy, (int)at, c);
            lc_load8(g, p.gamma, (int)at, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = b.get(j) * g.get(j);
                s += d;
                sn = fmaf(d, n_of(a.get(j)), sn);
            }
        }
        row_sums<0>(s, sn, WAVES, red[parity]);
        s /= (float)c;
        sn /= (float)c;
        for (long long at = tid * 8; at < c; at += kSpan) {
            lc_load8(a, h, (int)at, c);
            lc_load8(b, dy, (int)at, c);
            lc_load8(g, p.gamma, (int)at, c);
            if (dh) lc_load8(t, dh, (int)at, c);
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[j] = ((b.get(j) * g.get(j) - s) - n_of(a.get(j)) * sn) * n_of.rstd();
                if (dh) o[j] += t.get(j);
            }
            lc_store8(dx + at, o, c - (int)at);
        }
    }
}

lc_status check_desc(const lc_layernorm_desc* d) {
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

// Blocks of the forward pass: as many waves as the chip holds at once, the same number of blocks for each of its 256 units.  us, bf16, with 4096 waves, 8192 and a block a row: 8192 x 4096 48.2, 48.6, 49.4,
// 2048 x 16384 51, 51, 59; fp32 7000 x 4096 81, 83, 86; 3000 x 10240 122, 117, 117.  (Scale and shift read again for every row: 53 for the first.)
constexpr int kFwdWaves = 8192, kUnits = 256;
long long fwd_blocks(int waves) { return std::max(kUnits, kFwdWaves / waves / kUnits * kUnits); }

// Blocks of the backward pass: the RMS norm's number, in multiples of the units where a block has whole rows.  us, bf16, forward and backward, the RMS norm's / so, both passes': 7084 rows of 1536 50 / 46.5, 2816 77.5 / 66.5,
// 5120 116 / 110, 6144 152 / 137, 7168 181 / 152, 10240 325 / 281; fp32 4000 x 6144 171 / 154, 16409 x 1344 152 / 148; 2048, 4096 and 8192 columns have the same blocks.  (The step from 7168 to 10240: over
// 8192 columns a thread has 16, whose scale, two sums, three operands and the next row's three are more than the 128 registers that 1024 threads leave: 35 to 117 are spilled, in fp32's forward pass 16 and 17.)
long long grad_blocks(lc_dtype dtype, long long rows, int c) {
    const long long blocks = bwd_blocks(dtype, rows, c);
    return in_passes(dtype, c) || narrow(rows, c) || blocks < kUnits ? blocks : blocks / kUnits * kUnits;
}

template <typename T, int CH, bool NT>
void launch_fwd(const LayerArgs& a, hipStream_t stream) {
    const int waves = (a.c + 512 * CH - 1) / (512 * CH);
    const dim3 grid((unsigned)std::min<long long>(a.rows, fwd_blocks(waves))), block(waves * 64);
    if (a.c % (512 * CH) == 0) hipLaunchKernelGGL((layernorm_fwd_kernel<T, CH, NT, kWhole>), grid, block, 0, stream, a);
    else if (a.c % 8 == 0) hipLaunchKernelGGL((layernorm_fwd_kernel<T, CH, NT, kEights>), grid, block, 0, stream, a);
    else if constexpr (CH * sizeof(T) < 8) hipLaunchKernelGGL((layernorm_fwd_kernel<T, CH, NT, kAny>), grid, block, 0, stream, a);
}
template <typename T, bool NT, int LANES>
void launch_fwd_narrow(const LayerArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)std::min<long long>((a.rows + Rows<LANES>::kEach - 1) / Rows<LANES>::kEach, fwd_blocks(4))), block(kNarrowThreads);
    if (a.c % 8 == 0) hipLaunchKernelGGL((layernorm_fwd_kernel<T, 1, NT, kEights, LANES>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((layernorm_fwd_kernel<T, 1, NT, kAny, LANES>), grid, block, 0, stream, a);
}
template <typename T, bool NT>
void launch_fwd_narrow(const LayerArgs& a, hipStream_t stream) {
    const int lanes = lanes_of(a.c);
    lanes == 8 ? launch_fwd_narrow<T, NT, 8>(a, stream) : lanes == 16 ? launch_fwd_narrow<T, NT, 16>(a, stream) : launch_fwd_narrow<T, NT, 32>(a, stream);
}
template <typename T>
void launch_fwd(const LayerArgs& a, hipStream_t stream) {
    if (in_passes(sizeof(T) == 2 ? LC_BF16 : LC_F32, a.c)) {
        hipLaunchKernelGGL((layernorm_fwd_wide_kernel<T>), dim3((unsigned)std::min(a.rows, kMostBlocks)), dim3(1024), 0, stream, a);
        return;
    }
    if constexpr (sizeof(T) == 2) {
        if (a.rows * a.c * (4 + (a.r ? 2 : 0) + (a.total ? 2 : 0)) >= kStreamBytes) {
            if (narrow(a.rows, a.c)) return launch_fwd_narrow<T, true>(a, stream);
            return chunks_of<T>(a.c) == 1 ? launch_fwd<T, 1, true>(a, stream) : launch_fwd<T, 2, true>(a, stream);
        }
    }
    if (narrow(a.rows, a.c)) return launch_fwd_narrow<T, false>(a, stream);
    chunks_of<T>(a.c) == 1 ? launch_fwd<T, 1, false>(a, stream) : launch_fwd<T, 2, false>(a, stream);
}

template <typename T, int CH, bool NT>
void launch_bwd(const LayerBwdArgs& a, int blocks, hipStream_t stream) {
    const dim3 grid((unsigned)blocks), block((a.c + 512 * CH - 1) / (512 * CH) * 64);
    if (a.c % (512 * CH) == 0) hipLaunchKernelGGL((layernorm_bwd_kernel<T, CH, NT, kWhole>), grid, block, 0, stream, a);
    else if (a.c % 8 == 0) hipLaunchKernelGGL((layernorm_bwd_kernel<T, CH, NT, kEights>), grid, block, 0, stream, a);
    else if constexpr (CH * sizeof(T) < 8) hipLaunchKernelGGL((layernorm_bwd_kernel<T, CH, NT, kAny>), grid, block, 0, stream, a);
}
template <typename T, bool NT, int LANES>
void launch_bwd_narrow(const LayerBwdArgs& a, int blocks, hipStream_t stream) {
    if (a.c % 8 == 0) hipLaunchKernelGGL((layernorm_bwd_kernel<T, 1, NT, kEights, LANES>), dim3((unsigned)blocks), dim3(kNarrowThreads), 0, stream, a);
    else hipLaunchKernelGGL((layernorm_bwd_kernel<T, 1, NT, kAny, LANES>), dim3((unsigned)blocks), dim3(kNarrowThreads), 0, stream, a);
}
template <typename T, bool NT>
void launch_bwd_narrow(const LayerBwdArgs& a, int blocks, hipStream_t stream) {
    const int lanes = lanes_of(a.c);
    lanes == 8 ? launch_bwd_narrow<T, NT, 8>(a, blocks, stream) : lanes == 16 ? launch_bwd_narrow<T, NT, 16>(a, blocks, stream) : launch_bwd_narrow<T, NT, 32>(a, blocks, stream);
}
template <typename T>
void launch_bwd(const LayerBwdArgs& a, int blocks, hipStream_t stream) {
    if (in_passes(sizeof(T) == 2 ? LC_BF16 : LC_F32, a.c)) {
        hipLaunchKernelGGL((layernorm_parts_wide_kernel<T>), dim3((unsigned)(((long long)a.c + 2047) / 2048), (unsigned)blocks), dim3(256), 0, stream, a);
        hipLaunchKernelGGL((layernorm_bwd_wide_kernel<T>), dim3((unsigned)std::min(a.rows, kMostBlocks)), dim3(1024), 0, stream, a);
        return;
    }
    if constexpr (sizeof(T) == 2) {
        if (a.rows * a.c * (a.dh ? 8 : 6) >= kStreamBytes) {
            if (narrow(a.rows, a.c)) return launch_bwd_narrow<T, true>(a, blocks, stream);
            return bwd_chunks(a.c) == 1 ? launch_bwd<T, 1, true>(a, blocks, stream) : launch_bwd<T, 2, true>(a, blocks, stream);
        }
    }
    if (narrow(a.rows, a.c)) return launch_bwd_narrow<T, false>(a, blocks, stream);
    bwd_chunks(a.c) == 1 ? launch_bwd<T, 1, false>(a, blocks, stream) : launch_bwd<T, 2, false>(a, blocks, stream);
}

}  // namespace

extern "C" lc_status layernorm_fwd(const lc_layernorm_desc* desc, const void* x, const void* residual, const float* gamma, const float* beta, void* total,
                                   void* y, float* save_mean, float* save_rstd, void* hip_stream) {
    const lc_status st = check_desc(desc);
    if (st != LC_OK) return st;
    if (!residual && total) return LC_ERR_UNSUPPORTED;
    if (desc->rows == 0) return LC_OK;
    if (!x || !gamma || !y) return LC_ERR_NULL;
    const size_t e = desc->dtype == LC_BF16 ? 2 : 4;
    if (lc_off_element(x, e) || lc_off_element(residual, e) || lc_off_element(total, e) || lc_off_element(y, e) || lc_off_element(gamma, 4) ||
        lc_off_element(beta, 4) || lc_off_element(save_mean, 4) || lc_off_element(save_rstd, 4))
        return LC_ERR_ALIGN;
    const LayerArgs a{x, residual, gamma, beta, total, y, save_mean, save_rstd, desc->rows, desc->x_ld ? desc->x_ld : desc->c,
                      desc->residual_ld ? desc->residual_ld : desc->c, desc->c, desc->eps, 1.0 / desc->c};
    lc_begin_call();
    if (desc->dtype == LC_BF16) launch_fwd<uint16_t>(a, static_cast<hipStream_t>(hip_stream));
    else launch_fwd<float>(a, static_cast<hipStream_t>(hip_stream));
    return lc_end_call();
}

extern "C" size_t layernorm_bwd_workspace_bytes(const lc_layernorm_desc* desc) {
    if (check_desc(desc) != LC_OK) return 0;
    return ((size_t)grad_blocks(desc->dtype, desc->rows, desc->c) * 2 * desc->c * sizeof(float) + 255) & ~(size_t)255;
}

extern "C" lc_status layernorm_bwd(const lc_layernorm_desc* desc, const void* total, int64_t h_ld, const void* dy, const void* dtotal, const float* gamma,
                                   const float* save_mean, const float* save_rstd, void* dx, float* dgamma, float* dbeta, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
    const lc_status st = check_desc(desc);
    if (st != LC_OK) return st;
    if (h_ld && h_ld < desc->c) return LC_ERR_SHAPE;
    long long span;
    if (__builtin_mul_overflow((long long)desc->rows, (long long)h_ld, &span) || __builtin_mul_overflow(span, 4ll, &span)) return LC_ERR_SHAPE;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (!dgamma) return LC_ERR_NULL;
    if (lc_off_element(dgamma, 4) || lc_off_element(dbeta, 4)) return LC_ERR_ALIGN;
    if (desc->rows == 0) {                   // sums over no rows
        lc_begin_call();
        lc_fill_f32(dgamma, 0.f, (size_t)desc->c, stream);
        if (dbeta) lc_fill_f32(dbeta, 0.f, (size_t)desc->c, stream);
        return lc_end_call();
    }
    if (!total || !dy || !gamma || !save_mean || !save_rstd || !dx) return LC_ERR_NULL;
    const size_t e = desc->dtype == LC_BF16 ? 2 : 4;
    if (lc_off_element(total, e) || lc_off_element(dy, e) || lc_off_element(dtotal, e) || lc_off_element(dx, e) || lc_off_element(gamma, 4) ||
        lc_off_element(save_mean, 4) || lc_off_element(save_rstd, 4))
        return LC_ERR_ALIGN;
    if (!workspace || (((uintptr_t)workspace) & 255) || workspace_bytes < layernorm_bwd_workspace_bytes(desc)) return LC_ERR_WORKSPACE;
    const int blocks = (int)grad_blocks(desc->dtype, desc->rows, desc->c);
    const LayerBwdArgs a{total, dy, dtotal, gamma, save_mean, save_rstd, dx, static_cast<float*>(workspace), desc->rows, h_ld ? h_ld : desc->c,
                         (dbeta ? 2ll : 1ll) * desc->c, desc->c};
    lc_begin_call();
    if (desc->dtype == LC_BF16) launch_bwd<uint16_t>(a, blocks, stream);
    else launch_bwd<float>(a, blocks, stream);
    sum_parts(a.part, dgamma, dbeta, blocks, desc->c, stream);
    return lc_end_call();
}
