// What the norms over a row (rmsnorm.hip, layernorm.hip) share: how a block's threads take rows, how wide a thread's part is, how many blocks a backward pass has, and
// the sum of those blocks' shares of the gradients of scale and shift.  Figures are the RMS norm's.
#pragma once

#include <algorithm>

#include "token_common.h"

namespace {

constexpr int kMostWaves = 16;

// A value of each wave's own making, joined over a block of `waves` waves, every thread with the result; `red` (a float a wave) must not be in use by an
// earlier call that a slower wave may still read.
template <typename W, typename F>
__device__ __forceinline__ float block_join(float x, int waves, float* red, W&& in_wave, F&& f) {
    x = in_wave(x);
    if (waves == 1) return x;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = red[0];
    for (int w = 1; w < waves; ++w) s = f(s, red[w]);
    return s;
}

// How a block's threads share rows: all of them one row (LANES 0), or LANES neighbouring lanes of a wave each a row (of a block of kNarrowThreads).
constexpr int kNarrowThreads = 256;
template <int LANES>
struct Rows {
    static constexpr int kEach = LANES ? kNarrowThreads / LANES : 1;     // rows of a block
    static __device__ __forceinline__ int tid() { return LANES ? threadIdx.x & (LANES - 1) : threadIdx.x; }
    static __device__ __forceinline__ long long first() { return LANES ? (long long)blockIdx.x * kEach + threadIdx.x / (kNarrowThreads / kEach) : blockIdx.x; }
    static __device__ __forceinline__ long long step() { return LANES ? (long long)gridDim.x * kEach : gridDim.x; }

    template <typename W, typename F>
    static __device__ __forceinline__ float join(float v, int waves, float* red, W&& wave, F&& f) {
        if constexpr (LANES == 0) return block_join(v, waves, red, wave, f);
#pragma unroll
        for (int off = 1; off < LANES; off <<= 1) v = f(v, __shfl_xor(v, off, 64));
        return v;
    }
};

constexpr int kMostColumns = 16384;          // what a block's registers hold of a row
constexpr int kMostWidth = 1 << 30;          // columns are counted in 32 bits, eight past the end among them
constexpr long long kMostBlocks = 1 << 20;   // rows, or column tiles, beyond are dealt round

// first[k], k < c, and second[k - c] = the blocks' shares, `width` (c or 2 c) a block, added in a fixed order: COLS columns a block, whose 1024 / COLS groups of threads take every so many shares, eight of them under way at a
// time.  16 columns a block where 64 would leave most of the chip without one (16384 x 256, forward and backward, 29.6 us,
// so 25.9; from 1537 columns on 64 are as fast or faster).
constexpr int kNarrow = 1024;
template <int COLS>
__global__ void __launch_bounds__(1024) norm_parts_kernel(const float* __restrict__ part, float* __restrict__ first, float* __restrict__ second, int parts, int c, long long width) {
    constexpr int U = 8, kGroups = 1024 / COLS;
    __shared__ float sum[kGroups][COLS];
    const int column = threadIdx.x & (COLS - 1), group = threadIdx.x / COLS;
    for (long long at = (long long)blockIdx.x * COLS; at < width; at += (long long)gridDim.x * COLS) {
        const long long k = at + column;
        float s[U] = {};
        if (k < width) {
            int i = group;
            for (; i + kGroups * (U - 1) < parts; i += kGroups * U) {
                float v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = part[(i + kGroups * u) * width + k];
#pragma unroll
                for (int u = 0; u < U; ++u) s[u] += v[u];
            }
#pragma unroll
            for (int u = 0; u < U - 1; ++u)
                if (i + kGroups * u < parts) s[u] += part[(i + kGroups * u) * width + k];
        }
        sum[group][column] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
        __syncthreads();
        if (group == 0 && k < width) {
            float t[4] = {};
#pragma unroll
            for (int w = 0; w < kGroups; ++w) t[w & 3] += sum[w][column];
            *(k < c ? first + k : second + (k - c)) = (t[0] + t[1]) + (t[2] + t[3]);
        }
        __syncthreads();
    }
}
inline void sum_parts(const float* part, float* first, float* second, int parts, int c, hipStream_t stream) {
    const long long width = (second ? 2ll : 1ll) * c, tiles = std::min(c <= kNarrow ? (width + 15) / 16 : (width + 63) / 64, kMostBlocks);      // (a launch holds fewer than 2^32 threads)
    if (c <= kNarrow) hipLaunchKernelGGL((norm_parts_kernel<16>), dim3((unsigned)tiles), dim3(1024), 0, stream, part, first, second, parts, c, width);
    else hipLaunchKernelGGL((norm_parts_kernel<64>), dim3((unsigned)tiles), dim3(1024), 0, stream, part, first, second, parts, c, width);
}

// Bytes that a call reads and writes from which it goes past the caches, where the row's accesses take whole lines of 128 bytes (bf16; fp32's two halves of
// eight columns do not: 8192 x 4096 94 us, past the caches 105).  Three sets in turn, us, ordinary / past, c = 4096: 2048 rows (67 MB) 11.8 / 13.7, 3000 (98 MB) 19.9 / 18.9,
// 4096 (134 MB) 26.2 / 24.2, 8192 47.8 / 45.4.
constexpr long long kStreamBytes = 96 << 20;

// Columns of a wave by what a thread has in registers: 16 for bf16 (rows under 512 columns 8: 16384 x 256 7.7 us, with 16 9.2; 4099 x 5120 to 8 bits 36.0, with 16 32.2, with 32 34.7), 8 for
// fp32 (8192 x 4096 94 us, with 16 97), 16 where 16 waves would not do.
template <typename T>
int chunks_of(int c) {
    return sizeof(T) == 2 ? (c <= 512 ? 1 : 2) : (c <= 512 * kMostWaves ? 1 : 2);
}

// Lanes of a row where a wave takes several, from what a wave of its own per row takes, us, 2^25 elements in all: bf16 forward with c = 64, 128, 256 125, 69, 39, so 26;
// to 8 bits 216, 119, 65, so 42; forward and backward 250, 140, 88, so 66; fp32 forward 143, 82, 51, so 49.
constexpr int kMostNarrow = 256;             // columns
inline bool narrow(long long rows, int c) { return c <= kMostNarrow && rows > 256; }        // (fewer have a compute unit each; the same to 4096 rows, where a launch is what they take)
inline int lanes_of(int c) { return c <= 64 ? 8 : c <= 128 ? 16 : 32; }

// Rows that go by in passes: what a block's registers do not hold (of fp32 rows that end within a thread's columns 16 a thread neither: 3000 x 9001, forward and backward, 317 us, in
// passes 275), and under eight columns.
inline bool in_passes(const lc_dtype dtype, int c) { return c < 8 || c > kMostColumns || (dtype == LC_F32 && c % 8 && c > 512 * kMostWaves); }

// Blocks of the backward pass, each with a share of dgamma: 16 waves a compute unit, with four rows a block or more as long as every unit has one.  us, 8192 x 4096 bf16 forward and
// backward with 256, 512, 1024 blocks 110, 96.6, 104; 16384 x 1024 97, 70, 58; 2048 x 16384 105, 114, 128; 512 x 4096 14.8, 16.0, 16.0.  Narrow rows: the same with a wave's several rows
// for one (2^20 rows of 32 with 512, 1024, 2048 blocks of four waves 97, 83, 88).
inline int bwd_chunks(int c) { return c <= 512 * kMostWaves ? 1 : 2; }
inline long long bwd_blocks(lc_dtype dtype, long long rows, int c) {
    if (in_passes(dtype, c)) return std::min<long long>(rows, 64);
    if (narrow(rows, c)) {
        const long long each = kNarrowThreads / lanes_of(c), all = (rows + each - 1) / each;
        return std::min(all, std::max<long long>(256, std::min<long long>(1024, all / 4)));
    }
    const int columns = 512 * bwd_chunks(c), waves = (c + columns - 1) / columns;
    return std::min<long long>(rows, std::max<long long>(256, std::min<long long>(4096 / waves, rows / 4)));
}

}  // namespace
