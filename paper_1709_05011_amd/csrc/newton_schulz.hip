// Newton-Schulz steps that orthogonalise matrices, and the optimizer's step around them (momentum, orthogonalised update, decay), for gfx950.
//
// X = u / (|u| + eps), then `iterations` times X <- a X + (b A + c A A) X with A = X X^T on the shorter side: the singular values go through a x + b x^3 + c x^5, which takes all but the
// smallest near 1.  Three products a step, A and B = a I + b A + c A A symmetric: of those only tiles on and below the diagonal are made and written twice.
//
// Values are pairs of fp16, hi = x rounded, lo = (x - hi) rounded, 22 bits, scaled by 2^12: singular values stay below 1.21, hence every value of X below 1.21, of A below 1.46 and of B below 3.45,
// and fp16's range leaves room for more than four times that; a product is three matrix instructions, lo hi + hi lo + hi hi, summed in fp32.  One fp16 (or bf16) value each, a third of the instructions, was simulated in 64 bits and
// left: small singular values grow by up to 3.4445 a step, and the first rounding with them: errors of 1.4e-3 (bf16 1.3e-2) on a random matrix and 1.4e-2 (0.11) on one of rank 8 and noise, pairs 3e-7 to 3e-6, fp32 products
// 1e-6 to 6e-5.  On the card, means of 3 to 12 matrices, pairs / fp32 products: normal 2048 x 2048 2.4e-6 / 3.6e-6, 256 x 256 1.1e-6 / 1.8e-6, 100 x 2000 1.6e-6 / 1.5e-6, 64 x 2304 2.0e-6 / 1.4e-6, 4 x 4 8.8e-7 / 5.4e-7; rank 2 and
// noise 2048 x 2048 2.7e-5 / 3.0e-5, 16 x 64 5.0e-6 / 3.5e-6; the furthest apart, 16 x 2000 with rows and columns of different sizes, 2.5e-6 / 9.7e-7: short sums in fp32 lose less than the pairs' two bits.
//
// In memory a matrix is [row][32 columns: 32 hi, 32 lo], sides filled up with zeros to multiples of 32: a k-step of 32 is 128 bytes of a row, a whole line, and LDS holds it as the bf16 products of conv_dma.h do.  A
// and B are symmetric, so that two products read rows along their sums; B X reads rows of X from LDS the other way round.  (X kept both ways round as well, ResNet-50's filters,
// 94 MB: 110 us for B X, so 84; two layers of width 2048 1094, so 1003.)
//
// Bound by the matrix pipe and the card's power where products are large (4096 x 4096: 3.25 to 3.5 ms from card to card, B X 305 to 330 us, 1.25 to 1.35 PFLOP/s of the pairs' products, as a large library product of fp16), by
// what a unit fetches from L2 in between, by launches where they are small (three of 517 x 1031: 17 launches of 6 to 13 us, 168 to 175).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>
#include <vector>

#include "dma_common.h"
#include "internal.h"
#include "token_common.h"

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScale = 4096.f, kInvScale = 1.f / 4096.f;
constexpr int kPad = 32;                           // sides in memory are multiples of it
constexpr int kMostParts = 1024;                   // sums of squares of a matrix
constexpr int kTable = 64, kSmallTable = 8;        // matrices of a launch

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct Mat {
    const void* in;          // gradient, or the matrix itself
    float* m;                // momentum; null: no optimizer's step
    float* w;
    void* out;               // bf16 copy of w or null; the result
    long long ld;            // of in
    int rows, cols;
    int M, N;                // sides in memory, M <= N
    int tall;                // rows > cols: X is the transpose
    int chunk;               // vectors of four that a block sums the squares of
    unsigned char* base;     // its part of the workspace
    float step, lr_decay;    // lr * scale, lr * decay
    __host__ __device__ long long side() const { return (long long)M * N * 4; }
    __host__ __device__ unsigned char* x(int which) const { return base + kMostParts * 8 + which * side(); }
    __host__ __device__ unsigned char* a() const { return x(2); }
    __host__ __device__ unsigned char* b() const { return a() + (long long)M * M * 4; }
};

struct Scalars {
    int count;
    const float* grad_scale;
    float momentum, eps;
    int nesterov;
    int which;               // of the two places of X, the one that is read
};

template <int TABLE>
struct Args {
    Mat t[TABLE];
    int start[(TABLE + 63) / 64 * 64];   // first block of each, past the last the largest int
    uint8_t dies[TABLE], die[TABLE];     // products: how many dies take a matrix, from which on
    int cuts;                            // or: start[] counts tiles instead, and the tile of all that a die begins with, and the one behind its last
    int cut[9];
    Scalars s;
};

// The matrix that a block belongs to (the same for the block) and the block's number within it.
template <int TABLE>
__device__ __forceinline__ int owner_of(const Args<TABLE>& args, int bid, int* local) {
    const int lane = threadIdx.x & 63;
    const int owner = __builtin_amdgcn_readfirstlane(__popcll(__ballot(args.start[lane] <= bid)) - 1);
    *local = bid - args.start[owner];
    return owner;
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
template <bool NT = false>
__device__ __forceinline__ void load4(float* to, const float* p, int n) {
    if (n >= 4) {
        const lc_u32x4 x = lc_load16<NT>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = __uint_as_float(x[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = j < n ? p[j] : 0.f;
    }
}
template <bool NT = false>
__device__ __forceinline__ void load4(float* to, const uint16_t* p, int n) {
    u32x2 x = {0u, 0u};
    if (n >= 4) {
        if constexpr (NT) x = __builtin_nontemporal_load(reinterpret_cast<const u32x2_any*>(p));
        else x = *reinterpret_cast<const u32x2_any*>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) x[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) to[j] = __uint_as_float(j & 1 ? x[j >> 1] & 0xffff0000u : x[j >> 1] << 16);
}

// The first n of four values (none for n <= 0).
__device__ __forceinline__ void put4(float* p, const float* v, int n) {
    if (n >= 4) {
        lc_store16(p, lc_u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = v[j];
    }
}
__device__ __forceinline__ void put4(uint16_t* p, const float* v, int n) {
    const u32x2 x = {lc_bf16x2_rne(v[0], v[1]), lc_bf16x2_rne(v[2], v[3])};
    if (n >= 4) {
        *reinterpret_cast<u32x2_any*>(p) = x;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = (uint16_t)(x[j >> 1] >> (16 * (j & 1)));
    }
}

// The momentum's update and the sum of squares, in double, of what is orthogonalised: one block a chunk.  ResNet-50's filters (275 MB) 53 us, 5.2 TB/s.
template <typename T, bool MUON, int TABLE>
__global__ void __launch_bounds__(256) ns_squares_kernel(const Args<TABLE> args) {
    __shared__ double red[4];
    int part;
    const Mat& t = args.t[owner_of(args, blockIdx.x, &part)];
    const unsigned per_row = MUON ? 0u : (unsigned)((t.cols + 3) / 4);
    const long long all = MUON ? ((long long)t.rows * t.cols + 3) / 4 : (long long)t.rows * per_row;
    const long long end = std::min(all, (long long)(part + 1) * t.chunk);
    const float gs = args.s.grad_scale ? *args.s.grad_scale : 1.f, mu = args.s.momentum;
    double sum = 0.0;
    for (long long v = (long long)part * t.chunk + threadIdx.x; v < end; v += 256) {
        float u[4];
        if constexpr (MUON) {
            float m[4];
            const long long at = v * 4, left = (long long)t.rows * t.cols - at;
            const int n = (int)std::min(left, 4ll);
            load4(u, static_cast<const T*>(t.in) + at, n);
            load4(m, t.m + at, n);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float g = u[j] * gs;
                m[j] = fmaf(mu, m[j], g);
                u[j] = args.s.nesterov ? fmaf(mu, m[j], g) : m[j];
            }
            put4(t.m + at, m, n);
        } else {
            const unsigned row = (unsigned)v / per_row, col = ((unsigned)v - row * per_row) * 4;
            load4(u, static_cast<const T*>(t.in) + (long long)row * t.ld + col, t.cols - (int)col);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = fma((double)u[j], (double)u[j], sum);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) reinterpret_cast<double*>(t.base)[part] = (red[0] + red[1]) + (red[2] + red[3]);
}

// Four values as pairs: two conversions at a time, and the rest by an operation that takes hi as it is.
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void split4(const float* v, f16x4* hi, f16x4* lo) {
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
        const f16x2 h = __builtin_convertvector((f32x2{v[j], v[j + 1]}), f16x2);
        const f16x2 l = __builtin_convertvector((f32x2{fmaf((float)h[0], -1.f, v[j]), fmaf((float)h[1], -1.f, v[j + 1])}), f16x2);
        (*hi)[j] = h[0];
        (*hi)[j + 1] = h[1];
        (*lo)[j] = l[0];
        (*lo)[j + 1] = l[1];
    }
}
// Eight scaled values as pairs: hi in the first 16 bytes' place, lo 64 bytes behind.
__device__ __forceinline__ void store_pairs(unsigned char* p, const float* v) {
    f16x4 hi[2], lo[2];
    split4(v, hi, lo);
    split4(v + 4, hi + 1, lo + 1);
    *reinterpret_cast<f16x8*>(p) = __builtin_shufflevector(hi[0], hi[1], 0, 1, 2, 3, 4, 5, 6, 7);
    *reinterpret_cast<f16x8*>(p + 64) = __builtin_shufflevector(lo[0], lo[1], 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ void load_pairs(float* v, const unsigned char* p) {
    const f16x8 hi = *reinterpret_cast<const f16x8*>(p), lo = *reinterpret_cast<const f16x8*>(p + 64);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)hi[j] + (float)lo[j];
}
// Byte of element (row, col) of a matrix with `k` columns in memory, col a multiple of 8.
__device__ __forceinline__ long long pair_at(long long row, int col, int k) { return row * k * 4 + (col >> 5) * 128 + (col & 31) * 2; }

// u / (|u| + eps) as pairs: a block 64 x 64 values.  A step reads its gradient and momentum for the last time here, past the caches, which X then finds emptier (ResNet-50's filters 907 us, so 880; twelve layers of width 256
// 520 / 512).
template <typename T, bool MUON, int TABLE>
__global__ void __launch_bounds__(256) ns_split_kernel(const Args<TABLE> args) {
    __shared__ double red[4];
    __shared__ float tile[64][65];
    int local;
    const Mat& t = args.t[owner_of(args, blockIdx.x, &local)];
    const int tid = threadIdx.x;
    const int pcols = t.tall ? t.M : t.N;          // of the sides in memory, along the matrix's rows
    const int across = (pcols + 63) / 64, r0 = local / across * 64, c0 = local % across * 64;
    const float gs = args.s.grad_scale ? *args.s.grad_scale : 1.f, mu = args.s.momentum;
    float u[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int row = r0 + (tid >> 4) + 16 * k, col = c0 + 4 * (tid & 15);
        const int n = row < t.rows ? t.cols - col : 0;
        load4<MUON>(u[k], static_cast<const T*>(t.in) + (n > 0 ? (long long)row * t.ld + col : 0), n);
        if constexpr (MUON) {
            float m[4];
            load4<true>(m, t.m + (n > 0 ? (long long)row * t.cols + col : 0), n);
#pragma unroll
            for (int j = 0; j < 4; ++j) u[k][j] = args.s.nesterov ? fmaf(mu, m[j], u[k][j] * gs) : m[j];
        }
    }
    const long long vectors = MUON ? ((long long)t.rows * t.cols + 3) / 4 : (long long)t.rows * ((t.cols + 3) / 4);
    const int parts = (int)((vectors + t.chunk - 1) / t.chunk);
    double sum = 0.0;
    for (int i = tid; i < parts; i += 256) sum += reinterpret_cast<const double*>(t.base)[i];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if ((tid & 63) == 0) red[tid >> 6] = sum;
    __syncthreads();
    sum = (red[0] + red[1]) + (red[2] + red[3]);
    const double norm = sqrt(sum) + (double)args.s.eps, inv = sum == 0.0 ? 0.0 : (double)kScale / norm;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) tile[(tid >> 4) + 16 * k][4 * (tid & 15) + j] = (float)((double)u[k][j] * inv);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int line = (tid >> 3) + 32 * k, run = (tid & 7) * 8;
        const int row = (t.tall ? c0 : r0) + line, col = (t.tall ? r0 : c0) + run;
        if (row >= t.M || col >= t.N) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = t.tall ? tile[run + j][line] : tile[line][run + j];
        store_pairs(t.x(0) + pair_at(row, col, t.N), v);
    }
}

// What a product makes: A = X X^T; B = a I + b A + c A A; X <- B X, to the other place; the same as the result.  (a on B's diagonal costs X a rounding of 2^-22, as its own is, and saves reading X once more:
// ResNet-50's filters 124 us for X with it added at the end, so 110.)
enum Product { kGram, kSquare, kNext, kLast };

template <Product KIND>
__host__ __device__ inline int tiles_of(const Mat& t, int BM, int BN) {
    const int nm = (t.M + BM - 1) / BM, nn = (t.N + BN - 1) / BN;
    return KIND <= kSquare ? nm * (nm + 1) / 2 : nm * nn;
}

// Row and column of a tile: down the columns of groups of four rows of tiles (by 256 rows), so that the tiles that a die works on at a time are about as high as wide and share what they read.
template <Product KIND>
__device__ __forceinline__ void place_of(const Mat& t, int tile, int BM, int BN, int* ti, int* tj) {
    const int nm = (t.M + BM - 1) / BM, nn = (t.N + BN - 1) / BN;
    if constexpr (KIND <= kSquare) {
        constexpr int G = 4;
        int row = (int)((sqrtf(8.f * (float)tile + 1.f) - 1.f) * 0.5f);
        while ((row + 1) * (row + 2) / 2 <= tile) ++row;
        while (row * (row + 1) / 2 > tile) --row;
        const int first = row / G * G, high = std::min(G, nm - first);
        int at = tile - first * (first + 1) / 2;
        if (at < (first + 1) * high) {
            *tj = at / high;
            *ti = first + at % high;
        } else {                                   // the corner on the diagonal
            at -= (first + 1) * high;
            int d = 1;
            for (; at >= high - d; ++d) at -= high - d;
            *tj = first + d;
            *ti = *tj + at;
        }
    } else {
        const int G = std::max(1, 1024 / BM), first = tile / (G * nn) * G, high = std::min(G, nm - first), at = tile - first * nn;
        *tj = at / high;
        *ti = first + at % high;
    }
}

__device__ __forceinline__ f32x4 multiply(const f16x8& a, const f16x8& b, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

constexpr int leaving_columns(int TN) { return TN > 4 ? TN / 2 : TN; }

// Rows P[i] times rows Q[j] along their sum.  A block has WM x WN waves of 16 TM x 16 TN values each; NS stages of LDS, the next ones arriving while one is multiplied.
template <Product KIND, bool MUON, typename T, int TM, int TN, int WM, int WN, int NS, int TABLE>
__global__ void __launch_bounds__(WM * WN * 64, 2) ns_product_kernel(const Args<TABLE> args) {
    constexpr int BM = 16 * TM * WM, BN = 16 * TN * WN, NW = WM * WN;
    constexpr int LP = BM / 8 / NW, LQ = BN / 8 / NW;              // loads of a wave a stage
    constexpr int STAGE = (BM + BN) * 128;
    constexpr int TC = leaving_columns(TN), kPitch = TC * 16 + 4;   // floats
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && NW % 2 == 0, "tile shape");
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    // blocks are dealt round the dies
    int tile, owner;
    if (args.cuts) {
        const int die = blockIdx.x & 7, at = args.cut[die] + (int)(blockIdx.x >> 3);
        if (at >= args.cut[die + 1]) return;
        owner = owner_of(args, at, &tile);
    } else {                                       // a matrix's begin at a multiple of 8: its dies take neighbouring tiles each, the others' blocks have nothing to do
        int local;
        owner = owner_of(args, blockIdx.x, &local);
        const int dies = args.dies[owner], part = (local - args.die[owner]) & 7;
        const int tiles = tiles_of<KIND>(args.t[owner], BM, BN), per = (tiles + dies - 1) / dies;
        tile = part * per + (local >> 3);
        if (part >= dies || tile >= std::min(tiles, (part + 1) * per)) return;
    }
    const Mat& t = args.t[owner];
    const int M = t.M, N = t.N;
    int ti, tj;
    place_of<KIND>(t, tile, BM, BN, &ti, &tj);
    ti = __builtin_amdgcn_readfirstlane(ti);
    tj = __builtin_amdgcn_readfirstlane(tj);
    const int i0 = ti * BM, j0 = tj * BN;
    constexpr bool TURN = KIND >= kNext;           // Q[j] is column j of X: rows of X are loaded, and read from LDS the other way round
    const int K = KIND == kGram ? N : M;
    const unsigned pitch = (unsigned)K * 4u, x_pitch = (unsigned)N * 4u;
    const unsigned char* const P = KIND == kGram ? t.x(args.s.which) : KIND == kSquare ? t.a() : t.b();
    const unsigned char* const Q = KIND == kGram ? P : KIND == kSquare ? P : t.x(args.s.which) + (long long)j0 * 4;
    // rows past the matrix lie past the end of the buffer: zeros.  (Of TURN, columns past it are the next row's, or past the end; what they make is not stored.)
    const u32x4 p_rsrc = buffer_words(P + (long long)i0 * pitch, (unsigned)std::min(BM, M - i0) * pitch);
    u32x4 q_rsrc = TURN ? buffer_words(Q, 32u * x_pitch - (unsigned)j0 * 4u) : buffer_words(Q + (long long)j0 * pitch, (unsigned)std::min(BN, M - j0) * pitch);
    const int lrow = lane >> 3, piece = (lane & 7) ^ (((wave & 1) * 4 + (lrow >> 1)) & 7);
    const unsigned voff = (unsigned)(wave * 8 + lrow) * pitch + piece * 16;
    // TURN: LDS holds 32 rows of BN columns; pieces of 16 bytes at piece ^ 2 (row % 4 + row / 8 % 2 * 4), so that the 16 rows of a turning read lie on all banks
    unsigned q_voff[LQ];
#pragma unroll
    for (int l = 0; l < LQ; ++l) {
        const int at = (l * NW + wave) * 64 + lane, row = at / (BN / 4), slot = at - row * (BN / 4);
        q_voff[l] = TURN ? (unsigned)row * x_pitch + (slot ^ ((row & 3) | (row >> 1 & 4)) << 1) * 16 : voff + (unsigned)(l * NW * 8) * pitch;
    }
    const unsigned lds0 = lds_address(smem);
    const int steps = K / 32;
    unsigned long long q_base = (unsigned long long)q_rsrc[1] << 32 | q_rsrc[0];
    const auto load = [&](int k, int stage) __attribute__((always_inline)) {       // (called for k = 0, 1, 2, ...)
        const unsigned past = k < steps ? 0u : kBufferBytes;       // (behind the last step the loads fetch nothing, and their number stays the same)
#pragma unroll
        for (int l = 0; l < LP; ++l) load_to_lds(p_rsrc, (voff + (unsigned)(l * NW * 8) * pitch) | past, k * 128, lds0 + stage * STAGE + (l * NW + wave) * 1024);
#pragma unroll
        for (int l = 0; l < LQ; ++l) load_to_lds(q_rsrc, q_voff[l] | past, TURN ? 0 : k * 128, lds0 + stage * STAGE + BM * 128 + (l * NW + wave) * 1024);
        if constexpr (TURN) {
            q_base += 32ull * x_pitch;
            q_rsrc[0] = (unsigned)q_base;
            q_rsrc[1] = (unsigned)(q_base >> 32);
        }
    };
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int sw = (lane & 15) >> 1, fp = lane >> 4;
    const int hi = ((fp ^ sw) & 7) * 16, lo = (((4 + fp) ^ sw) & 7) * 16;
    const unsigned char* const p_lane = smem + (wm * TM * 16 + (lane & 15)) * 128;
    const unsigned char* const q_lane = smem + BM * 128 + (wn * TN * 16 + (lane & 15)) * 128;
    // TURN: a lane's four columns of a row, whose columns it then holds as 16 lanes' four rows: rows 8 (lane / 16) + 0 .. 3, and four further for the other half of its eight
    const unsigned char* turn_lane[TN][2];
    if constexpr (TURN) {
        const int row = (lane >> 4) * 8 + ((lane >> 2) & 3), turn = (((lane >> 2) & 3) | (lane >> 2 & 4)) << 1;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int col = (wn * TN + j) * 16, first = col / 32 * 8 + (col & 16) / 8;
#pragma unroll
            for (int h = 0; h < 2; ++h) turn_lane[j][h] = smem + BM * 128 + row * (BN * 4) + (((first + 4 * h) ^ turn) + ((lane >> 1) & 1)) * 16 + (lane & 1) * 8;
        }
    }
    f16x8 ph[2][TM], pl[2][TM], qh[2][TN], ql[2][TN];
    const auto read_q = [&](int j, int h, int at) __attribute__((always_inline)) {
        if constexpr (TURN) {
            const auto four = [&](int rows) __attribute__((always_inline)) {
                const unsigned char* const from = turn_lane[j][h] + at + rows * (BN * 4);
                return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)from);
            };
            const s16x4 a = four(0), b = four(4);
            return __builtin_bit_cast(f16x8, s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
        } else {
            return *reinterpret_cast<const f16x8*>(q_lane + at + (h ? lo : hi) + j * 2048);
        }
    };
    const auto read = [&](int to, int stage) __attribute__((always_inline)) {
        const int at = stage * STAGE;
#pragma unroll
        for (int i = 0; i < TM; ++i) pl[to][i] = *reinterpret_cast<const f16x8*>(p_lane + at + lo + i * 2048);
#pragma unroll
        for (int j = 0; j < TN; ++j) qh[to][j] = read_q(j, 0, at);
#pragma unroll
        for (int i = 0; i < TM; ++i) ph[to][i] = *reinterpret_cast<const f16x8*>(p_lane + at + hi + i * 2048);
#pragma unroll
        for (int j = 0; j < TN; ++j) ql[to][j] = read_q(j, 1, at);
    };
    // fragments of the next step are read while this one's are multiplied: with them read first a step took two and a half times its matrix instructions where a SIMD has one wave
    int stage = 0;
    const auto step = [&]<int BUF>(std::integral_constant<int, BUF>, int k) __attribute__((always_inline)) {
        wait_loads_and_barrier<(NS - 2) * (LP + LQ)>();             // the next stage has arrived, and all waves have read this one
        load(k + NS, stage);
        stage = stage == NS - 1 ? 0 : stage + 1;
        read(BUF ^ 1, stage);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = multiply(pl[BUF][i], qh[BUF][j], acc[i][j]);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = multiply(ph[BUF][i], ql[BUF][j], acc[i][j]);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = multiply(ph[BUF][i], qh[BUF][j], acc[i][j]);
#pragma unroll
        for (int i = 0; i < 2 * TM + (TURN ? 4 : 2) * TN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, std::max(1, 3 * TM * TN / (2 * TM + (TURN ? 4 : 2) * TN)), 0);
        }
    };
#pragma unroll
    for (int s = 0; s < NS; ++s) load(s, s);
    wait_loads_and_barrier<(NS - 1) * (LP + LQ)>();
    read(0, 0);
    for (int k = 0; k < steps; k += 2) {
        step(std::integral_constant<int, 0>{}, k);
        if (k + 1 < steps) step(std::integral_constant<int, 1>{}, k + 1);
    }
    wait_loads_and_barrier<0>();

    // the tile leaves through the wave's own LDS, some columns of pieces at a time, in runs of eight values along either side
    float* const mine = reinterpret_cast<float*>(smem) + wave * (TM * 16 * kPitch);
    const int iw = i0 + wm * TM * 16;
    constexpr int RA = TC * 2, RB = TM * 2;                        // runs of a row, of a column
    const bool along = KIND != kLast || !t.tall, turned = (KIND <= kSquare && ti != tj) || (KIND == kLast && t.tall);
    const int columns = KIND <= kSquare ? M : N;
    const auto leave = [&](int row, int col, const float* v) __attribute__((always_inline)) {        // eight results from (row, col) of the matrix as it lies
        if (row >= t.rows || col >= t.cols) return;
        const long long at = (long long)row * t.cols + col;
        const int n = t.cols - col;
        float o[8];
        if constexpr (MUON) {
            Packed<float> w;
            if (n >= 8) w.load(t.w + at);
            else w.load_some(t.w + at, n, 0u);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(-t.step, v[e], fmaf(-t.lr_decay, w.get(e), w.get(e)));
            lc_store8(t.w + at, o, n);
            if (t.out) lc_store8(static_cast<uint16_t*>(t.out) + at, o, n);
        } else {
            lc_store8(static_cast<T*>(t.out) + at, v, n);
        }
    };
#pragma unroll
    for (int part = 0; part < TN / TC; ++part) {
        const int jw = j0 + (wn * TN + part * TC) * 16;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TC; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) mine[(i * 16 + (lane >> 4) * 4 + r) * kPitch + j * 16 + (lane & 15)] = acc[i][part * TC + j][r];
        __syncthreads();
#pragma unroll 2
        for (int at = lane; at < TM * 16 * RA; at += 64) {
            const int row = at / RA, run = at % RA * 8, gi = iw + row, gj = jw + run;
            float* const p = mine + row * kPitch + run;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = p[e];
            if (gi < M && gj < columns) {
                if constexpr (KIND == kSquare) {
                    float o[8];
                    load_pairs(o, t.a() + pair_at(gi, gj, M));
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = fmaf(kC * kInvScale, v[e], kB * o[e]) + (gi == gj + e ? kA * kScale : 0.f);
                    store_pairs(t.b() + pair_at(gi, gj, M), v);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= KIND == kLast ? kInvScale * kInvScale : kInvScale;
                    if constexpr (KIND == kGram) store_pairs(t.a() + pair_at(gi, gj, M), v);
                    else if constexpr (KIND == kNext) store_pairs(t.x(args.s.which ^ 1) + pair_at(gi, gj, N), v);
                    else if (along) leave(gi, gj, v);
                }
            }
            if (turned) {
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = v[e];
            }
        }
        __syncthreads();
        if (turned) {
#pragma unroll 2
            for (int at = lane; at < TC * 16 * RB; at += 64) {
                const int col = at / RB, run = at % RB * 8, gj = jw + col, gi = iw + run;
                if (gj >= columns || gi >= M) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = mine[(run + e) * kPitch + col];
                if constexpr (KIND == kGram) store_pairs(t.a() + pair_at(gj, gi, M), v);
                else if constexpr (KIND == kSquare) store_pairs(t.b() + pair_at(gj, gi, M), v);
                else if constexpr (KIND == kLast) leave(gj, gi, v);
            }
        }
        if (part + 1 < TN / TC) __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------- small matrices

// Sides up to 64 and 256: a block takes a matrix through all steps in LDS (X both ways round and A, 144 KB), where launches for each product would be nearly all of the time (twelve matrices of 64 x 64 and 64 x 256 80 us, so 42).
constexpr int kSmallM = 64, kSmallN = 256, kSmallThreads = 512;
bool small(int M, int N) { return M <= kSmallM && N <= kSmallN; }

// A row in LDS: blocks of 32 columns of 128 bytes (16-byte pieces: 0 to 3 hi, 4 to 7 lo).  Sixteen rows' pieces lie on all banks: rows of an odd number of blocks begin on either half of them by themselves, others have
// their blocks swapped in pairs from eight rows to the next; pieces are turned by the row.  Rows 16 apart differ by the rows' bytes alone.
struct LdsRow {
    int base, turn, flip;
    __device__ __forceinline__ LdsRow(int row, int blocks) : base(row * blocks * 128), turn(((blocks & 1 ? row >> 1 : row) & 7) * 16), flip(blocks & 1 ? 0 : row * 16 & 128) {}
    __device__ __forceinline__ int block(int kb) const { return base + (kb * 128 ^ flip); }
    __device__ __forceinline__ int piece(int n) const { return n * 16 ^ turn; }                                       // within a block
    __device__ __forceinline__ int hi(int col) const { return block(col >> 5) + piece((col & 31) >> 3) + (col & 7) * 2; }
    __device__ __forceinline__ int lo(int col) const { return block(col >> 5) + piece(4 + ((col & 31) >> 3)) + (col & 7) * 2; }
};

template <typename T, bool MUON, int TABLE>
__global__ void __launch_bounds__(kSmallThreads) ns_small_kernel(const Args<TABLE> args, int iterations) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ double red[8];
    const Mat& t = args.t[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int M = t.M, N = t.N, mb = M / 32, nb = N / 32;          // blocks of 32 columns of a row of A and of the transpose, of X
    unsigned char* const X = smem;
    unsigned char* const XT = smem + kSmallM * kSmallN * 4;
    unsigned char* const A = XT + kSmallM * kSmallN * 4;
    for (int i = tid; i < 2 * kSmallM * kSmallN * 4 / 16; i += kSmallThreads) *reinterpret_cast<lc_u32x4*>(smem + i * 16) = lc_u32x4{0u, 0u, 0u, 0u};
    // the matrix, its momentum's update and its norm
    // (a wave takes 16 rows of 16 columns a time: their values the other way round lie on neighbouring banks)
    constexpr int kVectors = kSmallM * kSmallN / 4 / kSmallThreads;
    const int wide = (t.cols + 15) / 16;
    const float gs = args.s.grad_scale ? *args.s.grad_scale : 1.f, mu = args.s.momentum;
    float u[kVectors][4], m[kVectors][4];
    int row_of[kVectors], col_of[kVectors], count_of[kVectors];
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        const int part = wave + 8 * k, down = part / wide;
        row_of[k] = down * 16 + (lane & 15);
        col_of[k] = (part - down * wide) * 16 + (lane >> 4) * 4;
        count_of[k] = row_of[k] < t.rows ? std::min(4, t.cols - col_of[k]) : 0;
        const int n = count_of[k];
        load4(u[k], static_cast<const T*>(t.in) + (n > 0 ? row_of[k] * t.ld + col_of[k] : 0), n);
        if constexpr (MUON) load4(m[k], t.m + (n > 0 ? row_of[k] * t.cols + col_of[k] : 0), n);
    }
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        if constexpr (MUON) {
            const int row = row_of[k], col = col_of[k], n = count_of[k];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float g = u[k][j] * gs;
                m[k][j] = fmaf(mu, m[k][j], g);
                u[k][j] = args.s.nesterov ? fmaf(mu, m[k][j], g) : m[k][j];
            }
            put4(t.m + row * t.cols + col, m[k], n);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = fma((double)u[k][j], (double)u[k][j], sum);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane == 0) red[wave] = sum;
    __syncthreads();
    sum = ((red[0] + red[1]) + (red[2] + red[3])) + ((red[4] + red[5]) + (red[6] + red[7]));
    const double inv = sum == 0.0 ? 0.0 : (double)kScale / (sqrt(sum) + (double)args.s.eps);
    unsigned char* const along = t.tall ? XT : X;
    unsigned char* const turned = t.tall ? X : XT;
    const int ab = t.tall ? mb : nb, tb = t.tall ? nb : mb;
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        const int row = row_of[k], col = col_of[k];
        f16x4 hi, lo;                                             // (columns past the matrix are zeros)
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = (float)((double)u[k][j] * inv);
        split4(x, &hi, &lo);
        if (count_of[k] > 0) {
            const LdsRow to(row, ab);
            *reinterpret_cast<f16x4*>(along + to.hi(col)) = hi;
            *reinterpret_cast<f16x4*>(along + to.lo(col)) = lo;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const LdsRow turn(col + j, tb);
                *reinterpret_cast<_Float16*>(turned + turn.hi(row)) = hi[j];
                *reinterpret_cast<_Float16*>(turned + turn.lo(row)) = lo[j];
            }
        }
    }
    __syncthreads();

    // rows P[i] times rows Q[j] of pieces of 16 x 16, COUNT of them a time: the rows of one operand are the same, of the other `far` rows further for each; a lane then holds four neighbouring i of one j
    int lr = lane & 15, fp = lane >> 4;
    // (with `other` the same the other way round as well, a lane holding four neighbouring j of one i)
    const auto products = [&]<int COUNT, bool SAME_P>(std::integral_constant<int, COUNT>, std::integral_constant<bool, SAME_P>, f32x4 (&acc)[COUNT], f32x4* other,
                                                     const unsigned char* P, int i0, const unsigned char* Q, int j0, int far, int count, int blocks) __attribute__((always_inline)) {
        const LdsRow row((SAME_P ? i0 : j0) + lr, blocks), first((SAME_P ? j0 : i0) + lr, blocks);
        const unsigned char* const one = (SAME_P ? P : Q) + row.base;
        const unsigned char* const more = (SAME_P ? Q : P) + first.base;
        const int hi = row.piece(fp), lo = row.piece(4 + fp), his = first.piece(fp), los = first.piece(4 + fp), apart = far * blocks * 128;
#pragma unroll
        for (int q = 0; q < COUNT; ++q) {
            acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (SAME_P) other[q] = acc[q];
        }
        const auto block = [&]<int BLOCKS>(std::integral_constant<int, BLOCKS>, int kb) __attribute__((always_inline)) {       // that many blocks' pieces read before the first product
            f16x8 h[BLOCKS], l[BLOCKS], hs[BLOCKS][COUNT], ls[BLOCKS][COUNT];
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const unsigned char *at = one + ((kb + b) * 128 ^ row.flip), *ats = more + ((kb + b) * 128 ^ first.flip);
                h[b] = *reinterpret_cast<const f16x8*>(at + hi);
                l[b] = *reinterpret_cast<const f16x8*>(at + lo);
#pragma unroll
                for (int q = 0; q < COUNT; ++q) {
                    const unsigned char* const from = ats + std::min(q, count - 1) * apart;
                    hs[b][q] = *reinterpret_cast<const f16x8*>(from + his);
                    ls[b][q] = *reinterpret_cast<const f16x8*>(from + los);
                }
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
#pragma unroll
                for (int q = 0; q < COUNT; ++q) acc[q] = SAME_P ? multiply(l[b], hs[b][q], acc[q]) : multiply(ls[b][q], h[b], acc[q]);
#pragma unroll
                for (int q = 0; q < COUNT; ++q) acc[q] = SAME_P ? multiply(h[b], ls[b][q], acc[q]) : multiply(hs[b][q], l[b], acc[q]);
#pragma unroll
                for (int q = 0; q < COUNT; ++q) acc[q] = SAME_P ? multiply(h[b], hs[b][q], acc[q]) : multiply(hs[b][q], h[b], acc[q]);
                if constexpr (SAME_P) {                           // (the same products in the same order: the same bits)
#pragma unroll
                    for (int q = 0; q < COUNT; ++q) other[q] = multiply(hs[b][q], l[b], other[q]);
#pragma unroll
                    for (int q = 0; q < COUNT; ++q) other[q] = multiply(ls[b][q], h[b], other[q]);
#pragma unroll
                    for (int q = 0; q < COUNT; ++q) other[q] = multiply(hs[b][q], h[b], other[q]);
                }
            }
        };
        int kb = 0;
        if constexpr (COUNT <= 2) {
            for (; kb + 4 <= blocks; kb += 4) block(std::integral_constant<int, 4>{}, kb);
        }
        for (; kb < blocks; ++kb) block(std::integral_constant<int, 1>{}, kb);
    };
    const auto store4 = [&](unsigned char* hi_to, unsigned char* lo_to, const f32x4& v) __attribute__((always_inline)) {
        const float f[4] = {v[0], v[1], v[2], v[3]};
        f16x4 hi, lo;
        split4(f, &hi, &lo);
        *reinterpret_cast<f16x4*>(hi_to) = hi;
        *reinterpret_cast<f16x4*>(lo_to) = lo;
    };
    // pieces of a wave: of A column wave % across, rows from wave / across on; of X row wave % across, columns likewise
    constexpr int kSquares = kSmallM / 16 * (kSmallM / 16) / 8, kPieces = kSmallM / 16 * (kSmallN / 16) / 8;
    const int across = M / 16, step = 8 / across, own = wave & (across - 1), from = wave / across;
    const int squares = std::max(0, (across - from + step - 1) / step), pieces = std::max(0, (N / 16 - from + step - 1) / step);
    const std::integral_constant<int, kSquares> few;
    const std::integral_constant<int, kPieces> many;
    for (int it = 0; it < iterations; ++it) {
        asm volatile("" : "+v"(lr), "+v"(fp));                  // (addresses are made anew: kept over the steps they are more than the registers hold)
        f32x4 s[kSquares], x[kPieces], y[kPieces];
        const LdsRow col_a(own * 16 + lr, mb), row_x(own * 16 + lr, nb), row_t(from * 16 + lr, mb);
        if (squares) {
            products(few, std::false_type{}, s, nullptr, X, from * 16, X, own * 16, step * 16, squares, nb);
#pragma unroll
            for (int q = 0; q < kSquares; ++q)
                if (q < squares) store4(A + col_a.hi((from + q * step) * 16 + fp * 4), A + col_a.lo((from + q * step) * 16 + fp * 4), s[q] * kInvScale);      // (symmetric: the column's place)
        }
        __syncthreads();
        if (squares) {
            products(few, std::false_type{}, s, nullptr, A, from * 16, A, own * 16, step * 16, squares, mb);
#pragma unroll
            for (int q = 0; q < kSquares; ++q) {
                const int row = own * 16 + lr, col = (from + std::min(q, squares - 1) * step) * 16 + fp * 4;
                const f16x4 hi = *reinterpret_cast<const f16x4*>(A + col_a.hi(col)), lo = *reinterpret_cast<const f16x4*>(A + col_a.lo(col));
#pragma unroll
                for (int r = 0; r < 4; ++r) s[q][r] = fmaf(kC * kInvScale, s[q][r], kB * ((float)hi[r] + (float)lo[r])) + (row == col + r ? kA * kScale : 0.f);
            }
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kSquares; ++q)
            if (q < squares) store4(A + col_a.hi((from + q * step) * 16 + fp * 4), A + col_a.lo((from + q * step) * 16 + fp * 4), s[q]);
        __syncthreads();
        if (pieces) products(many, std::true_type{}, x, y, A, own * 16, XT, from * 16, step * 16, pieces, mb);
        __syncthreads();
        const bool last = it + 1 == iterations;
        const int i0 = own * 16 + fp * 4;
        if (!last) {
#pragma unroll
            for (int q = 0; q < kPieces; ++q) {
                if (q < pieces) {
                    store4(XT + row_t.hi(i0) + q * step * 16 * mb * 128, XT + row_t.lo(i0) + q * step * 16 * mb * 128, x[q] * kInvScale);
                    store4(X + row_x.hi((from + q * step) * 16 + fp * 4), X + row_x.lo((from + q * step) * 16 + fp * 4), y[q] * kInvScale);
                }
            }
        } else {
            // four neighbouring values of a row of the matrix as it lies
            const auto row_of_piece = [&](int q) __attribute__((always_inline)) { return t.tall ? (from + q * step) * 16 + lr : own * 16 + lr; };
            const auto col_of_piece = [&](int q) __attribute__((always_inline)) { return t.tall ? i0 : (from + q * step) * 16 + fp * 4; };
            const auto count = [&](int q) __attribute__((always_inline)) { return q < pieces && row_of_piece(q) < t.rows ? t.cols - col_of_piece(q) : 0; };
            float w[kPieces][4];
            if constexpr (MUON) {
#pragma unroll
                for (int q = 0; q < kPieces; ++q) load4(w[q], t.w + (count(q) > 0 ? row_of_piece(q) * t.cols + col_of_piece(q) : 0), count(q));
            }
#pragma unroll
            for (int q = 0; q < kPieces; ++q) {
                const int n = count(q), at = row_of_piece(q) * t.cols + col_of_piece(q);
                float o[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    o[r] = (t.tall ? x[q][r] : y[q][r]) * (kInvScale * kInvScale);
                    if constexpr (MUON) o[r] = fmaf(-t.step, o[r], fmaf(-t.lr_decay, w[q][r], w[q][r]));
                }
                if constexpr (MUON) {
                    put4(t.w + at, o, n);
                    if (t.out) put4(static_cast<uint16_t*>(t.out) + at, o, n);
                } else {
                    put4(static_cast<T*>(t.out) + at, o, n);
                }
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------- host

constexpr int kMostSide = 1 << 16;
constexpr int kMostIterations = 64;
constexpr long long kGroupBytes = 2ll << 30;       // of workspace that matrices go through the steps in together

long long padded(long long side) { return (side + kPad - 1) / kPad * kPad; }
long long bytes_of(long long rows, long long cols) {
    const long long M = padded(std::min(rows, cols)), N = padded(std::max(rows, cols));
    return kMostParts * 8 + 8 * M * N + 8 * M * M;
}

struct Matrix {                                    // of a call, before it has a place
    const void* in;
    float *m, *w;
    void* out;
    long long ld;
    int rows, cols;
    float step, lr_decay;
};

// Matrices by the length of their products, the longest first, so that a launch ends with short ones; in groups that share the workspace one after another.
template <typename F>
void for_groups(std::vector<int>& order, const int* rows, const int* cols, F&& f) {
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return std::max(rows[a], cols[a]) > std::max(rows[b], cols[b]); });
    for (size_t first = 0; first < order.size();) {
        long long bytes = 0;
        size_t n = 0;
        while (first + n < order.size() && n < kTable) {
            const long long more = bytes_of(rows[order[first + n]], cols[order[first + n]]);
            if (n > 0 && bytes + more > kGroupBytes) break;
            bytes += more;
            ++n;
        }
        f(first, n, bytes);
        first += n;
    }
}

size_t workspace_of(std::vector<int>& order, const int* rows, const int* cols) {
    long long most = 0;
    for_groups(order, rows, cols, [&](size_t, size_t, long long bytes) { most = std::max(most, bytes); });
    return (size_t)(most + 255) & ~(size_t)255;
}

template <int TABLE, typename F>
int set_starts(Args<TABLE>& args, F&& blocks) {
    long long at = 0;
    for (int i = 0; i < args.s.count; ++i) {
        args.start[i] = (int)at;
        at += blocks(args.t[i]);
    }
    std::fill(args.start + args.s.count, args.start + (TABLE + 63) / 64 * 64, 0x7fffffff);
    return (int)at;
}

// The tile of a launch's products, by what a launch is estimated to take, us: rounds of blocks (tiles of sums shorter than the longest count as parts of one), each the k-steps of the longest sum and what begins and ends a
// tile.  A k-step takes `alone` where a unit has one block (it fetches some 55 GB/s from beyond its die's L2 then, whatever the stages and waves), `step` with all slots at work; the matrix pipe's time at 128 x 128 is 0.32
// at full clock.  us of five iterations by the rule, with A and B in tiles of 64 / 128 with eight waves and four stages / 128 with two blocks a unit / 192, and with X in 64 / 128 and one / 128 and two / 256 x 128:
//   1024 x 1024     191    191   304   353   523    192   236   256   297      2048 x 2048     631    680   632   716   988    687   633   649   713
//   1024 x 4096     362    362   587   686  1015    385   364   369   408      two of them    1147   1119  1237  1147  1171   1301  1196  1163  1150
//   1536 x 1536     392    392   470   563   762    413   393   419   481      4096 x 4096    3338   3853  3855  3727  3342   4564  3545  3372  3346
//   ResNet-50's     891    885  1022  1143  1446   1060   942   874   899      twelve layers of width 256 496  498 555 638 732  563 537 513 557
enum Tile { kTile64, kTile128One, kTile128, kTile192, kTile256 };
struct TileCost {
    int rows, cols, slots;
    double alone, step, ends;
};
constexpr TileCost kTiles[] = {{64, 64, 512, 0.27, 0.64, 3.0}, {128, 128, 256, 0.6, 0.72, 4.0}, {128, 128, 512, 0.8, 1.42, 4.0}, {192, 192, 256, 1.5, 1.5, 8.0}, {256, 128, 256, 1.2, 1.27, 7.0}};
template <Product KIND, int TABLE>
Tile tile_of(const Args<TABLE>& args) {
    double least = 1e30, longest = 0.0;
    Tile best = kTile128;
    for (int i = 0; i < args.s.count; ++i) longest = std::max<double>(longest, KIND == kGram ? args.t[i].N : args.t[i].M);
    for (Tile tile : {kTile64, kTile128One, kTile128, kTile192, kTile256}) {
        if (tile == kTile256 && KIND <= kSquare) continue;
        const TileCost& k = kTiles[tile];
        double all = 0.0;
        for (int i = 0; i < args.s.count; ++i) all += (KIND == kGram ? args.t[i].N : args.t[i].M) * (double)tiles_of<KIND>(args.t[i], k.rows, k.cols);
        const double rounds = all / longest / k.slots, full = std::floor(rounds), rest = rounds - full;
        const double last = rest == 0.0 ? 0.0 : k.slots > 256 ? std::max(k.alone, k.step * rest) : rounds < 1.0 ? k.alone : k.step;
        const double cost = longest / 32 * (k.step * full + last) + k.ends * std::ceil(rounds);
        if (cost < least) {
            least = cost;
            best = tile;
        }
    }
    return best;
}

// How a launch's products are made: its tile, and the dies of each matrix.  A die has an L2 of its own, and what several dies work on each of them fetches: a matrix is shared by as few dies as leave their loads even, a
// part being half of a die's load at most.  Steps over a list, us, all dies a part of each / so: ResNet-50's filters 965 / 895 (A: 418 MB fetched for 94), twelve layers of width 256 530 / 484, four of 512 670 / 632, two of
// 2048 9810 / 9780, three of 333 285 / 294.
template <int TABLE>
struct LaunchPlan {
    Tile tile;
    uint8_t dies[TABLE], die[TABLE];
    bool cuts;
    int cut[9];
};
// Where all tiles of a launch have a place at once, or nearly, loads need not be even to the tile, and the list's tiles, matrix after matrix, are cut into eight parts of the same cost: a die then meets one or two matrices.  us, dies by
// matrices / so: three of 517 x 1031 177 / 170, four 231 / 205, ten 412 / 304, four of 700 x 700 221 / 197, two of 1024 x 1024 286 / 267, twenty of 256 x 512 185 / 146, four layers of width 512 640 / 590, two of 700 755 / 700; with twice as many tiles
// as places ResNet-50's filters 880 / 895, three layers of width 1298 4800 / 5115 (1.4 times: twelve layers of width 256 460 / 432, those two as before).
constexpr double kCutRounds = 1.4;
template <Product KIND, int TABLE>
LaunchPlan<TABLE> plan_of(const Args<TABLE>& args) {
    LaunchPlan<TABLE> plan{tile_of<KIND>(args), {}, {}, false, {}};
    const TileCost& k = kTiles[plan.tile];
    double cost[TABLE], all = 0.0, number = 0.0, load[8] = {};
    int order[TABLE];
    for (int i = 0; i < args.s.count; ++i) {
        cost[i] = (double)tiles_of<KIND>(args.t[i], k.rows, k.cols) * ((KIND == kGram ? args.t[i].N : args.t[i].M) / 32 * k.step + k.ends);
        all += cost[i];
        number += tiles_of<KIND>(args.t[i], k.rows, k.cols);
        order[i] = i;
    }
    if (number <= kCutRounds * k.slots) {
        plan.cuts = true;
        double before = 0.0;
        for (int i = 0; i < args.s.count; ++i) {
            const int tiles = tiles_of<KIND>(args.t[i], k.rows, k.cols);
            for (int d = 0; d <= 8; ++d) plan.cut[d] += (int)std::min<double>(tiles, std::max(0.0, std::round((all * d / 8 - before) / cost[i] * tiles)));
            before += cost[i];
        }
        return plan;
    }
    for (int i = 0; i < args.s.count; ++i) {
        int dies = 1;
        while (dies < 8 && cost[i] / dies > all / 16) dies *= 2;
        plan.dies[i] = (uint8_t)dies;
        cost[i] /= dies;
    }
    std::stable_sort(order, order + args.s.count, [&](int a, int b) { return cost[a] > cost[b]; });
    for (int n = 0; n < args.s.count; ++n) {             // the largest parts first, each to the dies that have least
        const int i = order[n], dies = plan.dies[i];
        int best = n & 7;                                // (for all dies: another one begins each time)
        if (dies < 8) {
            double least = 1e30;
            for (int d = 0; d < 8; ++d) {
                double most = 0.0;
                for (int q = 0; q < dies; ++q) most = std::max(most, load[(d + q) & 7]);
                if (most < least) {
                    least = most;
                    best = d;
                }
            }
        }
        plan.die[i] = (uint8_t)best;
        for (int q = 0; q < dies; ++q) load[(best + q) & 7] += cost[i];
    }
    return plan;
}

template <Product KIND, bool MUON, typename T, int TM, int TN, int WM, int WN, int NS, int TABLE>
bool launch_product(Args<TABLE>& args, hipStream_t stream) {
    constexpr int lds = std::max(NS * (TM * WM + TN * WN) * 16 * 128, WM * WN * TM * 16 * (leaving_columns(TN) * 16 + 4) * 4);
    int i = 0;
    int blocks = set_starts(args, [&](const Mat& t) {
        const int tiles = tiles_of<KIND>(t, 16 * TM * WM, 16 * TN * WN), dies = args.dies[i++];
        return args.cuts ? tiles : (tiles + dies - 1) / dies * 8;
    });
    if (args.cuts) {
        blocks = 0;
        for (int d = 0; d < 8; ++d) blocks = std::max(blocks, (args.cut[d + 1] - args.cut[d]) * 8);
    }
    static const bool once = hipFuncSetAttribute(reinterpret_cast<const void*>(ns_product_kernel<KIND, MUON, T, TM, TN, WM, WN, NS, TABLE>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
    if (once) hipLaunchKernelGGL((ns_product_kernel<KIND, MUON, T, TM, TN, WM, WN, NS, TABLE>), dim3((unsigned)blocks), dim3(WM * WN * 64), lds, stream, args);
    return once;
}
template <Product KIND, bool MUON, typename T, int TABLE>
bool launch_product(Args<TABLE>& args, const LaunchPlan<TABLE>& plan, hipStream_t stream) {
    std::copy(plan.dies, plan.dies + TABLE, args.dies);
    std::copy(plan.die, plan.die + TABLE, args.die);
    args.cuts = plan.cuts;
    std::copy(plan.cut, plan.cut + 9, args.cut);
    switch (plan.tile) {
        case kTile64: return launch_product<KIND, MUON, T, 2, 2, 2, 2, 4>(args, stream);
        case kTile128One: return launch_product<KIND, MUON, T, 2, 4, 4, 2, 4>(args, stream);
        case kTile192: return launch_product<KIND, MUON, T, 6, 3, 2, 4, 3>(args, stream);
        case kTile256:
            if constexpr (KIND >= kNext) return launch_product<KIND, MUON, T, 4, 4, 4, 2, 3>(args, stream);
        default: return launch_product<KIND, MUON, T, 4, 4, 2, 2, 2>(args, stream);
    }
}

template <bool MUON, typename T, int TABLE>
lc_status run_group(Args<TABLE>& args, int iterations, bool all_small, hipStream_t stream) {
    if (all_small) {
        constexpr int lds = 2 * kSmallM * kSmallN * 4 + kSmallM * kSmallM * 4;
        static const bool once = hipFuncSetAttribute(reinterpret_cast<const void*>(ns_small_kernel<T, MUON, TABLE>), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
        if (once) hipLaunchKernelGGL((ns_small_kernel<T, MUON, TABLE>), dim3((unsigned)args.s.count), dim3(kSmallThreads), lds, stream, args, iterations);
        return once ? LC_OK : LC_ERR_LAUNCH;
    }
    int blocks = set_starts(args, [](const Mat& t) {
        const long long v = MUON ? ((long long)t.rows * t.cols + 3) / 4 : (long long)t.rows * ((t.cols + 3) / 4);
        return (v + t.chunk - 1) / t.chunk;
    });
    hipLaunchKernelGGL((ns_squares_kernel<T, MUON, TABLE>), dim3((unsigned)blocks), dim3(256), 0, stream, args);
    blocks = set_starts(args, [](const Mat& t) { return (long long)((t.M + 63) / 64) * ((t.N + 63) / 64); });
    hipLaunchKernelGGL((ns_split_kernel<T, MUON, TABLE>), dim3((unsigned)blocks), dim3(256), 0, stream, args);
    const auto gram = plan_of<kGram>(args), square = plan_of<kSquare>(args), next = plan_of<kNext>(args);
    bool ok = true;
    for (int i = 0; i < iterations && ok; ++i) {
        args.s.which = i & 1;
        ok = launch_product<kGram, false, float>(args, gram, stream) && launch_product<kSquare, false, float>(args, square, stream) &&
             (i + 1 < iterations ? launch_product<kNext, false, float>(args, next, stream)
                                 : launch_product<kLast, MUON, std::conditional_t<MUON, float, T>>(args, next, stream));
    }
    return ok ? LC_OK : LC_ERR_LAUNCH;
}

template <bool MUON, typename T, int TABLE>
lc_status run_group(const std::vector<Matrix>& all, const std::vector<int>& order, size_t first, size_t n, const Scalars& s, int iterations, bool all_small,
                    void* workspace, hipStream_t stream) {
    Args<TABLE> args;
    args.s = s;
    args.s.count = (int)n;
    unsigned char* base = static_cast<unsigned char*>(workspace);
    for (size_t i = 0; i < n; ++i) {
        const Matrix& a = all[order[first + i]];
        const long long vectors = MUON ? ((long long)a.rows * a.cols + 3) / 4 : (long long)a.rows * ((a.cols + 3) / 4);
        Mat& t = args.t[i];
        t = Mat{a.in, a.m, a.w, a.out, a.ld, a.rows, a.cols, (int)padded(std::min(a.rows, a.cols)), (int)padded(std::max(a.rows, a.cols)), a.rows > a.cols,
                (int)std::max<long long>(1024, ((vectors + kMostParts - 1) / kMostParts + 255) / 256 * 256), base, a.step, a.lr_decay};
        base += bytes_of(a.rows, a.cols);
    }
    return run_group<MUON, T, TABLE>(args, iterations, all_small, stream);
}

template <bool MUON, typename T>
lc_status run_all(const std::vector<Matrix>& all, std::vector<int>& order, const int* rows, const int* cols, const Scalars& s, int iterations, void* workspace,
                  hipStream_t stream) {
    lc_status st = LC_OK;
    for_groups(order, rows, cols, [&](size_t first, size_t n, long long) {
        if (st != LC_OK) return;
        // (in a group with larger ones small matrices cost next to nothing; a launch of their own would be one more.  One of 330 x 350 and 300 of 64 x 256 491 us where all groups went by the first's sizes, so 295; each of
        // the two alone 114 and 219)
        const bool all_small = std::all_of(order.begin() + first, order.begin() + first + n, [&](int i) { return small((int)padded(std::min(rows[i], cols[i])), (int)padded(std::max(rows[i], cols[i]))); });
        st = n <= kSmallTable ? run_group<MUON, T, kSmallTable>(all, order, first, n, s, iterations, all_small, workspace, stream)
                              : run_group<MUON, T, kTable>(all, order, first, n, s, iterations, all_small, workspace, stream);
    });
    return st;
}

bool bad_side(int n) { return n < 0 || n > kMostSide; }

lc_status check_desc(const lc_newton_schulz_desc* d) {
    if (!d) return LC_ERR_NULL;
    if (d->dtype != LC_F32 && d->dtype != LC_BF16) return LC_ERR_UNSUPPORTED;
    if (d->batch < 0 || d->rows <= 0 || d->cols <= 0 || bad_side(d->rows) || bad_side(d->cols) || (d->ld && d->ld < d->cols) || d->ld > (int64_t)1 << 40) return LC_ERR_SHAPE;
    long long bytes;
    if (__builtin_mul_overflow((long long)d->batch * d->rows, std::max<long long>(d->ld, d->cols), &bytes) || __builtin_mul_overflow(bytes, 4ll, &bytes)) return LC_ERR_SHAPE;
    if (d->iterations < 1 || d->iterations > kMostIterations || !(d->eps >= 0.f)) return LC_ERR_UNSUPPORTED;
    return LC_OK;
}

// Whether a list's sides are right; the places of what is not empty.
lc_status check_sides(int n, const int* rows, const int* cols, std::vector<int>* order) {
    if (n < 0) return LC_ERR_SHAPE;
    if (n > 0 && (!rows || !cols)) return LC_ERR_NULL;
    for (int i = 0; i < n; ++i) {
        if (bad_side(rows[i]) || bad_side(cols[i])) return LC_ERR_SHAPE;
        if (rows[i] && cols[i]) order->push_back(i);
    }
    return LC_OK;
}

size_t ns_bytes(const lc_newton_schulz_desc* d) {
    std::vector<int> order(std::min(d->batch, kTable)), rows(order.size(), d->rows), cols(order.size(), d->cols);
    for (size_t i = 0; i < order.size(); ++i) order[i] = (int)i;
    return workspace_of(order, rows.data(), cols.data());
}

}  // namespace

extern "C" size_t newton_schulz_workspace_bytes(const lc_newton_schulz_desc* desc) {
    if (check_desc(desc) != LC_OK) return 0;
    try {
        return ns_bytes(desc);
    } catch (...) {
        return 0;
    }
}

extern "C" lc_status newton_schulz(const lc_newton_schulz_desc* desc, const void* x, void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const lc_status st = check_desc(desc);
    if (st != LC_OK) return st;
    if (desc->batch == 0) return LC_OK;
    if (!x || !y) return LC_ERR_NULL;
    const size_t e = desc->dtype == LC_BF16 ? 2 : 4;
    if (lc_off_element(x, e) || lc_off_element(y, e)) return LC_ERR_ALIGN;
    try {
        if (!workspace || (((uintptr_t)workspace) & 255) || workspace_bytes < ns_bytes(desc)) return LC_ERR_WORKSPACE;
        const long long ld = desc->ld ? desc->ld : desc->cols;
        std::vector<Matrix> all(desc->batch);
        std::vector<int> order(desc->batch), rows(desc->batch, desc->rows), cols(desc->batch, desc->cols);
        for (int i = 0; i < desc->batch; ++i) {
            order[i] = i;
            all[i] = Matrix{static_cast<const unsigned char*>(x) + (size_t)i * desc->rows * ld * e, nullptr, nullptr,
                            static_cast<unsigned char*>(y) + (size_t)i * desc->rows * desc->cols * e, ld, desc->rows, desc->cols, 0.f, 0.f};
        }
        const Scalars s{0, nullptr, 0.f, desc->eps, 0, 0};
        lc_begin_call();
        const lc_status run = desc->dtype == LC_BF16
                                  ? run_all<false, uint16_t>(all, order, rows.data(), cols.data(), s, desc->iterations, workspace, static_cast<hipStream_t>(hip_stream))
                                  : run_all<false, float>(all, order, rows.data(), cols.data(), s, desc->iterations, workspace, static_cast<hipStream_t>(hip_stream));
        const lc_status end = lc_end_call();
        return run != LC_OK ? run : end;
    } catch (...) {                                 // (host lists that do not fit)
        return LC_ERR_SHAPE;
    }
}

extern "C" size_t muon_workspace_bytes(int n_tensors, const int* rows, const int* cols) {
    try {
        std::vector<int> order;
        return check_sides(n_tensors, rows, cols, &order) == LC_OK ? workspace_of(order, rows, cols) : 0;
    } catch (...) {
        return 0;
    }
}

extern "C" lc_status muon_step(int n_tensors, float* const* w, const void* const* g, lc_dtype g_dtype, float* const* m, const int* rows, const int* cols, float lr,
                               float momentum, int nesterov, float weight_decay, int iterations, float eps, const float* scale_per_tensor,
                               const float* weight_decay_per_tensor, const float* grad_scale, void* const* w_lowp_out, void* workspace, size_t workspace_bytes,
                               void* hip_stream) {
    if (g_dtype != LC_F32 && g_dtype != LC_BF16) return LC_ERR_UNSUPPORTED;
    if (iterations < 1 || iterations > kMostIterations || !(eps >= 0.f) || !(momentum >= 0.f && momentum < 1.f)) return LC_ERR_UNSUPPORTED;
    try {
        std::vector<int> order;
        const lc_status st = check_sides(n_tensors, rows, cols, &order);
        if (st != LC_OK) return st;
        if (order.empty()) return LC_OK;
        if (!w || !g || !m) return LC_ERR_NULL;
        if (lc_off_element(grad_scale, 4)) return LC_ERR_ALIGN;
        std::vector<Matrix> all(n_tensors);
        for (int i : order) {
            if (!w[i] || !g[i] || !m[i]) return LC_ERR_NULL;
            void* const lowp = w_lowp_out ? w_lowp_out[i] : nullptr;
            if (lc_off_element(w[i], 4) || lc_off_element(m[i], 4) || lc_off_element(g[i], g_dtype == LC_BF16 ? 2 : 4) || lc_off_element(lowp, 2)) return LC_ERR_ALIGN;
            const double scale = scale_per_tensor ? scale_per_tensor[i] : std::sqrt(std::max(1.0, (double)rows[i] / cols[i]));
            all[i] = Matrix{g[i], m[i], w[i], lowp, cols[i], rows[i], cols[i], (float)(lr * scale),
                            (float)((double)lr * (weight_decay_per_tensor ? weight_decay_per_tensor[i] : weight_decay))};
        }
        if (!workspace || (((uintptr_t)workspace) & 255) || workspace_bytes < workspace_of(order, rows, cols)) return LC_ERR_WORKSPACE;
        const Scalars s{0, grad_scale, momentum, eps, nesterov != 0, 0};
        lc_begin_call();
        const lc_status run = g_dtype == LC_BF16 ? run_all<true, uint16_t>(all, order, rows, cols, s, iterations, workspace, static_cast<hipStream_t>(hip_stream))
                                                 : run_all<true, float>(all, order, rows, cols, s, iterations, workspace, static_cast<hipStream_t>(hip_stream));
        const lc_status end = lc_end_call();
        return run != LC_OK ? run : end;
    } catch (...) {
        return LC_ERR_SHAPE;
    }
}
