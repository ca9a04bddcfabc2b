// Lookup of token embeddings with a scale, and the gradient of their table, for gfx950.
//
// out[i] = scale * table[t_i];  dtable[v] (+)= scale * sum over the places i with t_i = v of dout[i], in a fixed order and without atomics: places are sorted by token (stable), the sorted
// list is cut into pieces of equal length, and a wave sums the rows of a token within a piece.  A token that lies within one is written at once; one that crosses pieces leaves a part in each, which
// are added up in a second launch, in 64 bits.  A token may occur any number of times.  Bound by memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "token_common.h"

namespace {

constexpr int kNone = 0x7fffffff;                  // the key of a place whose token is outside the table: behind all others

__device__ __forceinline__ int key_of(const int32_t* tokens, long long i, int vocab) {
    const int t = tokens[i];
    return t >= 0 && t < vocab ? t : kNone;
}

// What a row's columns are: a multiple of 8, another number from 8 on, or fewer.
enum Columns { kByEights, kFromEight, kUnderEight };

// Eight columns of a row, loaded (issue) and put in their places (settle) apart, so that loads of several rows are under way.  NT: past the caches.
template <Columns COLS, bool NT = false, typename T>
__device__ __forceinline__ void issue(Packed<T>& to, const T* row, int col, int c) {
    if constexpr (COLS == kByEights) to.template load<NT>(row + col);
    else if constexpr (COLS == kFromEight) to.template load<NT>(row + min(col, c - 8));
    else to.load_some(row, c, 0u);
}
template <Columns COLS, typename T>
__device__ __forceinline__ void settle(Packed<T>& x, int col, int c) {
    if constexpr (COLS == kFromEight) {
        if (c - col < 8) x.shift(8 - (c - col), 0u);
    }
}

// ---------------------------------------------------------------------------------------------- lookup

struct LookupArgs {
    const void* table;
    const int32_t* tokens;
    void* out;
    long long rows, table_ld;
    int vocab, c, lane_bits;   // a row has 2^lane_bits lanes, up to the block's 256
    float scale;
};

// Some lanes a row, eight columns a lane and access, kRowsAhead rows of a block (their tokens, then their values) under way at a time, neighbours unless every block has one at most.  16384 of 2048 bf16 20 to 22 us (4.9 to 5.4 TB/s), one 2.0.
// (By themselves, us, four rows a grid apart / two neighbours: 16384 x 2048 bf16 22.4 / 21.0, 30000 39.0 / 37.6, 8000 x 8200 52.6 / 50.6, 30011 x 1537 fp32 60 / 56.)
// PAST: out goes past the caches.
constexpr int kRowsAhead = 2;
template <typename S, typename T, Columns COLS, bool PAST>
__global__ void __launch_bounds__(256) embedding_fwd_kernel(const LookupArgs p) {
    const int lanes = 1 << p.lane_bits, lane = threadIdx.x & (lanes - 1), each = 256 >> p.lane_bits;
    const bool few = gridDim.x * (long long)each >= p.rows;
    const long long stride = few ? (long long)gridDim.x * each : each;
    for (long long row = (long long)blockIdx.x * each * (few ? 1 : kRowsAhead) + (threadIdx.x >> p.lane_bits); row < p.rows; row += (long long)gridDim.x * each * kRowsAhead) {
        int key[kRowsAhead];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) key[u] = key_of(p.tokens, std::min(row + u * stride, p.rows - 1), p.vocab);
        for (long long col = lane * 8; col < p.c; col += lanes * 8) {
            Packed<S> x[kRowsAhead];
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) issue<COLS>(x[u], static_cast<const S*>(p.table) + (key[u] == kNone ? 0 : key[u]) * p.table_ld, (int)col, p.c);
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {
                if (row + u * stride >= p.rows) break;
                settle<COLS>(x[u], (int)col, p.c);
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = key[u] == kNone ? 0.f : x[u].get(j) * p.scale;
                lc_store8<PAST>(static_cast<T*>(p.out) + (row + u * stride) * p.c + col, v, COLS == kByEights ? 8 : p.c - (int)col);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- order

struct SortArgs {
    const int32_t* tokens;     // of the first pass; later ones take keys and places
    const int* key_in;
    const int* place_in;
    int* key;
    int* place;
    int* counts;               // [blocks][bins]
    int rows, vocab, per, shift, bits;
    int sort_blocks;           // blocks behind them write zeros to
    float* zeros;              // this many bytes (a share of the table, whose rows that do not occur are to be zero)
    long long zero_bytes;
};

// Zeros past the caches, by the blocks of a sorting launch that have nothing to sort: few places keep few units busy, and their order is latency.  One vector a thread (two to 16 of them, 1024 blocks in all: with the rest of
// a pass 4096 places of 32768 x 2048 97 us, so 74; 64 of 130000 x 4096, 2.1 GB, 580, so 372).
__device__ __forceinline__ void fill_share(const SortArgs& p, int threads) {
    if ((int)blockIdx.x == p.sort_blocks && threadIdx.x < (p.zero_bytes & 15) / 4) p.zeros[p.zero_bytes / 16 * 4 + threadIdx.x] = 0.f;
    const long long vectors = p.zero_bytes / 16, step = (long long)(gridDim.x - p.sort_blocks) * threads;
    for (long long v = (long long)(blockIdx.x - p.sort_blocks) * threads + threadIdx.x; v < vectors; v += step) lc_store16<true>(p.zeros + v * 4, lc_u32x4{0u, 0u, 0u, 0u});
}

// Few places (3064 in a table of 10836 x 2048, with the lookup and all else 44 us): a block ranks 64 of them against all, which it holds in LDS; each of its 16 waves a share of them.
constexpr int kRankMost = 6144;
__global__ void __launch_bounds__(1024) embedding_rank_kernel(const SortArgs p) {
    if ((int)blockIdx.x >= p.sort_blocks) {
        fill_share(p, 1024);
        return;
    }
    __shared__ __attribute__((aligned(16))) int keys[kRankMost];
    __shared__ int before[16][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, padded = (p.rows + 63) & ~63;
    for (int i = tid; i < padded; i += 1024) keys[i] = i < p.rows ? key_of(p.tokens, i, p.vocab) : kNone;
    __syncthreads();
    const int mine = blockIdx.x * 64 + lane, key = keys[min(mine, padded - 1)];
    int n = 0;
    for (int group = wave; group < padded / 64; group += 16) {        // all of a group lies before the block's own, is it, or lies behind it
        const int4* k = reinterpret_cast<const int4*>(keys + group * 64);
        if (group < blockIdx.x) {
#pragma unroll 4
            for (int i = 0; i < 16; ++i) n += (k[i].x <= key) + (k[i].y <= key) + (k[i].z <= key) + (k[i].w <= key);
        } else if (group > blockIdx.x) {
#pragma unroll 4
            for (int i = 0; i < 16; ++i) n += (k[i].x < key) + (k[i].y < key) + (k[i].z < key) + (k[i].w < key);
        } else {
            for (int i = 0; i < 64; ++i) n += keys[group * 64 + i] < key || (keys[group * 64 + i] == key && i < lane);
        }
    }
    before[wave][lane] = n;
    __syncthreads();
    if (wave == 0 && mine < p.rows) {
        n = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) n += before[w][lane];
        p.key[n] = key;
        p.place[n] = mine;
    }
}

// More of them: passes over digits of `bits` bits from the lowest up.  A block counts the digits of its stretch ...
constexpr int kMostBits = 10, kSortBlocks = 128;
__device__ __forceinline__ int sort_key(const SortArgs& p, int i) { return p.tokens ? min(key_of(p.tokens, i, p.vocab), p.vocab) : p.key_in[i]; }       // (outside: one above the last)
__global__ void __launch_bounds__(1024) embedding_count_kernel(const SortArgs p) {
    if ((int)blockIdx.x >= p.sort_blocks) {
        fill_share(p, 1024);
        return;
    }
    __shared__ int count[1 << kMostBits];
    const int bins = 1 << p.bits, first = blockIdx.x * p.per, end = min(p.rows, first + p.per);
    for (int d = threadIdx.x; d < bins; d += 1024) count[d] = 0;
    __syncthreads();
    for (int i = first + threadIdx.x; i < end; i += 1024) atomicAdd(&count[(sort_key(p, i) >> p.shift) & (bins - 1)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += 1024) p.counts[blockIdx.x * bins + d] = count[d];
}
// ... and moves it: where a digit's places of the block begin follows from all blocks' counts, where a wave's begin from its share's, and within a wave places keep their order.
__global__ void __launch_bounds__(1024) embedding_move_kernel(const SortArgs p) {
    if ((int)blockIdx.x >= p.sort_blocks) {
        fill_share(p, 1024);
        return;
    }
    constexpr int kBins = 1 << kMostBits;
    __shared__ int next[16][kBins];
    __shared__ int sums[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bins = 1 << p.bits;
    const int first = blockIdx.x * p.per, end = min(p.rows, first + p.per), share = (p.per / 16 + 63) & ~63;
    const int from = min(end, first + wave * share), to = min(end, from + share);
    for (int d = tid; d < 16 * kBins; d += 1024) (&next[0][0])[d] = 0;
    __syncthreads();
    for (int i = from + lane; i < to; i += 64) atomicAdd(&next[wave][(sort_key(p, i) >> p.shift) & (bins - 1)], 1);
    int total = 0, before = 0;                     // of digit tid over all blocks; over those before this one
    if (tid < bins) {
#pragma unroll 8
        for (int b = 0; b < p.sort_blocks; ++b) {
            const int n = p.counts[b * bins + tid];
            total += n;
            before += b < blockIdx.x ? n : 0;
        }
    }
    int upto = total;                              // sums over digits: within a wave, then over waves
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int other = __shfl_up(upto, off, 64);
        upto += lane >= off ? other : 0;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += sums[w];
    if (tid < bins) {
        int at = upto - total + before;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            const int n = next[w][tid];
            next[w][tid] = at;
            at += n;
        }
    }
    __syncthreads();
    for (int i0 = from; i0 < to; i0 += 64) {
        const int i = i0 + lane;
        const bool in = i < to;
        const int key = in ? sort_key(p, i) : 0, digit = (key >> p.shift) & (bins - 1);
        unsigned long long same = __ballot(in);
        for (int b = 0; b < p.bits; ++b) {
            const unsigned long long set = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        int at = 0;
        if (in) at = next[wave][digit];
        asm volatile("" : : : "memory");               // (a wave's LDS accesses stay in order: all have read before one writes)
        if (in) {
            if (rank == 0) next[wave][digit] = at + __popcll(same);
            p.key[at + rank] = key;
            p.place[at + rank] = p.tokens ? i : p.place_in[i];
        }
        asm volatile("" : : : "memory");
    }
}

// ---------------------------------------------------------------------------------------------- sums

struct SumArgs {
    const int* key;            // sorted; what counts is below vocab
    const int* place;
    const void* dout;
    float* dtable;
    float* part;               // [pieces][2][c]: of the token that a piece begins with and an earlier one holds too; of the one that it ends with and that goes on
    long long pieces;          // of kPiece places
    int rows, vocab, c;
    int lane_bits, tiles;      // 2^lane_bits lanes take 8 columns each of a part of a row; how many parts a row has
    float scale;
};

constexpr int kPiece = 32;     // places whose rows one wave sums (16: sums as fast, their joining 2 to 13 us slower)

// Eight columns of a sum to their place: the table's, where nothing else of the token is, or the piece's part of it.
template <Columns COLS, bool ADD>
__device__ __forceinline__ void leave(const SumArgs& p, long long piece, int key, bool continued, bool goes_on, int col, const float* acc, Packed<float>& old) {
    const bool whole = !continued && !goes_on;
    float* const to = (whole ? p.dtable + (long long)key * p.c : p.part + (piece * 2 + (continued ? 0 : 1)) * p.c) + col;
    float v[8];
    if constexpr (ADD) settle<COLS>(old, col, p.c);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = ADD && whole ? fmaf(acc[j], p.scale, old.get(j)) : acc[j] * p.scale;
    lc_store8(to, v, COLS == kByEights ? 8 : p.c - col);
}

// A wave sums the rows of a piece, 512 columns of them: keys and places first, then AHEAD rows at a time, then their sums and stores.  No load stands behind a branch, and few behind a store: a wave's loads and stores
// complete in order, so that waiting for one waits for all before it.  16384 rows of 2048 bf16 (5600 tokens, 117 MB) 27.5 us, 30011 of 1537 fp32 added to what is there 77 (321 MB, 4.2 TB/s); a wave for each place, most of which are
// not a token's first, 40 where this took 31, with a longer joining.  Rows in whole lines are read past the caches, which nothing asks for them again (behind what
// wrote them: 16384 of 2048 bf16 109 us for 114, 30000 159 for 173; fp32, a line of which takes two loads, 155 for 155 and 81 for 78).  Sequential rows in the place of a token's take as long; without the stores 19 of 31: all waves load, then all store.
template <typename T, Columns COLS, bool ADD, int AHEAD>
__global__ void __launch_bounds__(256) embedding_sum_kernel(const SumArgs p) {
    const int lane = threadIdx.x & 63;
    const unsigned wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const unsigned piece = wave / (unsigned)p.tiles, tile0 = wave - piece * (unsigned)p.tiles;
    if (piece >= (unsigned)p.pieces) return;
    const int first = (int)piece * kPiece, n = std::min(kPiece, p.rows - first);
    const int at = std::min(std::max(first - 1 + lane, 0), p.rows - 1);       // lane 0: the place before the piece, lane n + 1: the one behind it
    int keys = p.key[at];
    const int places = p.place[at];
    if (first - 1 + lane < 0 || first - 1 + lane >= p.rows || keys >= p.vocab) keys = kNone;
    const T* const dout = static_cast<const T*>(p.dout);
    const auto key_of_place = [&](int k) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(keys, k + 1); };
    const int before = key_of_place(-1);
    const int own = ((int)tile0 * 64 + lane) * 8, col = std::min(own, COLS == kByEights ? p.c - 8 : p.c);
    float acc[8] = {};
#pragma unroll
    for (int ahead = 0; ahead < kPiece; ahead += AHEAD) {
        if (ahead >= n) break;
        Packed<T> x[AHEAD];
        Packed<float> old[ADD ? AHEAD : 1];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int row = __builtin_amdgcn_readlane(places, std::min(ahead + u, n - 1) + 1);
            issue<COLS, COLS == kByEights && sizeof(T) == 2>(x[u], dout + (long long)row * p.c, col, p.c);
            if constexpr (ADD) {
                const int key = key_of_place(std::min(ahead + u, n - 1));
                issue<COLS>(old[u], p.dtable + (long long)(key == kNone ? 0 : key) * p.c, col, p.c);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int k = ahead + u;
            if (k >= n) break;
            const int key = key_of_place(k);
            settle<COLS>(x[u], col, p.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += x[u].get(j);
            const bool last = k + 1 == n, ends = last || key_of_place(k + 1) != key;
            if (!ends) continue;
            if (key != kNone && own < p.c)
                leave<COLS, ADD>(p, piece, key, before == key, last && key_of_place(k + 1) == key, own, acc, old[ADD ? u : 0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        }
    }
}

// Rows of fewer columns than a wave takes: 2^lane_bits lanes a row sum a token's rows from a place to the end of its piece, if the token or the piece begins there.
template <typename T, Columns COLS, bool ADD>
__global__ void __launch_bounds__(256) embedding_sum_narrow_kernel(const SumArgs p) {
    const int lanes = 1 << p.lane_bits, lane = threadIdx.x & (lanes - 1), of = threadIdx.x & 63 & ~(lanes - 1);       // the first of these lanes in the wave
    const long long first = ((long long)blockIdx.x * 256 + threadIdx.x) >> p.lane_bits;
    if (first >= p.rows) return;
    const int i = (int)first, end = std::min(p.rows, (i / kPiece + 1) * kPiece), at0 = std::min(i + lane, end - 1);
    const int mine = p.key[at0], place = p.place[at0], before = i > 0 ? p.key[i - 1] : kNone, behind = end < p.rows ? p.key[end] : kNone;
    const int key = __shfl(mine, of, 64);
    if (key >= p.vocab || (before == key && i % kPiece != 0)) return;
    // the token's places: lanes look at the next keys, as many at a time as they are
    const unsigned long long every = p.lane_bits == 6 ? ~0ull : (1ull << lanes) - 1;
    const auto run_of = [&](bool same) __attribute__((always_inline)) {
        const unsigned long long bits = __ballot(same) >> of;
        return (bits & every) == every ? lanes : __builtin_ctzll(~bits);
    };
    int n = run_of(i + lane < end && mine == key);
    for (int run = n; run == lanes && i + n < end; n += run) run = run_of(i + n + lane < end && p.key[std::min(i + n + lane, end - 1)] == key);
    const bool goes_on = i + n == end && behind == key, continued = before == key;
    const T* const dout = static_cast<const T*>(p.dout);
    const int own = lane * 8, col = std::min(own, COLS == kByEights ? p.c - 8 : p.c);       // lanes past the row go along: the others ask them for places
    Packed<float> old;
    if constexpr (ADD) issue<COLS>(old, p.dtable + (long long)key * p.c, col, p.c);
    constexpr int U = 4;                           // rows under way
    float acc[8] = {};
    int places = place;
    for (int k = 0; k < n; k += U) {
        if (k > 0 && (k & (lanes - 1)) == 0) places = p.place[std::min(i + k + lane, end - 1)];
        Packed<T> x[U];
        int row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) row[u] = __shfl(places, of + (std::min(k + u, n - 1) & (lanes - 1)), 64);
#pragma unroll
        for (int u = 0; u < U; ++u) issue<COLS>(x[u], dout + (long long)row[u] * p.c, col, p.c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            settle<COLS>(x[u], col, p.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += k + u < n ? x[u].get(j) : 0.f;
        }
    }
    if (own < p.c) leave<COLS, ADD>(p, i / kPiece, key, continued, goes_on, own, acc, old);
}

// Tokens that cross pieces: the lanes of the piece where one begins add up its parts in the order of the pieces, eight at a time in a tree, and those sums in 64 bits: in 32 the error of a token that fills a batch would grow with
// its places (the same gradient at each of 140000 932 x 2^-24 of the sum, so 10; at 2^25 of them 0.4 %, so 2).  One group of lanes adds all parts of a token's columns, one eight after another: places spread evenly / half of them / all
// of them one token's, the gradient whole, us: 131072 of 5000 x 512 bf16 66 / 252 / 438 (in 32 bits 65 / 245 / 423), 16384 of 32768 x 2048 bf16 85 / 101 / 110, 30011 of 50021 x 1537 fp32 added 111 / 170 / 189, 65536 of
// 32000 x 64 bf16 32 / 166 / 291.
template <Columns COLS, bool ADD>
__global__ void __launch_bounds__(256) embedding_join_kernel(const SumArgs p) {
    const int lanes = 1 << p.lane_bits, lane = threadIdx.x & (lanes - 1), of = threadIdx.x & 63 & ~(lanes - 1);
    const unsigned group = (blockIdx.x * 256u + threadIdx.x) >> p.lane_bits, piece = group / (unsigned)p.tiles, tile = group - piece * (unsigned)p.tiles;
    if ((long long)piece + 1 >= p.pieces) return;
    const long long end = ((long long)piece + 1) * kPiece;
    const int key = p.key[end - 1], behind = p.key[end], start = p.key[end - kPiece], before = piece > 0 ? p.key[end - kPiece - 1] : kNone;
    if (key >= p.vocab || behind != key || (start == key && before == key)) return;          // (the last: it began earlier)
    const unsigned long long every = p.lane_bits == 6 ? ~0ull : (1ull << lanes) - 1;
    const int own = ((int)tile * lanes + lane) * 8, col = std::min(own, COLS == kByEights ? p.c - 8 : p.c);
    constexpr int U = 8;                           // parts under way
    double acc[8];
    Packed<float> x[U], old;
    issue<COLS>(x[0], p.part + ((long long)piece * 2 + 1) * p.c, col, p.c);
    if constexpr (ADD) issue<COLS>(old, p.dtable + (long long)key * p.c, col, p.c);
    settle<COLS>(x[0], col, p.c);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = x[0].get(j);
    for (long long next = (long long)piece + 1;;) {       // lanes look at the next pieces' first keys, as many at a time as they are
        const long long mine = next + lane;
        const unsigned long long bits = __ballot(mine < p.pieces && p.key[std::min(mine, p.pieces - 1) * kPiece] == key) >> of;
        const int run = (bits & every) == every ? lanes : __builtin_ctzll(~bits);
        for (int k = 0; k < run; k += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) issue<COLS>(x[u], p.part + (next + std::min(k + u, run - 1)) * 2 * p.c, col, p.c);
#pragma unroll
            for (int u = 0; u < U; ++u) settle<COLS>(x[u], col, p.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = k + u < run ? x[u].get(j) : 0.f;
                acc[j] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            }
        }
        next += run;
        if (run < lanes) break;
    }
    if (own >= p.c) return;
    if constexpr (ADD) {
        settle<COLS>(old, col, p.c);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += old.get(j);
    }
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)acc[j];
    lc_store8(p.dtable + (long long)key * p.c + own, v, COLS == kByEights ? 8 : p.c - own);
}

// ---------------------------------------------------------------------------------------------- host

constexpr long long kMostBlocks = 1 << 20;
constexpr long long kMostRows = 1ll << 25;        // a launch holds fewer than 2^32 threads, and a row has 64 of them at most

// Bytes of out from which it goes past the caches.  us, three sets in turn, ordinary / past: 24000 x 2048 bf16 (98 MB) 32.3 / 24.6, 40000 (164 MB) 51 / 39, 30011 x 1537 fp32 (184 MB) with the gradient 193 / 181 (then); but with a
// layer norm of out behind it 30000 x 2048 bf16 84 / 86, 40000 113 / 114, 60000 162 / 163, 100000 273 / 272, fp32 16000 (131 MB) 111 / 117, 20000 136 / 143, 30011 x 1537 160 / 161.
constexpr long long kPastBytes = 160 << 20;

lc_status check_desc(const lc_embedding_desc* d) {
    if (!d) return LC_ERR_NULL;
    if ((d->dtype != LC_F32 && d->dtype != LC_BF16) || (d->table_dtype != LC_F32 && d->table_dtype != LC_BF16)) return LC_ERR_UNSUPPORTED;
    if (d->rows < 0 || d->rows > kMostRows || d->vocab <= 0 || d->vocab > 1 << 30 || d->c <= 0 || d->c > 1 << 30 || (d->table_ld && d->table_ld < d->c)) return LC_ERR_SHAPE;
    long long bytes;
    if (__builtin_mul_overflow((long long)d->rows, (long long)d->c * 4, &bytes) ||
        __builtin_mul_overflow((long long)d->vocab, std::max<long long>(d->table_ld, d->c), &bytes) || __builtin_mul_overflow(bytes, 4ll, &bytes))
        return LC_ERR_SHAPE;
    return LC_OK;
}

template <typename F>
void by_columns(int c, F&& f) {
    c % 8 == 0 ? f.template operator()<kByEights>() : c > 8 ? f.template operator()<kFromEight>() : f.template operator()<kUnderEight>();
}

int lanes_of(int c) {                              // the smallest power of two from 8 on that takes a row at once, a block's threads at most
    int lanes = 8;
    while (lanes < 256 && lanes * 8 < c) lanes *= 2;
    return lanes;
}

// How the gradient is made, and where things lie in the workspace.
struct Plan {
    int lanes, tiles, passes, bits, per, sort_blocks;
    long long pieces, part_at, bytes;
};
Plan plan_of(const lc_embedding_desc* d) {
    Plan p{};
    const long long rows = d->rows;
    p.lanes = std::min(64, lanes_of(d->c));
    p.tiles = (int)(((long long)d->c + p.lanes * 8 - 1) / (p.lanes * 8));
    p.pieces = (rows + kPiece - 1) / kPiece;
    int bits = 1;
    while (bits < 31 && (1ll << bits) <= d->vocab) ++bits;                         // keys up to vocab
    const int passes = (bits + kMostBits - 1) / kMostBits;
    // ranks against all go by the square of the places: 5000 of 256 bf16 columns with the lookup, us, in passes / ranked: one pass 24 / 25, two 32 / 25; 8192 24.6 / 30, 32 / 30, and with 160 MB of zeros 56 / 57
    if (rows > (passes > 1 ? kRankMost : 4096)) {
        p.passes = passes;
        p.bits = (bits + p.passes - 1) / p.passes;
        // places a block: fewer, in more blocks, lengthen the sums over blocks that each makes.  Whole gradients, us, 1024 / 512 / 256: 30011 of 50021 x 64 bf16 28.6 / 29.6 / 35.8, x 1537 fp32 110 / 111 / 117, 16384 of 32768 x 64 bf16
        // 23.4 / 25.2 / 26.5, 65536 of 32000 x 64 31.4 / 35.8 / 36.0
        p.per = (int)std::max<long long>(1024, ((rows + kSortBlocks - 1) / kSortBlocks + 1023) / 1024 * 1024);
        p.sort_blocks = (int)((rows + p.per - 1) / p.per);
    }
    const long long lists = ((rows * 4 + 255) & ~255ll) * (p.passes > 1 ? 4 : 2);
    p.part_at = lists + ((p.sort_blocks * (4ll << p.bits) + 255) & ~255ll);
    p.bytes = p.part_at + p.pieces * 2 * d->c * 4;
    p.bytes = (p.bytes + 255) & ~255ll;
    return p;
}

}  // namespace

extern "C" lc_status embedding_fwd(const lc_embedding_desc* desc, const void* table, const int32_t* tokens, void* out, void* hip_stream) {
    const lc_status st = check_desc(desc);
    if (st != LC_OK || desc->rows == 0) return st;
    if (!table || !tokens || !out) return LC_ERR_NULL;
    if (lc_off_element(table, desc->table_dtype == LC_BF16 ? 2 : 4) || lc_off_element(out, desc->dtype == LC_BF16 ? 2 : 4) || lc_off_element(tokens, 4)) return LC_ERR_ALIGN;
    const int lanes = lanes_of(desc->c);
    const LookupArgs a{table, tokens, out, desc->rows, desc->table_ld ? desc->table_ld : desc->c, desc->vocab, desc->c, __builtin_ctz(lanes), desc->scale};
    const long long blocks = (desc->rows + 256 / lanes - 1) / (256 / lanes);
    const dim3 grid((unsigned)std::min<long long>(blocks <= 1024 ? blocks : (blocks + kRowsAhead - 1) / kRowsAhead, kMostBlocks));
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    lc_begin_call();
    const bool past = (long long)desc->rows * desc->c * (desc->dtype == LC_BF16 ? 2 : 4) >= kPastBytes;
    const auto launch = [&]<typename S, typename T>() {
        by_columns(desc->c, [&]<Columns COLS>() {
            if (past) hipLaunchKernelGGL((embedding_fwd_kernel<S, T, COLS, true>), grid, dim3(256), 0, stream, a);
            else hipLaunchKernelGGL((embedding_fwd_kernel<S, T, COLS, false>), grid, dim3(256), 0, stream, a);
        });
    };
    if (desc->table_dtype == LC_BF16) desc->dtype == LC_BF16 ? launch.template operator()<uint16_t, uint16_t>() : launch.template operator()<uint16_t, float>();
    else desc->dtype == LC_BF16 ? launch.template operator()<float, uint16_t>() : launch.template operator()<float, float>();
    return lc_end_call();
}

extern "C" size_t embedding_bwd_workspace_bytes(const lc_embedding_desc* desc) {
    if (check_desc(desc) != LC_OK || desc->rows == 0) return 0;
    return (size_t)plan_of(desc).bytes;
}

extern "C" lc_status embedding_bwd(const lc_embedding_desc* desc, const int32_t* tokens, const void* dout, float* dtable, int accumulate, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
    const lc_status st = check_desc(desc);
    if (st != LC_OK) return st;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (desc->rows == 0 && accumulate) return LC_OK;
    if (!dtable) return LC_ERR_NULL;
    if (lc_off_element(dtable, 4)) return LC_ERR_ALIGN;
    if (desc->rows == 0) {                   // sums over no rows
        lc_begin_call();
        lc_fill_f32(dtable, 0.f, (size_t)desc->vocab * desc->c, stream);
        return lc_end_call();
    }
    if (!tokens || !dout) return LC_ERR_NULL;
    if (lc_off_element(tokens, 4) || lc_off_element(dout, desc->dtype == LC_BF16 ? 2 : 4)) return LC_ERR_ALIGN;
    const Plan plan = plan_of(desc);
    if (!workspace || (((uintptr_t)workspace) & 255) || workspace_bytes < (size_t)plan.bytes) return LC_ERR_WORKSPACE;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const long long list = (desc->rows * 4 + 255) & ~255ll;
    int* lists[4];
    for (int i = 0; i < 4; ++i) lists[i] = reinterpret_cast<int*>(ws + list * i);
    // the whole table is set to zero by the launches that sort, in equal shares: what tokens then write is written twice, and the rest costs no search for what is absent and hides the launches' latency
    // (32768 rows of 2048, 16384 places: by the sums' launch, absent rows alone, 121 us with the lookup where this took 117)
    const long long launches = std::max(1, 2 * plan.passes), fill = accumulate ? 0 : (long long)desc->vocab * desc->c * 4, share = ((fill + launches - 1) / launches + 15) & ~15ll;
    long long zeroed = 0;
    SortArgs s{tokens, nullptr, nullptr, lists[0], lists[1], nullptr, (int)desc->rows, desc->vocab, plan.per, 0, plan.bits, 0, dtable, 0};
    const auto grid_of = [&](int sort_blocks) {
        s.sort_blocks = sort_blocks;
        s.zeros = dtable + zeroed / 4;
        s.zero_bytes = std::min(share, fill - zeroed);
        zeroed += s.zero_bytes;
        return dim3((unsigned)(sort_blocks + std::min<long long>((s.zero_bytes + 16 * 1024 - 1) / (16 * 1024), kMostBlocks)));
    };
    lc_begin_call();
    int last = 0;                                    // the pair of lists that holds the order
    if (plan.passes == 0) {
        const dim3 grid = grid_of((int)((desc->rows + 63) / 64));
        hipLaunchKernelGGL(embedding_rank_kernel, grid, dim3(1024), 0, stream, s);
    } else {
        s.counts = reinterpret_cast<int*>(ws + list * (plan.passes > 1 ? 4 : 2));
        for (int pass = 0; pass < plan.passes; ++pass) {
            last = pass & 1;
            s.tokens = pass == 0 ? tokens : nullptr;
            s.key_in = lists[last ? 0 : 2];
            s.place_in = lists[last ? 1 : 3];
            s.key = lists[last ? 2 : 0];
            s.place = lists[last ? 3 : 1];
            s.shift = pass * plan.bits;
            dim3 grid = grid_of(plan.sort_blocks);
            hipLaunchKernelGGL(embedding_count_kernel, grid, dim3(1024), 0, stream, s);
            grid = grid_of(plan.sort_blocks);
            hipLaunchKernelGGL(embedding_move_kernel, grid, dim3(1024), 0, stream, s);
        }
    }
    const SumArgs a{lists[last ? 2 : 0], lists[last ? 3 : 1], dout, dtable, reinterpret_cast<float*>(ws + plan.part_at), plan.pieces, (int)desc->rows, desc->vocab, desc->c,
                    __builtin_ctz(plan.lanes), plan.tiles, desc->scale};
    const auto launch = [&]<typename T, Columns COLS, bool ADD>() {
        const auto blocks = [](long long threads) { return dim3((unsigned)((threads + 255) / 256)); };
        if (plan.lanes < 64) hipLaunchKernelGGL((embedding_sum_narrow_kernel<T, COLS, ADD>), blocks(desc->rows * plan.lanes), dim3(256), 0, stream, a);
        else if constexpr (COLS != kUnderEight) hipLaunchKernelGGL((embedding_sum_kernel<T, COLS, ADD, 8>), blocks(plan.pieces * plan.tiles * 64), dim3(256), 0, stream, a);
        if (plan.pieces > 1) hipLaunchKernelGGL((embedding_join_kernel<COLS, ADD>), blocks(plan.pieces * plan.tiles * plan.lanes), dim3(256), 0, stream, a);
    };
    const auto with_type = [&]<typename T>() {
        by_columns(desc->c, [&]<Columns COLS>() { accumulate ? launch.template operator()<T, COLS, true>() : launch.template operator()<T, COLS, false>(); });
    };
    desc->dtype == LC_BF16 ? with_type.template operator()<uint16_t>() : with_type.template operator()<float>();
    return lc_end_call();
}
