// Lookup of token embeddings with a scale, and the gradient of their table, for gfx950.
//
// out[i] = scale * table[t_i];  dtable[v] (+)= scale * sum over the places i with t_i = v of dout[i], in a fixed order and without atomics: places are sorted by token (stable), the sorted
// list is cut into pieces of equal length, and a block sums the rows of a piece, whatever tokens they belong to.  A token that lies within a piece is written at once; one that crosses pieces
// leaves a part in each, which the block of its first piece adds up in a second launch.  How often a token occurs does not change how long a block takes.  Bound by memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "token_common.h"

namespace {

constexpr int kNone = 0x7fffffff;                  // the key of a place whose token is outside the table: behind all others

__device__ __forceinline__ int key_of(const int32_t* tokens, long long i, int vocab) {
    const int t = tokens[i];
    return t >= 0 && t < vocab ? t : kNone;
}

// ---------------------------------------------------------------------------------------------- lookup

struct LookupArgs {
    const void* table;
    const int32_t* tokens;
    void* out;
    long long rows, table_ld;
    int vocab, c, lanes;       // lanes: of a row, a power of two up to the block's 256
    float scale;
};

// Some lanes a row (rows dealt round the grid), eight columns a lane and access.
template <typename S, typename T>
__global__ void __launch_bounds__(256) embedding_fwd_kernel(const LookupArgs p) {
    const int lane = threadIdx.x & (p.lanes - 1), each = 256 / p.lanes;
    for (long long row = (long long)blockIdx.x * each + threadIdx.x / p.lanes; row < p.rows; row += (long long)gridDim.x * each) {
        const int key = key_of(p.tokens, row, p.vocab);
        const S* from = static_cast<const S*>(p.table) + (key == kNone ? 0 : key) * p.table_ld;
        T* to = static_cast<T*>(p.out) + row * p.c;
        for (long long col = lane * 8; col < p.c; col += p.lanes * 8) {
            Packed<S> x;
            float v[8];
            lc_load8(x, from, (int)col, p.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = key == kNone ? 0.f : x.get(j) * p.scale;
            lc_store8(to + col, v, p.c - (int)col);
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
};

// Few places: a block ranks 64 of them against all, which it holds in LDS; each of its 16 waves a share of them.
constexpr int kRankMost = 4096;
__global__ void __launch_bounds__(1024) embedding_rank_kernel(const SortArgs p) {
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
        for (int b = 0; b < (int)gridDim.x; ++b) {
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
    long long pieces;
    int rows, vocab, c, len, accumulate;
    int lanes;                 // of a piece; a block has 256 / lanes pieces, or `tiles` blocks have one
    int tiles;
    long long sum_blocks;      // the blocks behind them fill the rows of absent tokens
    float scale;
};

constexpr int kStaged = 2048;      // places of a block's pieces, at most

// Eight columns of a row, loaded (issue) and put in their places (settle) apart, so that loads of several rows are under way; EIGHTS: c is a multiple of 8.
template <bool EIGHTS, bool NT, typename T>
__device__ __forceinline__ void issue(Packed<T>& to, const T* row, int col, int c) {
    if constexpr (EIGHTS) {
        to.template load<NT>(row + col);
    } else if (c >= 8) {
        to.template load<NT>(row + min(col, c - 8));
    } else {
        to.load_some(row, c, 0u);
    }
}
template <bool EIGHTS, typename T>
__device__ __forceinline__ void settle(Packed<T>& x, int col, int c) {
    if constexpr (!EIGHTS) {
        if (c >= 8 && c - col < 8) x.shift(8 - (c - col), 0u);
    }
}
template <bool EIGHTS>
__device__ __forceinline__ void add_to(float* to, float* acc, int left, bool accumulate) {
    if (accumulate) {
        Packed<float> old;
        if (EIGHTS || left >= 8) old.load(to);
        else old.load_some(to, left, 0u);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += old.get(j);
    }
    lc_store8(to, acc, EIGHTS ? 8 : left);
}

template <typename T, bool EIGHTS>
__device__ __forceinline__ void sum_piece(const SumArgs& p) {
    __shared__ int keys[kStaged], places[kStaged];
    const int group = threadIdx.x / p.lanes, lane = threadIdx.x & (p.lanes - 1), each = 256 / p.lanes;
    const long long block = blockIdx.x / p.tiles, start = block * each * p.len;
    const int staged = (int)std::min<long long>((long long)each * p.len, p.rows - start);
    for (int i = threadIdx.x; i < staged; i += 256) {
        keys[i] = p.key[start + i];
        places[i] = p.place[start + i];
    }
    __syncthreads();
    const long long piece = block * each + group;
    const int col = ((int)(blockIdx.x % p.tiles) * p.lanes + lane) * 8;
    if (piece >= p.pieces || col >= p.c) return;
    const int first = group * p.len, end = min(staged, first + p.len);
    const T* const dout = static_cast<const T*>(p.dout);
    constexpr int U = 8;                           // rows under way
    Packed<T> x[U];
    float acc[8] = {};
    int key = keys[first];
    bool continued = start + first > 0 && p.key[start + first - 1] == key;
    const int behind = start + end < p.rows ? p.key[start + end] : kNone;
    const auto leave = [&](bool goes_on) __attribute__((always_inline)) {
        if (key < p.vocab) {
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] *= p.scale;
            if (continued || goes_on) lc_store8(p.part + (piece * 2 + (continued ? 0 : 1)) * p.c + col, acc, p.c - col);
            else add_to<EIGHTS>(p.dtable + (long long)key * p.c + col, acc, p.c - col, p.accumulate);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    };
#pragma unroll
    for (int u = 0; u < U; ++u) issue<EIGHTS, false>(x[u], dout + (long long)places[min(first + u, end - 1)] * p.c, col, p.c);
    for (int i = first; i < end; i += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u < end) {
                const int k = keys[i + u];
                if (k != key) {
                    leave(false);
                    key = k;
                    continued = false;
                }
                settle<EIGHTS>(x[u], col, p.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += x[u].get(j);
            }
            issue<EIGHTS, false>(x[u], dout + (long long)places[min(i + u + U, end - 1)] * p.c, col, p.c);
        }
    }
    leave(behind == key);
}

// Rows of tokens that do not occur: zeros.  A wave takes kFill tokens; each of as many lanes searches for its own.
constexpr int kFill = 16;
__device__ __forceinline__ void fill_absent(const SumArgs& p) {
    const int lane = threadIdx.x & 63;
    const float zero[8] = {};
    for (long long v0 = ((blockIdx.x - p.sum_blocks) * 4 + (threadIdx.x >> 6)) * kFill; v0 < p.vocab; v0 += (gridDim.x - p.sum_blocks) * 4 * kFill) {
        const long long v = v0 + (lane & (kFill - 1));
        int lo = 0, n = p.rows;                    // the first place with a key >= v is among the n + 1 from lo on
        while (n > 0) {
            const int half = n >> 1;
            const bool below = p.key[lo + half] < v;
            lo = below ? lo + half + 1 : lo;
            n = below ? n - half - 1 : half;
        }
        const unsigned there = (unsigned)__ballot(lo < p.rows && p.key[min(lo, p.rows - 1)] == v);
        const int most = (int)std::min<long long>(kFill, p.vocab - v0);
        for (int k = 0; k < most; ++k) {
            if (there >> k & 1) continue;
            float* row = p.dtable + (v0 + k) * p.c;
            for (long long col = lane * 8; col < p.c; col += 512) lc_store8(row + col, zero, p.c - (int)col);
        }
    }
}

template <typename T, bool EIGHTS>
__global__ void __launch_bounds__(256) embedding_sum_kernel(const SumArgs p) {
    if (blockIdx.x < p.sum_blocks) sum_piece<T, EIGHTS>(p);
    else fill_absent(p);
}

// Tokens that cross pieces: the lanes of the piece where one begins add up its parts in the order of the pieces.
template <bool EIGHTS>
__global__ void __launch_bounds__(256) embedding_join_kernel(const SumArgs p) {
    const int lane = threadIdx.x & (p.lanes - 1), each = 256 / p.lanes;
    const long long block = blockIdx.x / p.tiles;
    const long long piece = block * each + threadIdx.x / p.lanes;
    const int col = ((int)(blockIdx.x % p.tiles) * p.lanes + lane) * 8;
    if (piece + 1 >= p.pieces || col >= p.c) return;
    const long long end = (piece + 1) * p.len;
    const int key = p.key[end - 1];
    if (key >= p.vocab || p.key[end] != key) return;
    if (piece > 0 && p.key[piece * p.len - 1] == key) return;                     // it began earlier
    long long lo = piece + 1, n = p.pieces - lo;   // the first piece that does not begin with it
    while (n > 0) {
        const long long half = n >> 1;
        const bool same = p.key[(lo + half) * p.len] == key;
        lo = same ? lo + half + 1 : lo;
        n = same ? n - half - 1 : half;
    }
    constexpr int U = 8;
    float acc[8];
    Packed<float> x[U];
    issue<EIGHTS, false>(x[0], p.part + (piece * 2 + 1) * p.c, col, p.c);
    settle<EIGHTS>(x[0], col, p.c);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = x[0].get(j);
    for (long long next = piece + 1; next < lo; next += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) issue<EIGHTS, false>(x[u], p.part + std::min(next + u, lo - 1) * 2 * p.c, col, p.c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (next + u < lo) {
                settle<EIGHTS>(x[u], col, p.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += x[u].get(j);
            }
        }
    }
    add_to<EIGHTS>(p.dtable + (long long)key * p.c + col, acc, p.c - col, p.accumulate);
}

// ---------------------------------------------------------------------------------------------- host

constexpr long long kMostBlocks = 1 << 20;
constexpr long long kMostRows = 1ll << 30;

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

int lanes_of(int c) {                              // the smallest power of two from 8 on that takes a row at once, a block's threads at most
    int lanes = 8;
    while (lanes < 256 && lanes * 8 < c) lanes *= 2;
    return lanes;
}

// How the gradient is made: places of a piece, pieces, and where things lie in the workspace.
struct Plan {
    int len, lanes, tiles, passes, bits, per, sort_blocks;
    long long pieces, part_at, bytes;
};
Plan plan_of(const lc_embedding_desc* d) {
    Plan p{};
    const long long rows = d->rows;
    p.lanes = lanes_of(d->c);
    p.tiles = (int)(((long long)d->c + p.lanes * 8 - 1) / (p.lanes * 8));
    p.len = (int)std::min<long long>(kStaged * p.lanes / 256, std::min<long long>(256, std::max<long long>(16, rows / 1024)));
    p.pieces = (rows + p.len - 1) / p.len;
    if (rows > kRankMost) {
        int bits = 1;
        while (bits < 31 && (1ll << bits) <= d->vocab) ++bits;                     // keys up to vocab
        p.passes = (bits + kMostBits - 1) / kMostBits;
        p.bits = (bits + p.passes - 1) / p.passes;
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
    const LookupArgs a{table, tokens, out, desc->rows, desc->table_ld ? desc->table_ld : desc->c, desc->vocab, desc->c, lanes, desc->scale};
    const dim3 grid((unsigned)std::min<long long>((desc->rows + 256 / lanes - 1) / (256 / lanes), kMostBlocks));
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    lc_begin_call();
    if (desc->table_dtype == LC_BF16) {
        if (desc->dtype == LC_BF16) hipLaunchKernelGGL((embedding_fwd_kernel<uint16_t, uint16_t>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((embedding_fwd_kernel<uint16_t, float>), grid, dim3(256), 0, stream, a);
    } else {
        if (desc->dtype == LC_BF16) hipLaunchKernelGGL((embedding_fwd_kernel<float, uint16_t>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((embedding_fwd_kernel<float, float>), grid, dim3(256), 0, stream, a);
    }
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
    SortArgs s{tokens, nullptr, nullptr, lists[0], lists[1], nullptr, (int)desc->rows, desc->vocab, plan.per, 0, plan.bits};
    lc_begin_call();
    int last = 0;                                    // the pair of lists that holds the order
    if (plan.passes == 0) {
        hipLaunchKernelGGL(embedding_rank_kernel, dim3((unsigned)((desc->rows + 63) / 64)), dim3(1024), 0, stream, s);
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
            hipLaunchKernelGGL(embedding_count_kernel, dim3((unsigned)plan.sort_blocks), dim3(1024), 0, stream, s);
            hipLaunchKernelGGL(embedding_move_kernel, dim3((unsigned)plan.sort_blocks), dim3(1024), 0, stream, s);
        }
    }
    const int each = 256 / plan.lanes;
    SumArgs a{lists[last ? 2 : 0], lists[last ? 3 : 1], dout, dtable, reinterpret_cast<float*>(ws + plan.part_at), plan.pieces, (int)desc->rows, desc->vocab, desc->c,
              plan.len, accumulate != 0, plan.lanes, plan.tiles, (plan.pieces + each - 1) / each * plan.tiles, desc->scale};
    const long long fill = accumulate ? 0 : std::min<long long>(kMostBlocks, ((long long)desc->vocab + 4 * kFill - 1) / (4 * kFill));
    const dim3 grid((unsigned)(a.sum_blocks + fill));
    const auto launch = [&]<bool EIGHTS>() {
        if (desc->dtype == LC_BF16) hipLaunchKernelGGL((embedding_sum_kernel<uint16_t, EIGHTS>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((embedding_sum_kernel<float, EIGHTS>), grid, dim3(256), 0, stream, a);
        if (plan.pieces > 1) hipLaunchKernelGGL((embedding_join_kernel<EIGHTS>), dim3((unsigned)a.sum_blocks), dim3(256), 0, stream, a);
    };
    desc->c % 8 == 0 ? launch.template operator()<true>() : launch.template operator()<false>();
    return lc_end_call();
}
