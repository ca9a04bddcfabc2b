// Log probabilities of given tokens over a vocabulary, with entropy and the likeliest alternatives, and the gradient, for gfx950.
//
// Per row of logits z: m = max z, S = sum e^(z-m), T = sum e^(z-m) (z-m); lse = m + log S, log p = z - m - log S, entropy = log S - T/S.
// Bound by memory: the logits are read once, 16 bytes a lane at any alignment; 4096 rows of 32768 bf16 take 51 us, 5.2 TB/s (a value's four or five instructions and its
// exponential, at a quarter of their rate, are 30 us by themselves).  A wave takes 1024 values a round into registers, so that a round's maximum is known before its first
// exponential and the running maximum rescales once a round; the waves of a row are one block, whose first joins what the others leave, or, of few long rows, blocks that a second
// launch joins.  Few rows are bound by latency: one row of 131072 with 20 alternatives takes 5.7 us and 4.5 us for the join, of which 2.5 each are a launch.
//
// Alternatives: a value and its place make one 64-bit key (the value's order in the upper half, the complement of its place in the
// lower: equal values by rising place), all different.  A lower bound on the N-th largest of a slice comes from the lanes' own maxima -- N lanes
// have one at least as large -- found by halving over their order with a ballot a step; what reaches it, a few more than N as a
// rule, is gathered in LDS and ranked.  More than LDS has room for (many equal values): the bound is raised by halving over
// the keys themselves, which ends, as no two are equal, and takes many looks (2048 rows of 32000 equal logits with 5 alternatives 5.7 ms instead of 31 us, one of 131072 225 instead of 9).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "token_common.h"

namespace {

constexpr int kMostTop = 32;
constexpr int kMostWaves = 16, kMostListing = 8;      // of a block; with alternatives, for which a wave needs 6.5 KB of LDS
constexpr int kCandidates = 256;            // keys that a wave's LDS has room for
constexpr int kChunks = 128, kRounds = 32;  // places of a lane's values of a round, and rounds, that it has room for
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFar = -150.f;              // 2^-150 is 0 in fp32: distances are no longer than this where 0 * infinity would be formed

typedef unsigned long long Key;

struct TokenArgs {
    const void* z;
    const int32_t* tokens;
    float* logprob;
    float* entropy;          // or null
    float* lse;              // or null
    int32_t* top_tokens;
    float* top_logprobs;
    float4* stats;           // [rows][blocks]: m, S, T (T in units of log 2, as the exponentials' own arguments)
    Key* keys;               // [rows][blocks][top], falling; 0 where a block has fewer
    long long rows, ld;
    int vocab, top, blocks, slice;      // blocks of a row; values of a block, a multiple of 8
};

struct WaveTop {
    Key keys[kCandidates];
    uint16_t marks[kRounds][64];
    uint16_t chunks[kChunks];
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
};

struct Target {              // a row's token and its logit, asked for before the row's sums are known
    bool counts;
    float z;
};
template <typename T>
__device__ __forceinline__ Target target_of(const TokenArgs& p, long long row) {
    const int token = p.tokens[row];
    const bool counts = token >= 0 && token < p.vocab;
    return {counts, counts ? as_float<T>(static_cast<const T*>(p.z)[row * p.ld + token]) : 0.f};
}

// What a row gives but for its alternatives, from its m, S and T; a whole wave with the same values, lane 0 writes.
__device__ __forceinline__ Row finish_row(const TokenArgs& p, long long row, const Target& target, float3 w) {
    const bool empty = w.y == 0.f;
    Row r;
    r.m = w.x == -INFINITY ? 0.f : w.x;
    r.log_s = logf(w.y);
    if ((threadIdx.x & 63) == 0) {
        p.logprob[row] = !target.counts ? 0.f : empty ? -INFINITY : (target.z - r.m) - r.log_s;
        if (p.entropy) p.entropy[row] = empty ? 0.f : r.log_s - kLn2 * (w.z / w.y);
        if (p.lse) p.lse[row] = empty ? -INFINITY : r.m + r.log_s;
    }
    return r;
}

__device__ __forceinline__ void put_alternative(const TokenArgs& p, long long row, int place, Key key, const Row& r) {
    p.top_tokens[row * p.top + place] = key ? (int)~(uint32_t)key : -1;
    p.top_logprobs[row * p.top + place] = key ? (value_of((uint32_t)(key >> 32)) - r.m) - r.log_s : -INFINITY;
}

// Order of a value that at least `need` lanes of the wave reach with theirs, and few more; the least of all values where fewer lanes hold one.
__device__ __forceinline__ uint32_t lanes_bound(uint32_t mine, bool holds, int need) {
    const int holders = __popcll(__ballot(holds));
    if (holders < need) return 0x00800000u;           // order of the lowest finite float
    uint32_t lo = ~lc_wave_umax(holds ? ~mine : 0u), hi = lc_wave_umax(holds ? mine : 0u) + 1;      // every holder reaches lo, none hi
    for (int n = holders; n > need + need / 4 && hi - lo > 1;) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        const int c = __popcll(__ballot(holds && mine >= mid));
        if (c >= need) {
            lo = mid;
            n = c;
        } else {
            hi = mid;
        }
    }
    return lo;
}

// Appends the keys of the lanes that have one to `keys` (a wave's own); returns the new count, which may pass kCandidates.
__device__ __forceinline__ int append(Key* keys, int held, bool has, Key key) {
    const unsigned long long mask = __ballot(has);
    const int at = held + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
    if (has && at < kCandidates) keys[at] = key;
    return held + __popcll(mask);
}

// Ranks `count` different keys of a wave in LDS; emit(place, key) for the first `top` places, key 0 where there are fewer.
template <typename F>
__device__ __forceinline__ void rank_keys(const Key* keys, int count, int top, F&& emit) {
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < count; base += 64) {
        const Key mine = base + lane < count ? keys[base + lane] : 0;
        int place = 0;
#pragma unroll 8
        for (int j = 0; j < count; ++j) place += keys[j] > mine;
        if (base + lane < count && place < top) emit(place, mine);
    }
    for (int i = count + lane; i < top; i += 64) emit(i, (Key)0);
}

// (m, S, T) of n parts, by a wave.
__device__ __forceinline__ float3 join_sums(const float4* stats, int n) {
    const int lane = threadIdx.x & 63;
    const float4 own = lane < n ? stats[lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    float m = own.x;
    for (int i = lane + 64; i < n; i += 64) m = fmaxf(m, stats[i].x);
    m = lc_wave_max(m);
    float s = 0.f, t = 0.f;
    for (int i = lane; i < n; i += 64) {
        const float4 a = i == lane ? own : stats[i];
        const float shift = a.x == -INFINITY ? 0.f : (a.x - m) * kLog2e;      // (a part without a value keeps its sums: 0, or NaN)
        const float f = __builtin_amdgcn_exp2f(shift);
        s = fmaf(f, a.y, s);
        t = fmaf(f, fmaf(fmaxf(shift, kFar), a.y, a.z), t);
    }
    return make_float3(m, lc_wave_sum(s), lc_wave_sum(t));
}

// The `top` largest keys of n falling lists of `top`, by a wave; `keys`: kCandidates in LDS.  A lane answers for k keys no smaller than its own: the k-th of
// its list, or the first of the largest of its lists; then every list is walked from its head while its keys reach the bound that follows.  Where there are more keys than room, k is such that half of the
// lists answer for `top` of them: were it nearly all (25 lists, 20 keys), the bound would be their least, and more keys than there is room for would reach it (64 rows of 50021 27 us, so 14).
template <typename F>
__device__ __forceinline__ void join_lists(const Key* lists, int n, int top, Key* keys, F&& emit) {
    constexpr int kHead = 8;                        // keys of a lane that are asked for at once: of its list, or half of them of each of two lists
    const int lane = threadIdx.x & 63, lanes = min(n, 64), k = ((n * top > kCandidates ? 2 * top : top) + lanes - 1) / lanes, each = n > 64 ? kHead / 2 : kHead;
    Key head[kHead], own = 0;
#pragma unroll
    for (int j = 0; j < kHead; ++j) {
        const int list = j < each ? lane : lane + 64, at = j < each ? j : j - each;
        head[j] = list < n && at < top ? lists[(long long)list * top + at] : 0;
    }
    if (k > 1) {
        if (lane < n) own = lists[(long long)lane * top + k - 1];
    } else {
        own = each < kHead ? max(head[0], head[kHead / 2]) : head[0];
        for (int i = lane + 128; i < n; i += 64) own = max(own, lists[(long long)i * top]);
    }
    Key least = max((Key)lanes_bound((uint32_t)(own >> 32), own != 0, (top + k - 1) / k) << 32, (Key)1);
    int held = 0;
    const auto walk = [&](const Key* list, bool there, int j) __attribute__((always_inline)) {
        for (; j < top; ++j) {
            const Key key = there ? list[j] : 0;
            if (!__ballot(key >= least)) break;
            held = append(keys, held, key >= least, key);
        }
    };
    const auto gather = [&]() __attribute__((always_inline)) {
        held = 0;
        bool more = true;
#pragma unroll
        for (int j = 0; j < kHead; ++j) {
            if (j == kHead / 2 && each < kHead) {
                if (more) walk(lists + (long long)lane * top, lane < n, each);
                more = true;
            }
            if (more) more = __ballot(head[j] >= least) != 0;
            if (more) held = append(keys, held, head[j] >= least, head[j]);
        }
        const int last = each < kHead ? 64 : 0;
        if (more) walk(lists + (long long)(last + lane) * top, last + lane < n, each);
        for (int base = 128; base < n; base += 64) walk(lists + (long long)(base + lane) * top, base + lane < n, 0);
    };
    gather();
    if (held > kCandidates) {
        const long long all = (long long)n * top;
        Key hi = ~(Key)0;                           // fewer than `top` keys reach hi, more than there is room for reach least
        while (hi - least > 1) {
            const Key mid = least + ((hi - least) >> 1);
            int c = 0;
            for (long long base = 0; base < all; base += 64) c += __popcll(__ballot(base + lane < all && lists[base + lane] >= mid));
            if (c >= top) least = mid;
            else hi = mid;
            if (c >= top && c <= kCandidates) break;
        }
        gather();
    }
    __builtin_amdgcn_wave_barrier();
    rank_keys(keys, min(held, kCandidates), top, emit);
}

// The sums by one wave of columns [first, first + SPAN) of each `stride` up to `end`, of a row of c, from memory and from the distances themselves: where its maximum is further from
// zero than products with log2 e carry (see LaneSums).  KNOWN: m is the maximum already.
template <int SPAN, bool KNOWN, typename T>
__device__ __forceinline__ float3 sums_by_distances(const T* z, int c, int first, int stride, int end, float m = -INFINITY) {
    constexpr uint32_t kMaskedBits = sizeof(T) == 2 ? 0xff80u : 0xff800000u;
    const int lane = threadIdx.x & 63;
    const auto over = [&](auto&& f) __attribute__((always_inline)) {
        for (int start = first; start < end; start += stride)
            for (int at = start; at < start + SPAN; at += 512) {
                const auto column = [&](int) { return at + lane * 8; };
                Packed<T> v[1];
                lc_issue8(v, z, column, c, at + 512 <= end, kMaskedBits);
                lc_settle8(v, column, c, end, at + 512 <= end, kMaskedBits);
#pragma unroll
                for (int j = 0; j < 8; ++j) f(v[0].get(j));
            }
    };
    if constexpr (!KNOWN) {
        over([&](float x) { m = fmaxf(m, x); });
        m = lc_wave_max(m);
    }
    const float from = m == -INFINITY ? 0.f : m;
    float s = 0.f, t = 0.f;
    over([&](float x) {
        const float d = (x - from) * kLog2e, e = __builtin_amdgcn_exp2f(d);
        s += e;
        t = fmaf(e, fmaxf(d, kFar), t);
    });
    return make_float3(m, lc_wave_sum(s), lc_wave_sum(t));
}
constexpr float kProductsFloor = -0x1p31f;       // from here to 2^31 rounding a product to 24 bits takes 64 at most
constexpr float kProductsEnd = 1.48e9f;          // largest magnitude whose product with log2 e stays within that

// Larger of three, a NaN ignored: without the instruction that the compiler puts before fmaxf() for each operand from memory, against signalling NaN
// (one of those may cost a lane its maximum here; its row is NaN either way).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// What a lane has summed: S and T = sum e d over e = 2^d, d = z log2 e - ref, with ref the product m log2 e as rounded for the largest m so far.  One fused
// multiply-add a value, exact to its rounding because ref is.  What rounding takes from the product shifts every d alike, to be put right at the wave's end: by 64 at most within 2^31 of
// zero, where 2^64 for each of 2^30 values and its product with d are in range, and by hundreds beyond (a mask of -1e10 in all of a lane's values: 2^440).  So ref is -2^31 at
// least: what lies further down adds 0 beside any maximum that does not, and a wave whose maximum lies beyond that on either side sums its part again, now that it knows the
// maximum.  A masked value makes T 0 * infinity: the sum is then made again with the distance bounded (NaN and infinity among the logits come out NaN either way).
template <bool ENT>
struct LaneSums {
    float m = -INFINITY, ref = kProductsFloor, s = 0.f, t = 0.f;      // (t only with ENT)

    // Returns the largest of the values (at least `floor`).
    template <int N>
    __device__ __forceinline__ float add(const float (&v)[N], float floor) {
        static_assert(N % 2 == 0, "in pairs");
        float most = floor;
#pragma unroll
        for (int j = 0; j < N; j += 2) most = max3(v[j], v[j + 1], most);
        m = fmaxf(m, most);
        const float now = fmaxf(ref, most * kLog2e), less = -now;
        const float shift = fmaxf(ref + less, kFar), f = __builtin_amdgcn_exp2f(ref + less);
        if (ENT) t = f * fmaf(shift, s, t);
        s *= f;
        ref = now;
        float ds = 0.f, dt = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float d = fmaf(v[j], kLog2e, less), e = __builtin_amdgcn_exp2f(d);
            ds += e;
            if (ENT) dt = fmaf(e, d, dt);
        }
        if (ENT && __ballot(dt != dt)) {
            dt = 0.f;
            float again = less;
            asm("" : "+v"(again));                 // (the first sum's terms are not kept in registers for this one)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float d = fmaf(v[j], kLog2e, again);
                dt = fmaf(__builtin_amdgcn_exp2f(d), fmaxf(d, kFar), dt);
            }
        }
        s += ds;
        t += dt;
        return most;
    }

    // The wave's m, S and T about m itself; z to end: its part of the row, for sums_by_distances().
    template <int SPAN, typename T>
    __device__ __forceinline__ float3 join(const T* z, int c, int first, int stride, int end) const {
        const float all = lc_wave_max(m), less = -fmaxf(all * kLog2e, kProductsFloor);
        if (fabsf(all) > kProductsEnd && fabsf(all) < INFINITY) return sums_by_distances<SPAN, true>(z, c, first, stride, end, all);
        const float shift = fmaxf(ref + less, kFar), f = __builtin_amdgcn_exp2f(ref + less);      // (a lane whose sums are NaN keeps them so)
        const float ws = lc_wave_sum(f * s), wt = lc_wave_sum(f * fmaf(shift, s, t));
        // every exponent is off by what rounding the product took
        const float off = all == -INFINITY ? 0.f : fmaf(all, kLog2e, less), back = __builtin_amdgcn_exp2f(-off);
        return make_float3(all, ws * back, fmaf(-off, ws, wt) * back);
    }
};

// What a block of the forward pass has joined goes to the results, or, of a row in several blocks, to the workspace.
template <bool TOP>
__device__ __forceinline__ void leave(const TokenArgs& p, long long row, const Target& target, float3 w, const Key* lists, int n, Key* keys, bool ranked) {
    const long long unit = row * p.blocks + blockIdx.x;
    const int lane = threadIdx.x & 63;
    Row r;
    if (p.blocks == 1) r = finish_row(p, row, target, w);
    else if (lane == 0) p.stats[unit] = make_float4(w.x, w.y, w.z, 0.f);
    if constexpr (TOP) {
        const auto emit = [&](int place, Key k) {
            if (p.blocks == 1) put_alternative(p, row, place, k, r);
            else p.keys[unit * p.top + place] = k;
        };
        if (ranked) join_lists(lists, n, p.top, keys, emit);
        else rank_keys(keys, n, p.top, emit);
    }
}

// A slice of a row by a block of one wave or several, whose first joins what the others leave in LDS.  Rounds of 512 * CH values go to the waves in turn, so that a
// block reads one stretch at a time; a wave's next round is under way while one is summed.  ENT: with the entropy.  TOP: with the alternatives: a lane marks in LDS how
// large the largest of its values of each round is (the upper half of its order); of those that may reach the bound, a few more than N as a rule, one each a
// lane reads the values again.  LDS: WaveTop a wave and its list of `top`.
template <typename T, int CH, bool ENT, bool TOP>
__global__ void __launch_bounds__((TOP ? kMostListing : kMostWaves) * 64, TOP && sizeof(T) * CH == 8 ? 3 : 4) token_sums_kernel(const TokenArgs p) {
    __shared__ float4 stats[kMostWaves];
    extern __shared__ __align__(16) char lds[];
    constexpr uint32_t kMaskedBits = sizeof(T) == 2 ? 0xff80u : 0xff800000u;
    constexpr int kRound = 512 * CH;
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = (int)blockIdx.x * p.slice, end = min(p.vocab - part, p.slice) + part;
    const int first = min(part + wave * kRound, end), stride = waves * kRound;
    WaveTop* top = TOP ? reinterpret_cast<WaveTop*>(lds) + wave : nullptr;
    Key* keys = TOP ? top->keys : nullptr;
    Key* lists = TOP ? reinterpret_cast<Key*>(reinterpret_cast<WaveTop*>(lds) + waves) : nullptr;
    for (long long row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const T* z = static_cast<const T*>(p.z) + row * p.ld;
        Target target;
        if (wave == 0 && p.blocks == 1) target = target_of<T>(p, row);
        LaneSums<ENT> sums;
        Packed<T> now[CH], next[CH];
        const auto column = [&](int at) __attribute__((always_inline)) { return [at, lane](int i) { return at + (i * 64 + lane) * 8; }; };
        const auto issue = [&](Packed<T>(&to)[CH], int at) __attribute__((always_inline)) {
            if (at < end) lc_issue8(to, z, column(at), p.vocab, at + kRound <= end, kMaskedBits);
        };
        const auto settle = [&](Packed<T>(&of)[CH], int at) __attribute__((always_inline)) {
            lc_settle8(of, column(at), p.vocab, end, at + kRound <= end, kMaskedBits);
        };
        const bool single = first + stride >= end;              // one round, or none
        int round = 0;
        const auto add = [&](Packed<T>(&from)[CH], int at) __attribute__((always_inline)) {
            settle(from, at);
            float v[CH * 8];
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[8 * i + j] = from[i].get(j);
            if (TOP && !single) top->marks[round++][lane] = (uint16_t)(order_of(sums.add(v, -INFINITY)) >> 16);
            else sums.add(v, sums.m);
        };
        issue(now, first);
        for (int at = first; at < end; at += 2 * stride) {
            issue(next, at + stride);
            add(now, at);
            issue(now, at + 2 * stride);
            if (at + stride < end) add(next, at + stride);
        }
        const float3 w = sums.template join<kRound>(z, p.vocab, first, stride, end);
        int held = 0;
        if constexpr (TOP) {
            const uint32_t order = lanes_bound(order_of(sums.m), listable(sums.m), p.top);
            const float bound = value_of(order);
            const auto look = [&](bool there, auto&& column_of) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float x = now[i].get(j);
                        const bool is = there && x >= bound;
                        if (__ballot(is)) held = append(keys, held, is, key_of(x, column_of(i) + j));
                    }
            };
            if (single) {                                       // (the values are still there)
                if (first < end) look(true, column(first));
            } else {
                int chunks = 0;
                for (int r = 0; r < round; ++r) {
                    const bool may = top->marks[r][lane] >= (uint16_t)(order >> 16);
                    const unsigned long long mask = __ballot(may);
                    if (!mask) continue;
                    const int place = chunks + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
                    if (may && place < kChunks) top->chunks[place] = (uint16_t)(r * 64 + lane);
                    chunks += __popcll(mask);
                }
                __builtin_amdgcn_wave_barrier();
                for (int base = 0; base < chunks && chunks <= kChunks; base += 64) {
                    const bool there = base + lane < chunks;
                    const int chunk = there ? top->chunks[base + lane] : 0;
                    const int at = there ? first + (chunk >> 6) * stride : end, of = chunk & 63;
                    const auto where = [&](int i) { return at + (i * 64 + of) * 8; };
                    lc_issue8(now, z, where, p.vocab, false, kMaskedBits);
                    lc_settle8(now, where, p.vocab, there ? end : 0, false, kMaskedBits);
                    look(there, where);
                }
                if (chunks > kChunks) held = kCandidates + 1;
            }
            if (held > kCandidates) {
                Key least = (Key)order << 32, hi = ~(Key)0;        // fewer than `top` keys reach hi, more than there is room for reach least
                const auto each = [&](auto&& f) __attribute__((always_inline)) {
                    for (int at = first; at < end; at += stride)
                        for (int i = at + lane; i < at + kRound; i += 64) {
                            const float x = i < end ? as_float(z[i]) : -INFINITY;
                            f(listable(x), key_of(x, i));
                        }
                };
                while (hi - least > 1) {
                    const Key mid = least + ((hi - least) >> 1);
                    int n = 0;
                    each([&](bool is, Key k) { n += __popcll(__ballot(is && k >= mid)); });
                    if (n >= p.top) least = mid;
                    else hi = mid;
                    if (n >= p.top && n <= kCandidates) break;
                }
                held = 0;
                each([&](bool is, Key k) { held = append(keys, held, is && k >= least, k); });
            }
            held = min(held, kCandidates);
            __builtin_amdgcn_wave_barrier();
        }
        if (waves == 1) {
            leave<TOP>(p, row, target, w, nullptr, held, keys, false);
            if (TOP) __syncthreads();
            continue;
        }
        if constexpr (TOP) rank_keys(keys, held, p.top, [&](int place, Key k) { lists[wave * p.top + place] = k; });
        if (lane == 0) stats[wave] = make_float4(w.x, w.y, w.z, 0.f);
        __syncthreads();
        if (wave == 0) leave<TOP>(p, row, target, join_sums(stats, waves), lists, waves, keys, true);
        __syncthreads();
    }
}

// Joins the blocks of a row: a wave a row, which is latency from its first load to its last store (4.5 us for 128 blocks with lists of 20, 3.5 without).
template <typename T>
__global__ void __launch_bounds__(64) token_join_kernel(const TokenArgs p) {
    __shared__ Key keys[kCandidates];
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const Target target = target_of<T>(p, row);
        const Row r = finish_row(p, row, target, join_sums(p.stats + row * p.blocks, p.blocks));
        if (p.top) join_lists(p.keys + row * p.blocks * p.top, p.blocks, p.top, keys, [&](int place, Key k) { put_alternative(p, row, place, k, r); });
        __syncthreads();
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
    long long rows, ld, dld;
    int vocab;
};

// Beyond these magnitudes the rounding of lse (2^-24 of it) shows in p, and products with log2 e may overflow.
template <typename T>
constexpr float kLseEnd = sizeof(T) == 2 ? 16384.f : 256.f;

// Such a row's gradient, by one wave: its sums again, then all of it (dz may be the logits' own buffer: no other wave writes to the row).
template <typename T>
__device__ __forceinline__ void far_row(const TokenBwdArgs& p, long long row) {
    const T* z = static_cast<const T*>(p.z) + row * p.ld;
    T* out = static_cast<T*>(p.dz) + row * p.dld;
    const int token = p.tokens[row];
    const float a = p.dlogprob && token >= 0 && token < p.vocab ? p.dlogprob[row] : 0.f, b = p.dentropy ? p.dentropy[row] : 0.f, ent = p.dentropy ? p.entropy[row] : 0.f;
    const float3 w = sums_by_distances<512, false>(z, p.vocab, 0, 512, p.vocab);
    const float log_s = logf(w.y);
    for (int col = threadIdx.x * 8; col < p.vocab; col += 512) {
        Packed<T> v;
        lc_load8(v, z, col, p.vocab);
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = (v.get(j) - w.x) - log_s;
            o[j] = (col + j == token ? a : 0.f) - __builtin_amdgcn_exp2f(d * kLog2e) * (a + b * (fmaxf(d, kFar) + ent));
        }
        lc_store8(out + col, o, p.vocab - col);
    }
}

// One wave a block, CH times eight columns a lane.  With d = (z - lse) log2 e the result is 2^d (A + B d): a fused multiply-add, an exponential, another multiply-add and
// a product a value, the token's own term apart.  Bound by memory: 4096 rows of 32768 bf16 85 us, 6.3 TB/s of what it must read and write.  The results go past the caches (forward
// and backward together 135 us, with ordinary stores 152); 16 columns a lane (8: 1 % slower there, 3 % at 256 rows, 5 % faster at 1024).  Rows from the last to the first, as the
// memory-side cache would hold those the forward pass has just read, are no better: 3000 rows of 32000 fp32 218 us instead of 205, 2048 of 50000 227 instead of 241.
template <typename T, int CH>
__global__ void __launch_bounds__(64) token_bwd_kernel(const TokenBwdArgs p) {
    const int lane = threadIdx.x, first = blockIdx.x * 512 * CH;
    const auto column = [&](int i) { return first + (i * 64 + lane) * 8; };
    const bool full = first + 512 * CH <= p.vocab;
    const auto is_far = [](float lse) { return fabsf(lse) > kLseEnd<T> && lse != -INFINITY; };
    bool far = false;
    for (long long row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const T* z = static_cast<const T*>(p.z) + row * p.ld;
        T* out = static_cast<T*>(p.dz) + row * p.dld;
        Packed<T> v[CH];
        lc_issue8(v, z, column, p.vocab, full);
        const float lse = p.lse[row], da = p.dlogprob ? p.dlogprob[row] : 0.f, db = p.dentropy ? p.dentropy[row] : 0.f, ent = p.dentropy ? p.entropy[row] : 0.f;
        const int token = p.tokens[row];
        if (is_far(lse)) {
            far = true;
            continue;
        }
        const bool empty = lse == -INFINITY, counts = token >= 0 && token < p.vocab;
        const float a = counts && !empty ? da : 0.f, b = empty ? 0.f : db;
        lc_settle8(v, column, p.vocab, p.vocab, full);
        // (as in the forward pass: every exponent is off by what rounding the product takes, which goes into the factors)
        const float less = -lse * kLog2e, off = fmaf(lse, kLog2e, less), scale = -__builtin_amdgcn_exp2f(-off);
        const float A = scale * (a + b * (ent - off * kLn2)), B = scale * (b * kLn2);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int col = column(i);
            float o[8];
            if (empty) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = 0.f;
            } else if (b != 0.f) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = fmaf(v[i].get(j), kLog2e, less);
                    o[j] = __builtin_amdgcn_exp2f(d) * fmaf(B, fmaxf(d, kFar), A);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = __builtin_amdgcn_exp2f(fmaf(v[i].get(j), kLog2e, less)) * A;
            }
            if (token >= col && token < col + 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += col + j == token ? a : 0.f;
            }
            lc_store8<true>(out + col, o, full ? 8 : p.vocab - col);
        }
    }
    if (far && blockIdx.x == 0)                  // (behind the others: their loop has more registers so, and waits for nothing but what it has asked for at once)
        for (long long row = blockIdx.y; row < p.rows; row += gridDim.y)
            if (is_far(p.lse[row])) far_row<T>(p, row);
}

constexpr int kMostWidth = 1 << 30;
constexpr long long kMostThreads = 1ll << 31;       // of a launch, which has to hold fewer than 2^32

lc_status check_desc(const lc_token_desc* d) {
    if (!d) return LC_ERR_NULL;
    if (d->dtype != LC_F32 && d->dtype != LC_BF16) return LC_ERR_UNSUPPORTED;
    if (d->rows < 0 || d->vocab <= 0 || d->vocab > kMostWidth || (d->ld && d->ld < d->vocab)) return LC_ERR_SHAPE;
    if (d->top < 0 || d->top > kMostTop) return LC_ERR_UNSUPPORTED;
    long long bytes;          // every offset in bytes, the workspace's (at most 272 for 512 logits) among them, fits 63 bits
    if (__builtin_mul_overflow((long long)d->rows, std::max<long long>({d->ld, d->vocab, 512}), &bytes) || __builtin_mul_overflow(bytes, 8ll, &bytes))
        return LC_ERR_SHAPE;
    return LC_OK;
}

struct TokenPlan {
    int chunks, waves, blocks, slice;      // chunks: of 512 values, of a wave's round; waves of a block, blocks of a row, values of a block
    size_t keys, total;
};

constexpr int kResident = 4096;      // waves that the chip holds at a time, 16 a compute unit

// Waves of a row.  As a rule they are one block, which joins them itself: a second launch costs 3 us or more.  Too few leave the chip idle, and with more than it holds at
// once the last of them are too few.  us for bf16 rows by waves a row, or waves of a block x blocks (where both sides are within a tenth the rule takes one for all types and numbers of
// alternatives: 8 waves for 1024 rows of 32000, as longer rows and more of them have; with alternatives blocks from 48 thousand columns on up to 128 rows):
//   without alternatives           16 waves   8 waves   4 waves   1 wave    in blocks of one
//     64 rows of 131072              10.7       12.3        -       57         9.0 (32)
//     96 rows of 131072              11.1        -          -       -         10.4 (42)
//     128 rows of 131072             11.6       12.8        -       57        12.4 (32)
//     112 rows of 200000             16.0        -          -       -         14.5 (36)
//     128 rows of 200000             16.0        -          -       -         16.4 (32)
//     256 rows of 131072             14.4       13.9        -       -         17.7 (32)
//     256 rows of 32000               6.1        6.1       7.2      17         9.3 (8)
//     1024 rows of 32000             18         15.0      14.0      18.5      17.7 (4)
//     4096 rows of 32000             68         51.2      51.6      53.8      53.4 (8)
//     4096 rows of 131072           188.5 (12) 175.6     193       198       189.2 (8)
//     6000 rows of 16000              -         47.5      40.0      47.3      43.6 (4)
//   with 20 alternatives                       8 waves   4 waves   2 waves   1 wave      in blocks of one
//     1 row of 32000                            12.0      12.8       -        22           11.0 (32)
//     64 rows of 131072                         22.5       -         -         -           16.0 (64), 16.5 (32)
//     64 rows of 50000                          16.1      18         -         -           14.4 (25)         (with 5 alternatives 13.0, in blocks 13.8)
//     96 rows of 50000                          16.4       -         -         -           15.9 (17)         (with 5 13.1 and 14.6, fp32 14.7 and 14.0)
//     128 rows of 65536                         17.5       -         -         -           16.7 (16)         (with 5 14.7 and 15.7)
//     128 rows of 98304                         18.6       -         -         -           18.0 (14)
//     160 rows of 131072                        25.1      32.8       -         -           22.2 (16), 26.0 (32)
//     400 rows of 16000                         16.2      12.9      16.1      16.8         17.4 (4)
//     400 rows of 131072                        33.2      37.6       -         -           36.8 (16)
//     700 rows of 131072                        54.3      46.9       -         -           50.5 (4)
//     2048 rows of 32000                        59.2      41.7      36.9      39.9         41.6 (2)
//     3000 rows of 32000                        82.5      59.4      58.3      47.9         61.1 (2)
TokenPlan plan_of(const lc_token_desc* d) {
    TokenPlan p;
    // 16 values a lane of a round; eight of fp32 logits with alternatives where that fills the chip, whose registers then do for four waves a SIMD instead of three (us:
    // 300 rows of 32000 22.7, so 15.5; 1000 37.3, so 31; one row of 128000 10.2, so 11.9)
    const int thousands = (d->vocab + 1023) / 1024;
    const bool eight = d->top && d->dtype == LC_F32 && d->rows * thousands >= kResident;
    p.chunks = d->vocab <= 512 || eight ? 1 : 2;
    const int round = 512 * p.chunks, rounds = (d->vocab + round - 1) / round;
    const int fit = (int)(kResident / std::clamp<long long>(d->rows, 1, kResident));      // waves a row that the chip holds at once
    bool apart;                                        // every wave a block
    int waves;
    if (!d->top) {
        apart = rounds > 96 && d->rows <= 128;
        if (apart) waves = std::min(rounds, fit);
        else waves = d->rows < 256 ? std::min(rounds, kMostWaves) : std::clamp(rounds / 4, 1, 8);
    } else {
        // (a wave's own list takes as long as several rounds; of three, five, six or seven waves fewer fit: 700 rows of 70000 by four 28.7 us, by five 40)
        apart = (thousands >= 32 && d->rows <= 64) || (thousands >= 48 && d->rows <= 128);
        const int kilobytes = thousands * (d->dtype == LC_BF16 ? 2 : 4), least = (rounds + kRounds - 1) / kRounds;
        if (apart) waves = std::max(least, std::min(rounds, fit / 2));
        else waves = kilobytes >= 128 && fit >= 8 ? 8 : kilobytes >= 32 && fit >= 4 ? 4 : kilobytes >= 64 && fit >= 2 ? 2 : 1;
        if (waves < least) waves = std::max(least, 4);
    }
    const int most = apart ? 1 : d->top ? kMostListing : kMostWaves;
    p.blocks = (waves + most - 1) / most;
    p.waves = (waves + p.blocks - 1) / p.blocks;
    const int each = (rounds + p.blocks - 1) / p.blocks;                // rounds of a block
    p.blocks = (rounds + each - 1) / each;
    p.slice = each * round;
    const size_t units = (size_t)d->rows * p.blocks;
    p.keys = p.blocks == 1 ? 0 : (units * sizeof(float4) + 255) & ~(size_t)255;
    p.total = p.blocks == 1 ? 0 : p.keys + ((units * d->top * sizeof(Key) + 255) & ~(size_t)255);
    return p;
}

// A block for every part of every row; as many rows as a grid's second dimension and kMostThreads take, the others dealt round.
dim3 grid_of(int parts, long long rows, int threads) {
    return dim3((unsigned)parts, (unsigned)std::max(1ll, std::min<long long>({rows, 65535, kMostThreads / threads / parts})));
}

template <typename T, int CH>
void launch_fwd(const TokenArgs& a, int waves, hipStream_t stream) {
    const dim3 grid = grid_of(a.blocks, a.rows, waves * 64), block(waves * 64);
    if (a.top) hipLaunchKernelGGL((token_sums_kernel<T, CH, true, true>), grid, block, waves * (sizeof(WaveTop) + a.top * sizeof(Key)), stream, a);
    else if (a.entropy) hipLaunchKernelGGL((token_sums_kernel<T, CH, true, false>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((token_sums_kernel<T, CH, false, false>), grid, block, 0, stream, a);
    if (a.blocks > 1) hipLaunchKernelGGL((token_join_kernel<T>), dim3((unsigned)std::min(a.rows, kMostThreads / 64)), dim3(64), 0, stream, a);
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
    TokenArgs a{logits, tokens, logprob, entropy, lse, top_tokens, top_logprobs, plan.total ? reinterpret_cast<float4*>(base) : nullptr,
                plan.total ? reinterpret_cast<Key*>(base + plan.keys) : nullptr, desc->rows, desc->ld ? desc->ld : desc->vocab, desc->vocab, desc->top,
                plan.blocks, plan.slice};
    lc_begin_call();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (desc->dtype == LC_BF16) plan.chunks == 1 ? launch_fwd<uint16_t, 1>(a, plan.waves, stream) : launch_fwd<uint16_t, 2>(a, plan.waves, stream);
    else plan.chunks == 1 ? launch_fwd<float, 1>(a, plan.waves, stream) : launch_fwd<float, 2>(a, plan.waves, stream);
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
                   dlogits_ld ? dlogits_ld : desc->vocab, desc->vocab};
    const dim3 grid = grid_of((desc->vocab + 1023) / 1024, a.rows, 64);
    lc_begin_call();
    if (desc->dtype == LC_BF16) hipLaunchKernelGGL((token_bwd_kernel<uint16_t, 2>), grid, dim3(64), 0, static_cast<hipStream_t>(hip_stream), a);
    else hipLaunchKernelGGL((token_bwd_kernel<float, 2>), grid, dim3(64), 0, static_cast<hipStream_t>(hip_stream), a);
    return lc_end_call();
}
