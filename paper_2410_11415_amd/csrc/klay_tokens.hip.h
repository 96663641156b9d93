// Log probabilities of given tokens under a row of logits, with the weights of the negated literals, the entropy and the top alternatives,
// and their gradient.  For a row x of V logits:
//   M = max x, d_j = x_j - M, S = sum e^d_j = 1 + R (R: all terms but the maximum's own), ln S = log1p(R)
//   logp_k = d_{t_k} - ln S,  neg_k = ln(1 - p_{t_k}),  H = ln S - sum e^d_j d_j / S
// R is kept apart from the 1 because everything that a sure network answers lives in it: logp of the likely token is -log1p(R) and its
// neg ln R - log1p(R), both as exact, relative to themselves, as the others' exponents are (a few 2^-24 times their distance), where S itself has
// rounded R away.  Below 2^-64 (the others more than 44 under the
// maximum: a very sure network, or finite masks that leave one token) R = e^(M2 - M) R2 is held as M2, the largest of the others, and R2,
// their sum relative to it, since terms below 2^-126 are lost relative to M (2^31 of them are 2^-31 of an R that is not held so).
//
// Bound: memory, one read of the logits; the arithmetic stands close behind (an element of bf16 has 2 bytes, and its exponential takes
// four issue slots of a CU that has about ten per element at the rate of HBM).  A thread runs through its part of the row once with a
// reference `ref` that follows its running maximum from afar: it moves only when a value lies more than kSlack above it, so that almost
// every eight elements cost no rescaling; sums of terms up to e^kSlack lose nothing.  All sums and maxima are fp32.
// Measured with entropy, bf16 (reads alone reach 7.0 TB/s, a copy 6.1): 4096 x 131072 forward 165 us = 6.5 TB/s at 88% of the vector unit's issue
// slots, backward 352 us = 6.1 TB/s; 4096 x 32771 forward 53 us = 5.1 TB/s; 1 x 131072 with eight alternatives 17.7 us, of which one workgroup
// reads for five.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "klay_typed.hip.h"

namespace klay {

constexpr int kTokBlock = 256;              // threads of a workgroup; the kernels over rows also have 64 and 1024 of them
constexpr int kMaxTop = 64, kMaxTokens = 1024;
constexpr int kPartial = 8;                 // floats that a row part leaves for the join
constexpr float kSlack = 8.0f;
constexpr float kTokLog2e = 1.4426950408889634f, kTokLn2 = 0.6931471805599453f, kTokFltMax = 3.402823466e+38f;

// where row r of a tensor with two leading axes starts
struct RowMap {
    int64_t outer, inner_stride;
    int32_t inner;
    __device__ __forceinline__ int64_t at(int64_t r) const {
        const uint32_t q = (uint32_t)r / (uint32_t)inner, m = (uint32_t)r - q * (uint32_t)inner;
        return q * outer + m * inner_stride;
    }
};

// What a backward pass needs of a row.  below < max: a sure row, M2 and R2 in `below` and `sum`; otherwise `below` is +inf and `sum` ln S.
struct RowStats {
    float max, sum, entropy, below;
};

struct TokenArgs {
    const void* logits;
    RowMap logit_rows;
    const int64_t* tokens;
    RowMap token_rows;
    int64_t token_stride;
    int64_t rows;
    int32_t vocab, num_tokens, top;
    int32_t parts, part;                // workgroups per row, elements of each
    float *logp, *neg, *entropy;        // [rows, num_tokens], the same, [rows]; may be null
    RowStats* stats;                    // [rows]
    float* top_logp;                    // [rows, top]
    int64_t* top_tokens;
    float* partial;                     // [rows, parts, kPartial]: RowSums
    uint64_t* lists;                    // [rows, parts, top]
    // backward
    const float *dlogp, *dneg, *dentropy;
    void* dlogits;                      // [rows, vocab]
};

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// An element as one number that orders by value, then by the lowest index (a NaN as the smallest value; -0 as 0).  No two of a row are equal,
// and none is 0, which stands for "no element".
__device__ __forceinline__ uint64_t order_key(float x, uint32_t index) {
    x = x == x ? x + 0.0f : -INFINITY;
    const uint32_t b = __float_as_uint(x);
    return (uint64_t)(b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u)) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b ^ ((b >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return ~(uint32_t)key; }

// ---- what is said about a row once its M, R and T = sum e^d d (base 2: sum e^d d log2 e) are known -----------------
constexpr float kTinyRest = 0x1p-64f;
struct RowSums {
    float max, rest, weighted;
    float below = INFINITY, rest_below = 0.0f;       // of a sure row M2 and R2
    __device__ __forceinline__ bool sure() const { return below < max; }
};
__device__ __forceinline__ bool row_empty(const RowSums& s) { return s.max == -INFINITY && s.rest == 0.0f; }
__device__ __forceinline__ float row_log_sum(const RowSums& s) { return row_empty(s) ? 0.0f : log1pf(s.rest); }
__device__ __forceinline__ float row_entropy(const RowSums& s) {
    return row_empty(s) ? 0.0f : log1pf(s.rest) - kTokLn2 * s.weighted / (1.0f + s.rest);
}
__device__ __forceinline__ float row_log_rest(const RowSums& s) { return s.sure() ? (s.below - s.max) + logf(s.rest_below) : logf(s.rest); }
__device__ __forceinline__ float row_logp(float x, float max, float log_sum) { return max == -INFINITY ? -INFINITY : (x - max) - log_sum; }

// What is asked of a row: token k and its logit, loaded before the row is summed (two loads that wait for each other).
struct Asked {
    int64_t token;
    float x;
};
template <typename T>
__device__ __forceinline__ Asked asked_of(const TokenArgs& g, const T* row, int64_t r, int32_t k) {
    Asked a{-1, 0.0f};
    if (k < g.num_tokens) a.token = g.tokens[g.token_rows.at(r) + k * g.token_stride];
    if (a.token >= 0 && a.token < g.vocab) a.x = (float)row[a.token];
    return a;
}

__device__ __forceinline__ void write_token(const TokenArgs& g, int64_t r, int32_t k, const Asked& a, const RowSums& s, float log_sum) {
    float lp = 0.0f, neg = 0.0f;
    if (a.token >= g.vocab) {
        lp = neg = __int_as_float(0x7fc00000);
    } else if (a.token >= 0) {
        lp = row_logp(a.x, s.max, log_sum) + (log_sum - log_sum);             // (a NaN of the row reaches every token)
        if (g.neg) {
            if (row_empty(s)) neg = 0.0f;
            else if (a.x == s.max && s.rest < 1.0f) neg = row_log_rest(s) - log_sum;
            else neg = log1pf(-expf(lp));
        }
    }
    g.logp[r * g.num_tokens + k] = lp;
    if (g.neg) g.neg[r * g.num_tokens + k] = neg;
}

// Thread `thread` of `threads` writes its tokens; `first` is what asked_of said about its first one.
template <typename T>
__device__ __forceinline__ void write_tokens(const TokenArgs& g, const T* row, int64_t r, int32_t thread, int32_t threads, const Asked& first,
                                             const RowSums& s, float log_sum) {
    for (int32_t k = thread; k < g.num_tokens; k += threads)
        write_token(g, r, k, k == thread ? first : asked_of<T>(g, row, r, k), s, log_sum);
}

__device__ __forceinline__ void write_row(const TokenArgs& g, int64_t r, const RowSums& s, float log_sum) {
    const float h = g.entropy ? row_entropy(s) : 0.0f;
    if (g.entropy) g.entropy[r] = h;
    if (g.stats) g.stats[r] = s.sure() ? RowStats{s.max, s.rest_below, h, s.below} : RowStats{s.max, log_sum, h, INFINITY};
}

__device__ __forceinline__ void write_top(const TokenArgs& g, int64_t r, int32_t k, uint64_t key, float max, float log_sum) {
    g.top_logp[r * g.top + k] = row_logp(key_value(key), max, log_sum) + (log_sum - log_sum);
    g.top_tokens[r * g.top + k] = key_index(key);
}

// ---- sums over the threads of a workgroup -------------------------------------------------------------------------
// A value of another lane by the lane's own instruction (a shuffle through LDS takes some hundred cycles): within four lanes, eight, sixteen,
// then the last lane of one row of sixteen into the next row, and of the first two rows into the others.  Lanes that get none keep `none`.
template <int CONTROL> __device__ __forceinline__ int from_lane(int none, int x) { return __builtin_amdgcn_update_dpp(none, x, CONTROL, 0xf, 0xf, false); }
enum : int { LANES_XOR1 = 0xB1, LANES_XOR2 = 0x4E, LANES_HALF_MIRROR = 0x141, LANES_MIRROR = 0x140, LANES_NEXT_ROW = 0x142, LANES_NEXT_HALF = 0x143 };
template <int CONTROL> __device__ __forceinline__ float with_lane_max(float x) {
    return fmaxf(x, __int_as_float(from_lane<CONTROL>(__float_as_int(x), __float_as_int(x))));
}
template <int CONTROL> __device__ __forceinline__ float with_lane_sum(float x) { return x + __int_as_float(from_lane<CONTROL>(0, __float_as_int(x))); }
template <int CONTROL> __device__ __forceinline__ uint64_t with_lane_max(uint64_t x) {
    const uint64_t y = (uint64_t)(uint32_t)from_lane<CONTROL>(0, (int)(x >> 32)) << 32 | (uint32_t)from_lane<CONTROL>(0, (int)x);
    return y > x ? y : x;
}
// Over the G lanes (16 or 64) of a group; all of them get the result.
template <int G> __device__ __forceinline__ float group_max(float x) {
    x = with_lane_max<LANES_MIRROR>(with_lane_max<LANES_HALF_MIRROR>(with_lane_max<LANES_XOR2>(with_lane_max<LANES_XOR1>(x))));
    if constexpr (G == 16) return x;
    x = with_lane_max<LANES_NEXT_HALF>(with_lane_max<LANES_NEXT_ROW>(x));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
template <int G> __device__ __forceinline__ float group_sum(float x) {
    x = with_lane_sum<LANES_MIRROR>(with_lane_sum<LANES_HALF_MIRROR>(with_lane_sum<LANES_XOR2>(with_lane_sum<LANES_XOR1>(x))));
    if constexpr (G == 16) return x;
    x = with_lane_sum<LANES_NEXT_HALF>(with_lane_sum<LANES_NEXT_ROW>(x));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
template <int G> __device__ __forceinline__ uint64_t group_max(uint64_t x) {
    x = with_lane_max<LANES_MIRROR>(with_lane_max<LANES_HALF_MIRROR>(with_lane_max<LANES_XOR2>(with_lane_max<LANES_XOR1>(x))));
    if constexpr (G == 16) return x;
    x = with_lane_max<LANES_NEXT_HALF>(with_lane_max<LANES_NEXT_ROW>(x));
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
// All threads get the result; `at` is scratch (a float a wave; two) that no earlier call since the last barrier has used.
constexpr int kScratch = 16;
template <int THREADS> __device__ __forceinline__ float block_max(float x, float* at) {
    x = group_max<64>(x);
    if constexpr (THREADS == 64) return x;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
    __syncthreads();
    x = at[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) x = fmaxf(x, at[w]);
    return x;
}
template <int THREADS> __device__ __forceinline__ void block_sum2(float& x, float& y, float* at) {
    x = group_sum<64>(x);
    y = group_sum<64>(y);
    if constexpr (THREADS == 64) return;
    if ((threadIdx.x & 63) == 0) { at[threadIdx.x >> 6] = x; at[kScratch + (threadIdx.x >> 6)] = y; }
    __syncthreads();
    x = at[0];
    y = at[kScratch];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) { x += at[w]; y += at[kScratch + w]; }
}

// One thread's run over its elements.  y = (x - ref) log2 e is one multiply-add, x log2 e - shift with shift = ref log2 e rounded once: what that
// rounding puts into the terms it also puts into `shift`, relative to which the sums are read (term).  WIDE takes the difference first, for rows whose maximum
// is so far from 0 that the product would leave the range of fp32 (a row of nothing but the type's lowest value, for one).
constexpr float kFar = 2e38f;
template <bool ENT, bool TOP, bool WIDE = false>
struct Run {
    float ref = WIDE ? -kTokFltMax : -kFar, shift = -kFar * kTokLog2e, s = 0.0f, t = 0.0f, max = -INFINITY;
    int32_t where = -1;           // first element of the vector that holds the maximum
    __device__ __forceinline__ float term(float x) const { return WIDE ? (x - ref) * kTokLog2e : fmaf(x, kTokLog2e, -shift); }
    template <int N> __device__ __forceinline__ void take(const float (&x)[N], int32_t base) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
        if constexpr (TOP) where = top > max || where < 0 ? base : where;
        max = fmaxf(max, top);
        if (top > ref + kSlack) {
#pragma clang fp contract(off)
            const float to = WIDE ? fmaxf(top, -kTokFltMax) : __builtin_amdgcn_fmed3f(top, -kFar, kFar);
            const float next = to * kTokLog2e;              // rounded by itself: the terms to come are taken relative to it
            const float d = WIDE ? (to - ref) * kTokLog2e : next - shift;
            const float f = exp2_of(-d);
            if constexpr (ENT) t = f > 0.0f ? f * (t - d * s) : 0.0f;
            s *= f;
            ref = to;
            shift = next;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = term(x[i]), e = exp2_of(y);
            s += e;
            if constexpr (ENT) t = fmaf(e, fmaxf(y, -200.0f), t);       // (no term of -inf: 0 times infinity)
        }
    }
};

// How the THREADS threads of a workgroup share the elements [lo, hi) of a row: single ones up to the first multiple of 16 bytes (at `p`, element lo), one
// a thread; vectors of N from `begin` to `full`, thread after thread; single ones behind.  (Vectors from odd addresses on: 4096 x 32771 bf16
// read at 4.5 TB/s instead of 5.5.)
template <int N, int THREADS> struct Share {
    int32_t lo, begin, full, hi, vectors;
    template <typename T> __device__ __forceinline__ Share(const T* p, int32_t from, int32_t to) {
        lo = from;
        hi = to;
        const int32_t head = (int32_t)((0 - reinterpret_cast<uintptr_t>(p)) & 15) / (int32_t)sizeof(T);
        begin = from + (head < to - from ? head : to - from);
        vectors = (to - begin) / N;
        full = begin + vectors * N;
    }
    __device__ __forceinline__ int32_t head() const { return begin - lo; }
    __device__ __forceinline__ int32_t tail() const { return hi - full; }
    __device__ __forceinline__ int32_t at(int32_t i, int32_t thread) const { return begin + (i * THREADS + thread) * N; }
    __device__ __forceinline__ bool in_vector(int32_t j) const { return j >= begin && j < full; }
};

// The key of rank `which` (0: the largest) among those of a wave, of which only zeros are equal.
__device__ __forceinline__ uint64_t of_rank_in_wave(uint64_t key, int32_t which) {
    if (which < 8) {
        for (;; --which) {
            const uint64_t most = group_max<64>(key);
            if (which == 0 || most == 0) return most;
            if (key == most) key = 0;
        }
    }
    const uint32_t lo = (uint32_t)key, hi = (uint32_t)(key >> 32);
    int32_t rank = 0;
#pragma unroll 16
    for (int j = 0; j < 64; ++j) {
        const uint64_t other = (uint64_t)__builtin_amdgcn_readlane(hi, j) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, j);
        rank += other > key;
    }
    return group_max<64>(rank == which ? key : 0);
}

// The first `columns` threads hold the largest key of a column each (or one not above it).  Of the full waves among them the one of
// rank top / waves has as many above it, so the least of these is reached by `top` keys or more: a lower bound of the top-th largest key (0 where there
// are too few columns to tell).  Ends with a barrier behind it.
__device__ __forceinline__ uint64_t bound_of_columns(uint64_t mine, int32_t columns, int32_t top, uint64_t* quota) {
    const int32_t wave = threadIdx.x >> 6;
    const int32_t waves = columns < 128 ? 1 : columns >> 6, each = (top + waves - 1) / waves;
    if (wave < waves) {
        const uint64_t key = of_rank_in_wave(mine, each - 1);
        if ((threadIdx.x & 63) == 0) quota[wave] = key;
    }
    __syncthreads();
    uint64_t limit = quota[0];
    for (int w = 1; w < waves; ++w) limit = quota[w] < limit ? quota[w] : limit;
    return limit;
}

// Keys in LDS, and the best of them.
template <int ROOM, int THREADS> struct Best {
    uint64_t keys[ROOM];
    uint64_t best[kMaxTop];
    uint64_t quota[THREADS / 64];
    uint64_t limit;
    int32_t count;
};
// Of a row part: the candidates of one round on top of those kept before.
template <int THREADS> struct TopShared : Best<THREADS * 8 + 256, THREADS> {
    uint64_t first_quota[THREADS / 64];
    int32_t chosen[THREADS];
    int32_t columns;
};

// Sorts the `top` largest of keys[0 .. count) into best (0 where there are fewer; a key of 0 is none).  `again`: leaves them as the only ones in
// keys, and raises limit to the last of them.
template <int ROOM, int THREADS>
__device__ __forceinline__ void keep_best(Best<ROOM, THREADS>& sh, int32_t top, bool again) {
    const int32_t tid = threadIdx.x;
    int32_t n = sh.count;
    if (n > 128) {            // most of them are out after one look at the columns keys[tid], keys[tid + THREADS], ..
        constexpr int kEach = (ROOM + THREADS - 1) / THREADS;
        const int32_t each = (n + THREADS - 1) / THREADS;
        uint64_t mine[kEach], most = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            mine[j] = 0;
            if (j < each) mine[j] = tid + j * THREADS < n ? sh.keys[tid + j * THREADS] : 0;
            most = mine[j] > most ? mine[j] : most;
        }
        const uint64_t limit = bound_of_columns(most, n < THREADS ? n : THREADS, top, sh.quota);
        if (tid == 0) sh.count = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (mine[j] != 0 && mine[j] >= limit) sh.keys[atomicAdd(&sh.count, 1)] = mine[j];
        __syncthreads();
        n = sh.count;
    }
    for (int32_t i = tid; i < n; i += THREADS) {
        const uint64_t mine = sh.keys[i];
        int32_t rank = 0;
#pragma unroll 4
        for (int32_t j = 0; j < n; ++j) rank += sh.keys[j] > mine;
        if (rank < top && mine != 0) sh.best[rank] = mine;
    }
    if (n + tid < top) sh.best[n + tid] = 0;
    __syncthreads();
    if (!again) return;
    const int32_t kept = n < top ? n : top;
    for (int32_t i = tid; i < kept; i += THREADS) sh.keys[i] = sh.best[i];
    if (tid == 0) {
        sh.count = kept;
        if (n >= top && sh.best[top - 1] > sh.limit) sh.limit = sh.best[top - 1];
    }
    __syncthreads();
}

// The `top` largest elements of [lo, hi).  A thread's own maximum as a key lies between its `low` and its `high`.  Only the columns of threads whose
// `high` reaches the bound that the `low` give hold anything that does: those are read again (from the cache).
// However the logits are ordered, a round adds at most 8 THREADS keys, and more than 256 of them are cut to the best ones before the next.
template <typename T, int N, int THREADS>
__device__ __forceinline__ void top_of_part(TopShared<THREADS>& sh, const T* row, const Share<N, THREADS>& share, uint64_t low, uint64_t high,
                                            int32_t top) {
    const int32_t tid = threadIdx.x;
    if (tid == 0) sh.count = sh.columns = 0;
    const int32_t singles = share.head() > share.tail() ? share.head() : share.tail();
    const int32_t columns_in_use = share.vectors >= THREADS ? THREADS : share.vectors > singles ? share.vectors : singles;
    uint64_t limit = bound_of_columns(low, columns_in_use, top, sh.first_quota);
    if (tid == 0) sh.limit = limit;
    if (high != 0 && high >= limit) sh.chosen[atomicAdd(&sh.columns, 1)] = tid;
    __syncthreads();
    const int32_t columns = sh.columns;
    const int32_t deep = (share.vectors + THREADS - 1) / THREADS, work = columns * deep;
    if (tid < share.head() + share.tail()) {             // the single ones
        const int32_t j = tid < share.head() ? share.lo + tid : share.full + tid - share.head();
        const uint64_t key = order_key((float)row[j], (uint32_t)j);
        if (key >= limit) sh.keys[atomicAdd(&sh.count, 1)] = key;
    }
    for (int32_t w0 = 0; w0 < work; w0 += THREADS) {
        limit = sh.limit;
        const int32_t w = w0 + tid;
        if (w < work) {
            const int32_t i = w / columns, thread = sh.chosen[w - i * columns];
            if (i * THREADS + thread < share.vectors) {
                const int32_t base = share.at(i, thread);
                float x[N];
                load_elements<N>(x, row + base);
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const uint64_t key = order_key(x[q], (uint32_t)(base + q));
                    if (key >= limit) sh.keys[atomicAdd(&sh.count, 1)] = key;
                }
            }
        }
        __syncthreads();
        if (w0 + THREADS >= work) break;
        const bool many = sh.count > 256;
        __syncthreads();
        if (many) keep_best(sh, top, true);
    }
    __syncthreads();
    keep_best(sh, top, false);
}

// f(element, its number) for every element of a thread.
template <typename T, int N, int THREADS, typename F>
__device__ __forceinline__ void each_element(const T* row, const Share<N, THREADS>& share, F&& f) {
    const int32_t tid = threadIdx.x;
    for (int32_t i = 0; i * THREADS + tid < share.vectors; ++i) {
        float x[N];
        load_elements<N>(x, row + share.at(i, tid));
#pragma unroll
        for (int q = 0; q < N; ++q) f(x[q], share.at(i, tid) + q);
    }
    if (tid < share.head()) f((float)row[share.lo + tid], share.lo + tid);
    if (tid < share.tail()) f((float)row[share.full + tid], share.full + tid);
}

// What a workgroup finds out about the elements [lo, hi) of a row.  `tell`: M2 and R2 are of use to somebody.
template <typename T, bool ENT, bool TOP, int THREADS, bool WIDE>
__device__ __forceinline__ RowSums sums_of_part(const T* row, const Share<16 / sizeof(T), THREADS>& share, bool tell, float* scratch, int32_t* owner,
                                                uint64_t* low, uint64_t* high) {
    constexpr int N = 16 / sizeof(T), U = 4;
    const int32_t tid = threadIdx.x, vectors = share.vectors;
    if (tid == 0) *owner = THREADS;
    Run<ENT, TOP, WIDE> run;
    if (tid < share.head()) {
        const float x[1] = {(float)row[share.lo + tid]};
        run.take(x, share.lo + tid);
    }
    int32_t i = 0;
    if (U * THREADS <= vectors) {
        // U vectors a step, the next step's on their way meanwhile
        Raw<T, N> next[U];
#pragma unroll
        for (int u = 0; u < U; ++u) next[u] = stream_raw<N>(row + share.at(u, tid));
        for (;;) {
            Raw<T, N> now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) now[u] = next[u];
            const int32_t at = i;
            i += U;
            const bool more = (i + U) * THREADS <= vectors;
            if (more) {
#pragma unroll
                for (int u = 0; u < U; ++u) next[u] = stream_raw<N>(row + share.at(i + u, tid));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[N];
#pragma unroll
                for (int q = 0; q < N; ++q) x[q] = piece<N, T>(now[u], q);
                run.take(x, share.at(at + u, tid));
            }
            if (!more) break;
        }
    }
    for (; i * THREADS + tid < vectors; ++i) {
        float x[N];
        load_elements<N>(x, row + share.at(i, tid));
        run.take(x, share.at(i, tid));
    }
    if (tid < share.tail()) {
        const float x[1] = {(float)row[share.full + tid]};
        run.take(x, share.full + tid);
    }

    RowSums p;
    p.max = block_max<THREADS>(run.max, scratch);
    const float to = fmaxf(p.max, -kTokFltMax);
    const float d = run.term(to), f = exp2_of(-d);
    float s = run.s, t = 0.0f;
    if (s > 0.0f) {                 // (a thread without terms, or one with a NaN, stays as it is)
        t = ENT && f > 0.0f ? f * (run.t - d * s) : 0.0f;
        s *= f;
    }
    float sum = s;                  // 1 + rest, as far as fp32 tells
    p.weighted = t;
    block_sum2<THREADS>(sum, p.weighted, scratch + kScratch);
    p.rest = sum == 0.0f ? 0.0f : sum - 1.0f;
    if (sum > 0.0f && sum < 1.5f) {
        // One element holds most of the sum: `sum - 1` would keep little of the others.  Its thread's terms are taken again, without it.
        if (run.max == p.max) atomicMin(owner, tid);
        __syncthreads();
        const int32_t who = *owner;
        if (tid == who) s = t = 0.0f;
        const int32_t deep = (vectors - who + THREADS - 1) / THREADS;       // its vectors (none for a thread behind them)
        for (int32_t v = tid; v < deep; v += THREADS) {
            float x[N];
            load_elements<N>(x, row + share.at(v, who));
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float y = (x[q] - to) * kTokLog2e, e = x[q] == p.max ? 0.0f : exp2_of(y);
                s += e;
                t = fmaf(e, fmaxf(y, -200.0f), t);
            }
        }
        if (tid < 2) {              // and its single ones
            const int32_t j = tid == 0 ? share.lo + who : share.full + who;
            if (who < (tid == 0 ? share.head() : share.tail()) && (float)row[j] != p.max) {
                const float y = ((float)row[j] - to) * kTokLog2e, e = exp2_of(y);
                s += e;
                t = fmaf(e, fmaxf(y, -200.0f), t);
            }
        }
        p.rest = s;
        p.weighted = t;
        block_sum2<THREADS>(p.rest, p.weighted, scratch + 3 * kScratch);
        if (tell && p.rest < kTinyRest) {
            float below = -INFINITY, of_below = 0.0f, none = 0.0f;
            each_element(row, share, [&](float x, int32_t) { below = fmaxf(below, x == p.max ? -INFINITY : x); });
            below = block_max<THREADS>(below, scratch + 5 * kScratch);
            if (below > -INFINITY) {
                each_element(row, share, [&](float x, int32_t) { of_below += x == p.max ? 0.0f : exp2_of((x - below) * kTokLog2e); });
                block_sum2<THREADS>(of_below, none, scratch + 6 * kScratch);
                p.below = below;
                p.rest_below = of_below;
            }
        }
    }
    if constexpr (TOP) {
        // the thread's largest element as a key lies between these two (the vector is known, the place in it is not)
        *low = *high = 0;
        if (run.where >= 0) {
            const int32_t last = share.in_vector(run.where) ? run.where + N - 1 : run.where;
            *high = order_key(run.max, (uint32_t)run.where);
            *low = order_key(run.max, (uint32_t)last);
        }
    }
    return p;
}

// A workgroup per row part.  parts == 1: everything is written here; otherwise the part's sums and its best elements, for the join kernel.
template <typename T, bool ENT, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS) token_row_kernel(TokenArgs g) {
    constexpr int N = 16 / sizeof(T);
    __shared__ float scratch[8 * kScratch];
    __shared__ int32_t owner;
    __shared__ std::conditional_t<TOP, TopShared<THREADS>, int> tops;
    const int32_t tid = threadIdx.x;
    const bool tell = g.neg || g.stats;
    for (int64_t unit = blockIdx.x; unit < g.rows * g.parts; unit += gridDim.x) {
        const int64_t r = unit / g.parts;
        const int32_t part = (int32_t)(unit - r * g.parts);
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        const int32_t lo = part * g.part, hi = g.vocab - lo < g.part ? g.vocab : lo + g.part;
        const Share<N, THREADS> share(row + lo, lo, hi);
        Asked asked{-1, 0.0f};
        if (g.parts == 1) asked = asked_of<T>(g, row, r, tid);
        uint64_t low = 0, high = 0;
        RowSums sums = sums_of_part<T, ENT, TOP, THREADS, false>(row, share, tell, scratch, &owner, &low, &high);
        if (fabsf(sums.max) > 0.5f * kFar && fabsf(sums.max) < INFINITY) {
            __syncthreads();
            sums = sums_of_part<T, ENT, TOP, THREADS, true>(row, share, tell, scratch, &owner, &low, &high);
        }
        if constexpr (TOP) top_of_part<T, N, THREADS>(tops, row, share, low, high, g.top);
        if (g.parts == 1) {
            const float log_sum = row_log_sum(sums);
            write_tokens<T>(g, row, r, tid, THREADS, asked, sums, log_sum);
            if (tid == 0) write_row(g, r, sums, log_sum);
            if constexpr (TOP)
                if (tid < g.top) write_top(g, r, tid, tops.best[tid], sums.max, log_sum);
        } else {
            if (tid == 0) *reinterpret_cast<RowSums*>(g.partial + unit * kPartial) = sums;
            if constexpr (TOP)
                if (tid < g.top) g.lists[unit * g.top + tid] = tops.best[tid];
        }
        __syncthreads();            // the scratch is free again
    }
}

constexpr int kMaxParts = 64;
static_assert(sizeof(RowSums) <= kPartial * sizeof(float), "a row part leaves a RowSums");

// Joins the parts of a row.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kTokBlock) token_join_kernel(TokenArgs g) {
    __shared__ float scratch[6 * kScratch];
    __shared__ int32_t owner;
    __shared__ std::conditional_t<TOP, Best<kMaxParts * kMaxTop, kTokBlock>, int> tops;
    const int32_t tid = threadIdx.x, parts = g.parts;
    const int64_t r = blockIdx.x;
    const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
    const Asked asked = asked_of<T>(g, row, r, tid);
    if (tid == 0) owner = kMaxParts;
    if constexpr (TOP) {
        const int32_t all = parts * g.top;
        const uint64_t* lists = g.lists + r * all;
        for (int32_t p = tid; p < all; p += kTokBlock) tops.keys[p] = lists[p];
        if (tid == 0) tops.count = all;
    }
    RowSums mine{-INFINITY, 0.0f, 0.0f};
    if (tid < parts) mine = *reinterpret_cast<const RowSums*>(g.partial + (r * parts + tid) * kPartial);
    const bool none = row_empty(mine);
    const float max = block_max<kTokBlock>(mine.max, scratch);
    if (tid < parts && mine.max == max) atomicMin(&owner, tid);
    __syncthreads();
    // the part that holds the maximum keeps its R; the others bring their own maximum's term along
    const float d = (fmaxf(max, -kTokFltMax) - fmaxf(mine.max, -kTokFltMax)) * kTokLog2e, f = exp2_of(-d), whole = 1.0f + mine.rest;
    float s = mine.rest, t = mine.weighted;
    if (tid != owner && tid < parts) {
        s = none ? 0.0f : f * whole;
        t = !none && f > 0.0f ? f * (mine.weighted - d * whole) : 0.0f;
        if (mine.rest != mine.rest) s = mine.rest;
    }
    block_sum2<kTokBlock>(s, t, scratch + kScratch);
    RowSums sums{max, s, t};
    if ((g.neg || g.stats) && s < kTinyRest && max > -INFINITY) {
        // M2 and R2 likewise: the owner's part brings its own (its R is no larger), the others their maximum and sum
        const float top = tid != owner ? mine.max : mine.sure() ? mine.below : -INFINITY;
        const float below = block_max<kTokBlock>(top, scratch + 3 * kScratch);
        if (below > -INFINITY) {
            float of_below = top > -INFINITY ? exp2_of((top - below) * kTokLog2e) * (tid != owner ? whole : mine.rest_below) : 0.0f, zero = 0.0f;
            block_sum2<kTokBlock>(of_below, zero, scratch + 4 * kScratch);
            sums.below = below;
            sums.rest_below = of_below;
        }
    }
    const float log_sum = row_log_sum(sums);
    write_tokens<T>(g, row, r, tid, kTokBlock, asked, sums, log_sum);
    if (tid == 0) write_row(g, r, sums, log_sum);
    if constexpr (TOP) {
        keep_best(tops, g.top, false);
        if (tid < g.top) write_top(g, r, tid, tops.best[tid], max, log_sum);
    }
}

// ---- short rows: G lanes of a wave per row, E elements per lane, everything in registers ----------------------------
template <typename T, int G, int E, bool ENT, bool TOP>
__global__ void __launch_bounds__(kTokBlock) token_short_kernel(TokenArgs g) {
    const int32_t lane = threadIdx.x % G;
    for (int64_t r = ((int64_t)blockIdx.x * kTokBlock + threadIdx.x) / G; r < g.rows; r += (int64_t)gridDim.x * (kTokBlock / G)) {
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        const Asked asked = asked_of<T>(g, row, r, lane);
        float x[E], max = -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = lane + G * e < g.vocab ? (float)row[lane + G * e] : -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) max = fmaxf(max, x[e]);
        max = group_max<G>(max);
        int32_t first = 1 << 30;
#pragma unroll
        for (int e = E - 1; e >= 0; --e) first = x[e] == max ? lane + G * e : first;
        first = (1 << 30) - (int32_t)group_max<G>((uint64_t)((1 << 30) - first));
        const float to = fmaxf(max, -kTokFltMax);
        float rest = 0.0f, weighted = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float y = (x[e] - to) * kTokLog2e, p = lane + G * e == first ? 0.0f * y : exp2_of(y);    // (0 y: a NaN for +inf)
            rest += p;
            if constexpr (ENT) weighted = fmaf(p, fmaxf(y, -200.0f), weighted);
        }
        if (max == -INFINITY) {          // nothing but -inf (0 * -inf above), or NaN
            rest = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) rest += x[e] != x[e] ? x[e] : 0.0f;
        }
        rest = group_sum<G>(rest);
        if constexpr (ENT) weighted = group_sum<G>(weighted);
        RowSums sums{max, rest, weighted};
        if ((g.neg || g.stats) && rest < kTinyRest && max > -INFINITY) {
            float below = -INFINITY, of_below = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) below = fmaxf(below, lane + G * e == first ? -INFINITY : x[e]);
            below = group_max<G>(below);
#pragma unroll
            for (int e = 0; e < E; ++e) of_below += lane + G * e == first ? 0.0f : exp2_of((x[e] - below) * kTokLog2e);
            of_below = group_sum<G>(of_below);
            if (below > -INFINITY) {
                sums.below = below;
                sums.rest_below = of_below;
            }
        }
        const float log_sum = row_log_sum(sums);
        write_tokens<T>(g, row, r, lane, G, asked, sums, log_sum);
        if (lane == 0) write_row(g, r, sums, log_sum);
        if constexpr (TOP) {
            uint64_t key[E];
#pragma unroll
            for (int e = 0; e < E; ++e) key[e] = lane + G * e < g.vocab ? order_key(x[e], lane + G * e) : 0;
            for (int32_t k = 0; k < g.top; ++k) {
                uint64_t best = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) best = key[e] > best ? key[e] : best;
                best = group_max<G>(best);
#pragma unroll
                for (int e = 0; e < E; ++e) key[e] = key[e] == best ? 0 : key[e];
                if (lane == 0) write_top(g, r, k, best, max, log_sum);
            }
        }
    }
}

// ---- gradient -----------------------------------------------------------------------------------------------------
//   dx_j = sum_{k: t_k != j} p_j (n_k p_k / (1 - p_k) - g_k) + sum_{k: t_k = j} (g_k (1 - p_j) - n_k p_j) - h p_j (ln p_j + H)
// with g, n, h the adjoints of logp, neg, H.  The two sums are kept apart: where p is near 1 n p / (1 - p) is large, and its share for the
// token itself must not be the difference of two large numbers.  In a sure row p_j / (1 - p) for the token of the maximum, the share of
// element j in the others' sum, is q_j = e^(x_j - M2) / R2 (neither p_j nor 1 - p needs to be in fp32's range).
struct BackRow {
    float max, log_sum, entropy, below, rest_below;
    explicit __device__ __forceinline__ BackRow(const RowStats& s)
        : max(s.max), log_sum(s.sum), entropy(s.entropy), below(s.below), rest_below(s.sum) {
        if (sure()) log_sum = expf(below - max) * rest_below;
    }
    __device__ __forceinline__ bool sure() const { return below < max; }
    // nothing but -inf (a row of NaN, or of NaN and -inf, has a log_sum of NaN)
    __device__ __forceinline__ bool empty() const { return max == -INFINITY && log_sum == 0.0f; }
    __device__ __forceinline__ float share(float x) const { return x < max ? exp2_of((x - below) * kTokLog2e) / rest_below : 0.0f; }
};
struct TokenGrad {
    int32_t token;          // < 0: nothing (not asked, out of range, or no adjoint)
    float others, itself;   // n p / (1 - p) - g;  g (1 - p) - n p
};

// `sure` += n p of a sure row's token of the maximum, which goes to the other elements by their shares.
template <typename T>
__device__ __forceinline__ TokenGrad token_grad(const TokenArgs& g, const T* row, int64_t r, int32_t k, const BackRow& s, float& sure) {
    TokenGrad out{-1, 0.0f, 0.0f};
    const int64_t t = g.tokens[g.token_rows.at(r) + k * g.token_stride];
    if (t < 0) return out;
    const float gk = g.dlogp ? g.dlogp[r * g.num_tokens + k] : 0.0f, nk = g.dneg ? g.dneg[r * g.num_tokens + k] : 0.0f;
    if (gk == 0.0f && nk == 0.0f) return out;
    if (t >= g.vocab) {             // its log probability was NaN, and so is the gradient of the row
        out.others = __int_as_float(0x7fc00000);
        return out;
    }
    const float x = (float)row[t], lp = row_logp(x, s.max, s.log_sum) + (s.log_sum - s.log_sum);       // (a NaN of the row reaches every token)
    const float p = expf(lp), away = -expm1f(lp);
    out.token = (int32_t)t;
    float w = nk != 0.0f && away > 0.0f ? nk * p / away : 0.0f;
    if (fabsf(w) > 1e38f) w = copysignf(1e38f, w);      // (an adjoint beyond 2^60: no infinity that meets a p_j of 0)
    if (s.sure() && x == s.max) {
        sure += nk * p;
        w = 0.0f;
    }
    out.others = w - gk;
    out.itself = gk * away - nk * p;
    if (lp != lp) out.others = out.itself = lp;
    return out;
}

// Everything else than the tokens' own entries: p_j (others - h (ln p_j + H)).
struct BulkGrad {
    float max, shift, others, h2, hh;      // shift = ln S log2 e; h2 = -h ln 2, hh = -h H
    bool ent;
    __device__ __forceinline__ float at(float x) const {
        const float y = fmaf(x - max, kTokLog2e, -shift);
        const float p = exp2_of(y);
        return p * (ent ? fmaf(h2, fmaxf(y, -200.0f), others + hh) : others);
    }
    __device__ __forceinline__ float entropy_at(float x) const {       // without `others`
        const float y = fmaf(x - max, kTokLog2e, -shift);
        return ent ? exp2_of(y) * fmaf(h2, fmaxf(y, -200.0f), hh) : 0.0f;
    }
    __device__ __forceinline__ float p(float x) const { return exp2_of(fmaf(x - max, kTokLog2e, -shift)); }
};
__device__ __forceinline__ BulkGrad bulk_grad(const BackRow& s, float others, float h) {
    BulkGrad b;
    b.max = s.max;
    b.shift = s.log_sum * kTokLog2e;
    b.others = others;
    b.h2 = -h * kTokLn2;
    b.hh = -h * s.entropy;
    b.ent = h != 0.0f;
    return b;
}

// A workgroup per row part, as forward.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) token_back_kernel(TokenArgs g) {
    constexpr int N = 16 / sizeof(T), U = 4;
    __shared__ TokenGrad grads[kMaxTokens];
    __shared__ float scratch[4 * kScratch];
    const int32_t tid = threadIdx.x, K = g.num_tokens;
    for (int64_t unit = blockIdx.x; unit < g.rows * g.parts; unit += gridDim.x) {
        const int64_t r = unit / g.parts;
        const int32_t part = (int32_t)(unit - r * g.parts);
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        T* out = static_cast<T*>(g.dlogits) + r * g.vocab;
        const int32_t lo = part * g.part, hi = g.vocab - lo < g.part ? g.vocab : lo + g.part;
        const Share<N, THREADS> share(out + lo, lo, hi);
        // the first vectors come while the adjoints are looked at (of a row without any in vain)
        Raw<T, N> next[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * THREADS + tid < share.vectors) next[u] = stream_raw<N>(row + share.at(u, tid));
        const BackRow s(g.stats[r]);
        float others = 0.0f, asked = 0.0f, sure = 0.0f, none = 0.0f;
        for (int32_t k = tid; k < K; k += THREADS) {
            const TokenGrad t = token_grad<T>(g, row, r, k, s, sure);
            grads[k] = t;
            others += t.others;
            asked += t.token >= 0 || t.others != t.others ? 1.0f : 0.0f;
        }
        block_sum2<THREADS>(others, asked, scratch);
        if (s.sure()) block_sum2<THREADS>(sure, none, scratch + 2 * kScratch);
        const float h = g.dentropy ? g.dentropy[r] : 0.0f;
        // a row that nothing was asked of, or that allows nothing, has no gradient, whatever it holds
        const bool live = !s.empty() && (asked > 0.0f || h != 0.0f);
        const BulkGrad bulk = bulk_grad(s, others, h);
        if (live && sure != 0.0f) {
            for (int32_t i = 0; i * THREADS + tid < share.vectors; ++i) {
                float x[N];
                load_elements<N>(x, row + share.at(i, tid));
#pragma unroll
                for (int q = 0; q < N; ++q) x[q] = bulk.at(x[q]) + sure * s.share(x[q]);
                stream_elements<N>(out + share.at(i, tid), x);
            }
            const int32_t at[2] = {share.lo + tid, share.full + tid};
            if (tid < share.head()) out[at[0]] = (T)(bulk.at((float)row[at[0]]) + sure * s.share((float)row[at[0]]));
            if (tid < share.tail()) out[at[1]] = (T)(bulk.at((float)row[at[1]]) + sure * s.share((float)row[at[1]]));
        } else if (live) {
            for (int32_t i = 0; i * THREADS + tid < share.vectors; i += U) {
                Raw<T, N> now[U];
#pragma unroll
                for (int u = 0; u < U; ++u) now[u] = next[u];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if ((i + U + u) * THREADS + tid < share.vectors) next[u] = stream_raw<N>(row + share.at(i + U + u, tid));
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if ((i + u) * THREADS + tid >= share.vectors) break;
                    float x[N];
#pragma unroll
                    for (int q = 0; q < N; ++q) x[q] = bulk.at(piece<N, T>(now[u], q));
                    stream_elements<N>(out + share.at(i + u, tid), x);
                }
            }
            if (tid < share.head()) out[share.lo + tid] = (T)bulk.at((float)row[share.lo + tid]);
            if (tid < share.tail()) out[share.full + tid] = (T)bulk.at((float)row[share.full + tid]);
        } else {
            const float zeros[N] = {};
            for (int32_t i = 0; i * THREADS + tid < share.vectors; ++i) stream_elements<N>(out + share.at(i, tid), zeros);
            if (tid < share.head()) out[share.lo + tid] = (T)0.0f;
            if (tid < share.tail()) out[share.full + tid] = (T)0.0f;
        }
        __syncthreads();            // the entries of the tokens are written once more
        if (live) {
            for (int32_t k = tid; k < K; k += THREADS) {
                const int32_t j = grads[k].token;
                if (j < lo || j >= hi) continue;
                float itself = 0.0f, rest = 0.0f;
                bool first = true;
                for (int32_t o = 0; o < K; ++o) {
                    const TokenGrad t = grads[o];
                    if (t.token == j) {
                        first = first && o >= k;
                        itself += t.itself;
                    } else {
                        rest += t.others;
                    }
                }
                const float x = (float)row[j];
                if (first)
                    out[j] = (T)(itself + (rest != 0.0f ? rest * bulk.p(x) : 0.0f) + (sure != 0.0f ? sure * s.share(x) : 0.0f) + bulk.entropy_at(x));
            }
        }
        __syncthreads();            // grads and scratch are free again
    }
}

// Short rows, laid out as forward.
template <typename T, int G, int E>
__global__ void __launch_bounds__(kTokBlock) token_back_short_kernel(TokenArgs g) {
    const int32_t lane = threadIdx.x % G;
    for (int64_t r = ((int64_t)blockIdx.x * kTokBlock + threadIdx.x) / G; r < g.rows; r += (int64_t)gridDim.x * (kTokBlock / G)) {
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        T* out = static_cast<T*>(g.dlogits) + r * g.vocab;
        const BackRow s(g.stats[r]);
        const float h = g.dentropy ? g.dentropy[r] : 0.0f;
        const BulkGrad bulk = bulk_grad(s, 0.0f, h);
        float p[E], y[E], asked = 0.0f, sure = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool in = lane + G * e < g.vocab && !s.empty();
            const float x = in ? (float)row[lane + G * e] : -INFINITY;
            p[e] = in ? bulk.p(x) : 0.0f;
            y[e] = in ? bulk.entropy_at(x) : 0.0f;
        }
        for (int32_t k0 = 0; k0 < g.num_tokens; k0 += G) {
            TokenGrad mine{-1, 0.0f, 0.0f};
            if (k0 + lane < g.num_tokens) mine = token_grad<T>(g, row, r, k0 + lane, s, sure);
            const int32_t n = g.num_tokens - k0 < G ? g.num_tokens - k0 : G;
            for (int32_t o = 0; o < n; ++o) {
                const int32_t token = __shfl(mine.token, o, G);
                const float others = __shfl(mine.others, o, G), itself = __shfl(mine.itself, o, G);
                if (token < 0 && others == 0.0f) continue;
                asked = 1.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] += lane + G * e == token ? itself : (others != 0.0f ? others * p[e] : 0.0f);
            }
        }
        if (s.sure()) {
            sure = group_sum<G>(sure);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (sure != 0.0f && lane + G * e < g.vocab) y[e] += sure * s.share((float)row[lane + G * e]);
        }
        const bool live = !s.empty() && (asked > 0.0f || h != 0.0f);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (lane + G * e < g.vocab) out[lane + G * e] = (T)(live ? y[e] : 0.0f);
    }
}

}  // namespace klay
