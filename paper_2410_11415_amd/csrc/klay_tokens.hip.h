// Log probabilities of given tokens under a row of logits, with the weights of the negated literals, the entropy and the top alternatives,
// and their gradient.  For a row x of V logits:
//   M = max x, d_j = x_j - M, S = sum e^d_j = 1 + R (R: all terms but the maximum's own), ln S = log1p(R)
//   logp_k = d_{t_k} - ln S,  neg_k = ln(1 - p_{t_k}),  H = ln S - sum e^d_j d_j / S
// R is kept apart from the 1 because everything that a sure network answers lives in it: logp of the likely token is -log1p(R) and its
// neg ln R - log1p(R), both to fp32's relative accuracy, where S itself has rounded R away.
//
// Bound: memory, one read of the logits; the arithmetic stands close behind (an element of bf16 has 2 bytes, and its exponential takes
// four issue slots of a CU that has about ten per element at the rate of HBM).  A thread runs through its part of the row once with a
// reference `ref` that follows its running maximum from afar: it moves only when a value lies more than kSlack above it, so that almost
// every eight elements cost no rescaling; sums of terms up to e^kSlack lose nothing.  All sums and maxima are fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "klay_typed.hip.h"

namespace klay {

constexpr int kTokBlock = 256;              // threads per row part
constexpr int kMaxTop = 64, kMaxTokens = 1024;
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

struct RowStats {       // what a backward pass needs of a row
    float max, log_sum, entropy, pad;
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
    float* partial;                     // [rows, parts, 4]: maximum, R, sum e^d d, unused
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
struct RowSums {
    float max, rest, weighted;
};
__device__ __forceinline__ bool row_empty(const RowSums& s) { return s.max == -INFINITY && s.rest == 0.0f; }
__device__ __forceinline__ float row_log_sum(const RowSums& s) { return row_empty(s) ? 0.0f : log1pf(s.rest); }
__device__ __forceinline__ float row_entropy(const RowSums& s) {
    return row_empty(s) ? 0.0f : log1pf(s.rest) - kTokLn2 * s.weighted / (1.0f + s.rest);
}
__device__ __forceinline__ float row_logp(float x, float max, float log_sum) { return max == -INFINITY ? -INFINITY : (x - max) - log_sum; }

template <typename T>
__device__ __forceinline__ void write_token(const TokenArgs& g, const T* row, int64_t r, int32_t k, const RowSums& s, float log_sum) {
    const int64_t t = g.tokens[g.token_rows.at(r) + k * g.token_stride];
    float lp = 0.0f, neg = 0.0f;
    if (t >= g.vocab) {
        lp = neg = __int_as_float(0x7fc00000);
    } else if (t >= 0) {
        const float x = (float)row[t];
        lp = row_logp(x, s.max, log_sum) + (log_sum - log_sum);             // (a NaN of the row reaches every token)
        if (g.neg) {
            if (row_empty(s)) neg = 0.0f;
            else if (x == s.max && s.rest < 1.0f) neg = logf(s.rest) - log_sum;
            else neg = log1pf(-expf(lp));
        }
    }
    g.logp[r * g.num_tokens + k] = lp;
    if (g.neg) g.neg[r * g.num_tokens + k] = neg;
}

__device__ __forceinline__ void write_row(const TokenArgs& g, int64_t r, const RowSums& s, float log_sum) {
    const float h = g.entropy ? row_entropy(s) : 0.0f;
    if (g.entropy) g.entropy[r] = h;
    if (g.stats) g.stats[r] = RowStats{s.max, log_sum, h, 0.0f};
}

__device__ __forceinline__ void write_top(const TokenArgs& g, int64_t r, int32_t k, uint64_t key, float max, float log_sum) {
    g.top_logp[r * g.top + k] = row_logp(key_value(key), max, log_sum) + (log_sum - log_sum);
    g.top_tokens[r * g.top + k] = key_index(key);
}

// ---- sums over the threads of a workgroup -------------------------------------------------------------------------
template <int G> __device__ __forceinline__ float group_max(float x) {
#pragma unroll
    for (int s = G / 2; s > 0; s >>= 1) x = fmaxf(x, __shfl_xor(x, s, 64));
    return x;
}
template <int G> __device__ __forceinline__ float group_sum(float x) {
#pragma unroll
    for (int s = G / 2; s > 0; s >>= 1) x += __shfl_xor(x, s, 64);
    return x;
}
// All threads get the result; `at` is scratch that no earlier call since the last barrier has used.
__device__ __forceinline__ float block_max(float x, float* at) {
    x = group_max<64>(x);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(at[0], at[1]), fmaxf(at[2], at[3]));
}
__device__ __forceinline__ void block_sum2(float& x, float& y, float* at) {
    x = group_sum<64>(x);
    y = group_sum<64>(y);
    if ((threadIdx.x & 63) == 0) { at[threadIdx.x >> 6] = x; at[4 + (threadIdx.x >> 6)] = y; }
    __syncthreads();
    x = (at[0] + at[1]) + (at[2] + at[3]);
    y = (at[4] + at[5]) + (at[6] + at[7]);
}

// One thread's run over its elements.
template <bool ENT, bool TOP>
struct Run {
    float ref = -kTokFltMax, s = 0.0f, t = 0.0f, max = -INFINITY;
    int32_t where = -1;           // first element of the vector that holds the maximum
    template <int N> __device__ __forceinline__ void take(const float (&x)[N], int32_t base) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
        if constexpr (TOP) where = top > max || where < 0 ? base : where;
        max = fmaxf(max, top);
        if (top > ref + kSlack) {
            const float to = fmaxf(top, -kTokFltMax);
            const float d = (to - ref) * kTokLog2e, f = exp2_of(-d);
            if constexpr (ENT) t = f > 0.0f ? f * (t - d * s) : 0.0f;
            s *= f;
            ref = to;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = (x[i] - ref) * kTokLog2e, e = exp2_of(y);
            s += e;
            if constexpr (ENT) t = fmaf(e, fmaxf(y, -200.0f), t);       // (no term of -inf: 0 times infinity)
        }
    }
};

// The N elements of thread `thread`'s vector number i in a part that starts at lo.
template <int N> __device__ __forceinline__ int32_t vector_at(int32_t lo, int32_t i, int32_t thread) { return lo + (i * kTokBlock + thread) * N; }

constexpr int kKeysRoom = kTokBlock * 8 + 256;      // candidates of one round on top of those kept before

struct TopShared {
    uint64_t keys[kKeysRoom];
    uint64_t best[kMaxTop];
    uint64_t column[kTokBlock];
    int32_t chosen[kMaxTop];
    uint64_t limit;
    int32_t count;
};

// Sorts the `top` largest of keys[0 .. count) into best (0 where there are fewer), and leaves them as the only ones in keys.
__device__ __forceinline__ void keep_best(TopShared& sh, int32_t top) {
    const int32_t n = sh.count, tid = threadIdx.x;
    for (int32_t i = tid; i < top; i += kTokBlock) sh.best[i] = 0;
    __syncthreads();
    for (int32_t i = tid; i < n; i += kTokBlock) {
        const uint64_t mine = sh.keys[i];
        int32_t rank = 0;
        for (int32_t j = 0; j < n; ++j) rank += sh.keys[j] > mine;
        if (rank < top) sh.best[rank] = mine;
    }
    __syncthreads();
    const int32_t kept = n < top ? n : top;
    for (int32_t i = tid; i < kept; i += kTokBlock) sh.keys[i] = sh.best[i];
    if (tid == 0) {
        sh.count = kept;
        if (n >= top && sh.best[top - 1] > sh.limit) sh.limit = sh.best[top - 1];
    }
    __syncthreads();
}

// The `top` largest elements of [lo, hi).  The threads' own maxima are given (column); the top-th largest of them is a lower bound
// of what is sought, and only the columns of the threads above it hold anything that reaches it: those are read again (from the
// cache), whatever the order of the logits.
template <typename T, int N>
__device__ __forceinline__ void top_of_part(TopShared& sh, const T* row, int32_t lo, int32_t hi, uint64_t mine, int32_t top) {
    const int32_t tid = threadIdx.x;
    const int32_t vectors = (hi - lo) / N, full = lo + vectors * N;
    sh.column[tid] = mine;
    if (tid == 0) { sh.limit = 0; sh.count = 0; }
    __syncthreads();
    int32_t rank = 0;
    for (int32_t j = 0; j < kTokBlock; ++j) {
        const uint64_t other = sh.column[j];
        rank += other > mine || (other == mine && j < tid);
    }
    if (rank < top) sh.chosen[rank] = tid;
    if (rank == top - 1) sh.limit = mine;
    __syncthreads();
    const int32_t columns = top < kTokBlock ? top : kTokBlock;
    const int32_t deep = (vectors + kTokBlock - 1) / kTokBlock, work = columns * deep;
    for (int32_t w0 = 0; w0 < work + kTokBlock; w0 += kTokBlock) {
        const uint64_t limit = sh.limit;
        const int32_t w = w0 + tid;
        if (w < work) {
            const int32_t i = w / columns, base = vector_at<N>(lo, i, sh.chosen[w - i * columns]);
            if (base < full) {
                float x[N];
                load_elements<N>(x, row + base);
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const uint64_t key = order_key(x[q], (uint32_t)(base + q));
                    if (key >= limit) sh.keys[atomicAdd(&sh.count, 1)] = key;
                }
            }
        } else if (w0 >= work && full + tid < hi) {          // the last round: what is left behind the full vectors
            const uint64_t key = order_key((float)row[full + tid], (uint32_t)(full + tid));
            if (key >= limit) sh.keys[atomicAdd(&sh.count, 1)] = key;
        }
        __syncthreads();
        const bool many = sh.count > 256;
        __syncthreads();
        if (many) keep_best(sh, top);
    }
    keep_best(sh, top);
}

// A workgroup per row part.  parts == 1: everything is written here; otherwise the part's sums and its best elements, for join_kernel.
template <typename T, bool ENT, bool TOP>
__global__ void __launch_bounds__(kTokBlock) token_row_kernel(TokenArgs g) {
    constexpr int N = 16 / sizeof(T), U = 4;
    __shared__ float scratch[32];
    __shared__ int32_t owner;
    __shared__ std::conditional_t<TOP, TopShared, int> tops;
    const int32_t tid = threadIdx.x;
    for (int64_t unit = blockIdx.x; unit < g.rows * g.parts; unit += gridDim.x) {
        const int64_t r = unit / g.parts;
        const int32_t part = (int32_t)(unit - r * g.parts);
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        const int32_t lo = part * g.part, hi = g.vocab - lo < g.part ? g.vocab : lo + g.part;
        const int32_t vectors = (hi - lo) / N, full = lo + vectors * N;
        if (tid == 0) owner = kTokBlock;
        Run<ENT, TOP> run;
        int32_t i = 0;
        for (; (i + U) * kTokBlock <= vectors; i += U) {
            float x[U][N];
#pragma unroll
            for (int u = 0; u < U; ++u) load_elements<N>(x[u], row + vector_at<N>(lo, i + u, tid));
#pragma unroll
            for (int u = 0; u < U; ++u) run.take(x[u], vector_at<N>(lo, i + u, tid));
        }
        for (; i * kTokBlock + tid < vectors; ++i) {
            float x[N];
            load_elements<N>(x, row + vector_at<N>(lo, i, tid));
            run.take(x, vector_at<N>(lo, i, tid));
        }
        if (full + tid < hi) {
            const float x[1] = {(float)row[full + tid]};
            run.take(x, full + tid);
        }

        const float max = block_max(run.max, scratch);
        const float to = fmaxf(max, -kTokFltMax);
        const float d = (to - run.ref) * kTokLog2e, f = exp2_of(-d);
        float s = run.s * f, t = ENT && f > 0.0f ? f * (run.t - d * run.s) : 0.0f;
        if (run.s != run.s) s = run.s;
        float sum = s, weighted = t;
        block_sum2(sum, weighted, scratch + 8);
        float rest = sum - 1.0f;
        if (sum > 0.0f && sum < 1.5f) {
            // One element holds most of the sum: `sum - 1` would keep little of the others.  Its thread's terms are taken again, without it.
            if (run.max == max) atomicMin(&owner, tid);
            __syncthreads();
            const int32_t who = owner;
            if (tid == who) s = t = 0.0f;
            const int32_t deep = (vectors - who + kTokBlock - 1) / kTokBlock;       // its vectors (none for a thread behind them)
            for (int32_t v = tid; v < deep; v += kTokBlock) {
                float x[N];
                load_elements<N>(x, row + vector_at<N>(lo, v, who));
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const float y = (x[q] - to) * kTokLog2e, e = x[q] == max ? 0.0f : exp2_of(y);
                    s += e;
                    t = fmaf(e, fmaxf(y, -200.0f), t);
                }
            }
            if (tid == 0 && full + who < hi && (float)row[full + who] != max) {
                const float y = ((float)row[full + who] - to) * kTokLog2e, e = exp2_of(y);
                s += e;
                t = fmaf(e, fmaxf(y, -200.0f), t);
            }
            rest = s;
            weighted = t;
            block_sum2(rest, weighted, scratch + 16);
        }
        if (sum == 0.0f) rest = 0.0f;
        const RowSums sums{max, rest, weighted};
        if constexpr (TOP) {
            uint64_t mine = 0;
            if (run.where >= 0) {
                const int32_t n = run.where < full ? N : 1;
                for (int32_t q = 0; q < n; ++q) {
                    const uint64_t key = order_key((float)row[run.where + q], (uint32_t)(run.where + q));
                    mine = key > mine ? key : mine;
                }
            }
            top_of_part<T, N>(tops, row, lo, hi, mine, g.top);
        }
        if (g.parts == 1) {
            const float log_sum = row_log_sum(sums);
            for (int32_t k = tid; k < g.num_tokens; k += kTokBlock) write_token<T>(g, row, r, k, sums, log_sum);
            if (tid == 0) write_row(g, r, sums, log_sum);
            if constexpr (TOP)
                if (tid < g.top) write_top(g, r, tid, tops.best[tid], max, log_sum);
        } else {
            if (tid == 0) {
                float* p = g.partial + unit * 4;
                p[0] = max; p[1] = rest; p[2] = weighted;
            }
            if constexpr (TOP)
                if (tid < g.top) g.lists[unit * g.top + tid] = tops.best[tid];
        }
        __syncthreads();            // the scratch is free again
    }
}

constexpr int kMaxParts = 64;

// Joins the parts of a row.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kTokBlock) token_join_kernel(TokenArgs g) {
    __shared__ float scratch[32];
    __shared__ int32_t owner;
    __shared__ uint64_t keys[TOP ? kMaxParts * kMaxTop : 1], best[TOP ? kMaxTop : 1], heads[TOP ? kMaxParts : 1];
    __shared__ uint64_t limit;
    __shared__ int32_t count;
    const int32_t tid = threadIdx.x, parts = g.parts;
    const int64_t r = blockIdx.x;
    const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
    if (tid == 0) { owner = kMaxParts; limit = 0; count = 0; }
    float m = -INFINITY, rest = 0.0f, weighted = 0.0f;
    if (tid < parts) {
        const float* p = g.partial + (r * parts + tid) * 4;
        m = p[0]; rest = p[1]; weighted = p[2];
    }
    const bool none = m == -INFINITY && rest == 0.0f;
    const float max = block_max(m, scratch);
    if (tid < parts && m == max) atomicMin(&owner, tid);
    __syncthreads();
    // the part that holds the maximum keeps its R; the others bring their own maximum's term along
    const float d = (fmaxf(max, -kTokFltMax) - fmaxf(m, -kTokFltMax)) * kTokLog2e, f = exp2_of(-d);
    float s = rest, t = weighted;
    if (tid != owner && tid < parts) {
        const float whole = 1.0f + rest;
        s = none ? 0.0f : f * whole;
        t = !none && f > 0.0f ? f * (weighted - d * whole) : 0.0f;
        if (rest != rest) s = rest;
    }
    block_sum2(s, t, scratch + 8);
    const RowSums sums{max, s, t};
    const float log_sum = row_log_sum(sums);
    for (int32_t k = tid; k < g.num_tokens; k += kTokBlock) write_token<T>(g, row, r, k, sums, log_sum);
    if (tid == 0) write_row(g, r, sums, log_sum);
    if constexpr (TOP) {
        // The lists are sorted.  Of the lists' j-th elements the q-th largest, q j >= top, is a lower bound of what is sought.
        const int32_t top = g.top;
        int32_t j = 1;
        while (j * parts < 2 * top && j < top) j *= 2;
        if (j > top) j = top;
        const int32_t q = (top + j - 1) / j;
        const uint64_t* lists = g.lists + r * parts * top;
        uint64_t head = 0;
        if (tid < parts) {
            head = lists[tid * top + j - 1];
            heads[tid] = head;
        }
        __syncthreads();
        if (tid < parts) {
            int32_t rank = 0;
            for (int32_t p = 0; p < parts; ++p) rank += heads[p] > head || (heads[p] == head && p < tid);
            if (rank == q - 1) limit = head;
        }
        __syncthreads();
        const uint64_t least = limit;
        for (int32_t p = tid; p < parts * top; p += kTokBlock) {
            const uint64_t key = lists[p];
            if (key != 0 && key >= least) keys[atomicAdd(&count, 1)] = key;
        }
        __syncthreads();
        const int32_t n = count;
        for (int32_t p = tid; p < n; p += kTokBlock) {
            const uint64_t mine = keys[p];
            int32_t rank = 0;
            for (int32_t o = 0; o < n; ++o) rank += keys[o] > mine;
            if (rank < top) best[rank] = mine;
        }
        __syncthreads();
        if (tid < top) write_top(g, r, tid, best[tid], max, log_sum);
    }
}

// ---- short rows: G lanes of a wave per row, E elements per lane, everything in registers ----------------------------
template <typename T, int G, int E, bool ENT, bool TOP>
__global__ void __launch_bounds__(kTokBlock) token_short_kernel(TokenArgs g) {
    const int32_t lane = threadIdx.x % G;
    for (int64_t r = ((int64_t)blockIdx.x * kTokBlock + threadIdx.x) / G; r < g.rows; r += (int64_t)gridDim.x * (kTokBlock / G)) {
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        float x[E], max = -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = lane + G * e < g.vocab ? (float)row[lane + G * e] : -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) max = fmaxf(max, x[e]);
        max = group_max<G>(max);
        int32_t first = 1 << 30;
#pragma unroll
        for (int e = E - 1; e >= 0; --e) first = x[e] == max ? lane + G * e : first;
#pragma unroll
        for (int s = G / 2; s > 0; s >>= 1) {
            const int32_t other = __shfl_xor(first, s, 64);
            first = other < first ? other : first;
        }
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
        const RowSums sums{max, rest, weighted};
        const float log_sum = row_log_sum(sums);
        for (int32_t k = lane; k < g.num_tokens; k += G) write_token<T>(g, row, r, k, sums, log_sum);
        if (lane == 0) write_row(g, r, sums, log_sum);
        if constexpr (TOP) {
            uint64_t key[E];
#pragma unroll
            for (int e = 0; e < E; ++e) key[e] = lane + G * e < g.vocab ? order_key(x[e], lane + G * e) : 0;
            for (int32_t k = 0; k < g.top; ++k) {
                uint64_t best = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) best = key[e] > best ? key[e] : best;
#pragma unroll
                for (int s = G / 2; s > 0; s >>= 1) {
                    const uint64_t other = __shfl_xor((unsigned long long)best, s, 64);
                    best = other > best ? other : best;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) key[e] = key[e] == best ? 0 : key[e];
                if (lane == 0) write_top(g, r, k, best, max, log_sum);
            }
        }
    }
}

// ---- gradient -----------------------------------------------------------------------------------------------------
//   dx_j = sum_{k: t_k != j} p_j (n_k p_k / (1 - p_k) - g_k) + sum_{k: t_k = j} (g_k (1 - p_j) - n_k p_j) - h p_j (ln p_j + H)
// with g, n, h the adjoints of logp, neg, H.  The two sums are kept apart: in a sure row n p / (1 - p) is large, and its share for the
// token itself must not be the difference of two large numbers.
struct TokenGrad {
    int32_t token;          // < 0: nothing (not asked, out of range, or no adjoint)
    float others, itself;   // n p / (1 - p) - g;  g (1 - p) - n p
};

template <typename T>
__device__ __forceinline__ TokenGrad token_grad(const TokenArgs& g, const T* row, int64_t r, int32_t k, const RowStats& s) {
    TokenGrad out{-1, 0.0f, 0.0f};
    const int64_t t = g.tokens[g.token_rows.at(r) + k * g.token_stride];
    if (t < 0) return out;
    const float gk = g.dlogp ? g.dlogp[r * g.num_tokens + k] : 0.0f, nk = g.dneg ? g.dneg[r * g.num_tokens + k] : 0.0f;
    if (gk == 0.0f && nk == 0.0f) return out;
    if (t >= g.vocab) {             // its log probability was NaN, and so is the gradient of the row
        out.others = __int_as_float(0x7fc00000);
        return out;
    }
    const float lp = row_logp((float)row[t], s.max, s.log_sum);
    const float p = expf(lp), away = -expm1f(lp);
    out.token = (int32_t)t;
    float w = nk != 0.0f && away > 0.0f ? nk * p / away : 0.0f;
    if (fabsf(w) > 1e38f) w = copysignf(1e38f, w);      // (1 - p at the end of the range: finite, as what it stands for is)
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
__device__ __forceinline__ BulkGrad bulk_grad(const RowStats& s, float others, float h) {
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
template <typename T>
__global__ void __launch_bounds__(kTokBlock) token_back_kernel(TokenArgs g) {
    constexpr int N = 16 / sizeof(T);
    __shared__ TokenGrad grads[kMaxTokens];
    __shared__ float scratch[16];
    const int32_t tid = threadIdx.x, K = g.num_tokens;
    for (int64_t unit = blockIdx.x; unit < g.rows * g.parts; unit += gridDim.x) {
        const int64_t r = unit / g.parts;
        const int32_t part = (int32_t)(unit - r * g.parts);
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        T* out = static_cast<T*>(g.dlogits) + r * g.vocab;
        const int32_t lo = part * g.part, hi = g.vocab - lo < g.part ? g.vocab : lo + g.part;
        const int32_t vectors = (hi - lo) / N, full = lo + vectors * N;
        const RowStats s = g.stats[r];
        float others = 0.0f, asked = 0.0f;
        for (int32_t k = tid; k < K; k += kTokBlock) {
            const TokenGrad t = token_grad<T>(g, row, r, k, s);
            grads[k] = t;
            others += t.others;
            asked += t.token >= 0 || t.others != t.others ? 1.0f : 0.0f;
        }
        block_sum2(others, asked, scratch);
        const float h = g.dentropy ? g.dentropy[r] : 0.0f;
        // a row that nothing was asked of, or that allows nothing, has no gradient, and is not read (it may hold anything)
        const bool live = s.max != -INFINITY && (asked > 0.0f || h != 0.0f);
        const BulkGrad bulk = bulk_grad(s, others, h);
        for (int32_t i = tid; i < vectors; i += kTokBlock) {
            float x[N] = {};
            if (live) {
                load_elements<N>(x, row + lo + i * N);
#pragma unroll
                for (int q = 0; q < N; ++q) x[q] = bulk.at(x[q]);
            }
            store_elements<N>(out + lo + i * N, x);
        }
        if (full + tid < hi) out[full + tid] = (T)(live ? bulk.at((float)row[full + tid]) : 0.0f);
        __syncthreads();            // the entries of the tokens are written once more
        if (live) {
            for (int32_t k = tid; k < K; k += kTokBlock) {
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
                if (first) out[j] = (T)(itself + (rest != 0.0f ? rest * bulk.p(x) : 0.0f) + bulk.entropy_at(x));
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
        const RowStats s = g.stats[r];
        const float h = g.dentropy ? g.dentropy[r] : 0.0f;
        const BulkGrad bulk = bulk_grad(s, 0.0f, h);
        float p[E], y[E], asked = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool in = lane + G * e < g.vocab && s.max != -INFINITY;
            const float x = in ? (float)row[lane + G * e] : -INFINITY;
            p[e] = in ? bulk.p(x) : 0.0f;
            y[e] = in ? bulk.entropy_at(x) : 0.0f;
        }
        for (int32_t k0 = 0; k0 < g.num_tokens; k0 += G) {
            TokenGrad mine{-1, 0.0f, 0.0f};
            if (k0 + lane < g.num_tokens) mine = token_grad<T>(g, row, r, k0 + lane, s);
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
        const bool live = s.max != -INFINITY && (asked > 0.0f || h != 0.0f);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (lane + G * e < g.vocab) out[lane + G * e] = (T)(live ? y[e] : 0.0f);
    }
}

}  // namespace klay
