// Divergence of rows of logits from a teacher's list, and its gradient (the formulas: klay_lists.hip.h).  Bound: memory, one read of the
// logits forward, a read and a write backward.  A thread runs through its vectors of the row once, with a reference that follows its maximum
// from afar, and leaves out the vectors that hold a listed token (a bit each, set before); those few are read again, element by element.
#pragma once

#include "klay_lists.hip.h"

namespace klay {

struct DistillArgs {
    const void* logits;
    RowMap logit_rows;
    ListArgs list;                          // its sorted, slots: where they are kept
    float* sums;                            // [rows, kRowFloats]: of a row what the run over it leaves
    float scale;                            // log2 e / T
    TeachArgs teach;                        // moved: as sorted
    // backward
    const float* dloss;
    void* dlogits;                          // [rows, vocab]
    int32_t parts, part;                    // workgroups a row, elements of each
};

// A thread's run over its elements: sum of 2^((x - ref) scale).
struct MassRun {
    float ref = -kTokFltMax, s = 0.0f, max = -INFINITY;
    template <int N> __device__ __forceinline__ void take(const float (&x)[N], float scale) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
        max = fmaxf(max, top);
        if ((top - ref) * scale > kSlack) {
            s = s == 0.0f ? 0.0f : s * exp2_of((ref - top) * scale);
            ref = top;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) s += exp2_of((x[i] - ref) * scale);
    }
};

constexpr int kChunk = 64;                  // vectors of a thread whose bits are held at a time

// Few rows: a workgroup of sixteen waves each, whose first one puts the row together (FINISH).  Many: four waves each, which leave a row's sums, and a wave a
// row afterwards, since the 64-bit arithmetic takes twice the registers of the run over the row (4096 x 131072 bf16 in one / in two: 334 / 212 us).
template <typename T, int THREADS, bool FINISH>
__global__ void __launch_bounds__(THREADS, FINISH ? 4 : 6) distill_row_kernel(DistillArgs g) {
    constexpr int N = 16 / sizeof(T), U = 4;
    __shared__ int32_t mark[kMaxListed], sorted[kMaxListed], slots[kMaxListed];
    __shared__ float listed[kMaxListed];
    __shared__ uint64_t skip[THREADS];
    __shared__ float scratch[6 * kScratch];
    const int32_t tid = threadIdx.x, K = g.list.num_tokens, vocab = g.list.vocab;
    for (int64_t r = blockIdx.x; r < g.list.rows; r += gridDim.x) {
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        if (K <= 64) {
            if (tid < 64) {
                bool first;
                const int32_t token = tid < K ? token_of(g.list, r, tid) : kNothing, slot = slot_in_wave(token, K, first);
                if (tid < K) {
                    slots[tid] = slot;
                    sorted[tid] = kNoToken;
                }
                wave_ordered();             // (a lane's token may belong where another lane has just said that there is none)
                if (first) {
                    sorted[slot] = token;
                    listed[slot] = (float)row[token];
                }
            }
            __syncthreads();
        } else {
            make_list(g.list, r, true, tid, THREADS, mark, sorted, slots);
            for (int32_t u = tid; u < K; u += THREADS) listed[u] = sorted[u] < kNoToken ? (float)row[sorted[u]] : 0.0f;
        }
        const Share<N, THREADS> share(row, 0, vocab);
        MassRun run;
        auto single = [&](int32_t j) {
            int32_t lo = 0, hi = K;
            while (lo < hi) {
                const int32_t mid = (lo + hi) >> 1;
                if (sorted[mid] < j) lo = mid + 1;
                else hi = mid;
            }
            if (lo < K && sorted[lo] == j) return;
            const float x[1] = {(float)row[j]};
            run.take(x, g.scale);
        };
        if (tid < share.head()) single(share.lo + tid);
        if (tid < share.tail()) single(share.full + tid);
        for (int32_t c0 = 0; c0 * THREADS < share.vectors; c0 += kChunk) {
            const int32_t left = share.vectors - c0 * THREADS - tid, rounds = left <= 0 ? 0 : (left + THREADS - 1) / THREADS;
            const int32_t count = rounds < kChunk ? rounds : kChunk;
            Raw<T, N> next[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < count) next[u] = stream_raw<N>(row + share.at(c0 + u, tid));
            skip[tid] = 0;
            __syncthreads();
            for (int32_t u = tid; u < K; u += THREADS) {
                const int32_t j = sorted[u];
                if (j == kNoToken || !share.in_vector(j)) continue;
                const int32_t v = (j - share.begin) / N - c0 * THREADS;
                if (v >= 0 && v < kChunk * THREADS)
                    atomicOr(reinterpret_cast<unsigned long long*>(&skip[v % THREADS]), 1ull << (v / THREADS));
            }
            __syncthreads();
            const uint64_t out = skip[tid];
            int32_t i = 0;
            // whole steps of U vectors, the next step's on their way meanwhile
            for (; i + U <= count; i += U) {
                Raw<T, N> now[U];
#pragma unroll
                for (int u = 0; u < U; ++u) now[u] = next[u];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + U + u < count) next[u] = stream_raw<N>(row + share.at(c0 + i + U + u, tid));
                const uint32_t skipped = (uint32_t)(out >> i) & ((1u << U) - 1u);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float x[N];
#pragma unroll
                    for (int q = 0; q < N; ++q) x[q] = piece<N, T>(now[u], q);
                    if (!(skipped >> u & 1u)) run.take(x, g.scale);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u >= count || (out >> (i + u) & 1ull)) continue;
                float x[N];
#pragma unroll
                for (int q = 0; q < N; ++q) x[q] = piece<N, T>(next[u], q);
                run.take(x, g.scale);
            }
            __syncthreads();                // the bits are read
        }
        // the vectors left out, by the thread of the first of their listed tokens
        for (int32_t u = tid; u < K; u += THREADS) {
            const int32_t j = sorted[u];
            if (j == kNoToken || !share.in_vector(j)) continue;
            const int32_t v = (j - share.begin) / N;
            if (u > 0 && share.in_vector(sorted[u - 1]) && (sorted[u - 1] - share.begin) / N == v) continue;
            int32_t at = u;
            float x[N];
            load_elements<N>(x, row + share.begin + v * N);
#pragma unroll
            for (int q = 0; q < N; ++q) {
                if (at < K && sorted[at] == share.begin + v * N + q) { ++at; continue; }
                const float one[1] = {x[q]};
                run.take(one, g.scale);
            }
        }
        Others o;
        o.max = block_max<THREADS>(run.max, scratch);
        const float to = fmaxf(o.max, -kTokFltMax);
        float s = run.s, none = 0.0f;
        if (s > 0.0f) s *= exp2_of((run.ref - to) * g.scale);
        block_sum2<THREADS>(s, none, scratch + kScratch);
        o.sum = s;
        if constexpr (FINISH) {
            if (tid < 64) finish_distill(g.teach, r, K, sorted, slots, listed, o);
        } else {
            if (tid == 0) {
                g.sums[r * kRowFloats] = o.max;
                g.sums[r * kRowFloats + 1] = s;
            }
            for (int32_t u = tid; u < K; u += THREADS) {
                g.list.slots[r * K + u] = slots[u];
                g.teach.moved[r * K + u] = listed[u];
            }
        }
        for (int32_t u = tid; u < K; u += THREADS) g.list.sorted[r * K + u] = sorted[u];
        __syncthreads();                    // shared memory is free again
    }
}
__global__ void __launch_bounds__(256) distill_finish_kernel(DistillArgs g) {
    for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < g.list.rows; r += (int64_t)gridDim.x * 4) {
        const int64_t at = r * g.list.num_tokens;
        Others o;
        o.max = g.sums[r * kRowFloats];
        o.sum = g.sums[r * kRowFloats + 1];
        finish_distill(g.teach, r, g.list.num_tokens, g.list.sorted + at, g.list.slots + at, g.teach.moved + at, o);
    }
}

// Rows of at most 512: a wave each, the logits in its registers; lists of at most LISTED.
constexpr int kShortDistill = 512;
template <typename T, int LISTED>
__global__ void __launch_bounds__(256) distill_short_kernel(DistillArgs g) {
    constexpr int E = kShortDistill / 64;
    __shared__ int32_t mark[4][LISTED], sorted[4][LISTED], slots[4][LISTED];
    __shared__ float listed[4][LISTED];
    __shared__ uint32_t bits[4][kShortDistill / 32];
    const int w = threadIdx.x >> 6;
    const int32_t lane = threadIdx.x & 63, K = g.list.num_tokens;
    for (int64_t first_row = (int64_t)blockIdx.x * 4; first_row < g.list.rows; first_row += (int64_t)gridDim.x * 4) {
        const int64_t r = first_row + w;
        const bool there = r < g.list.rows;
        const T* row = static_cast<const T*>(g.logits) + (there ? g.logit_rows.at(r) : 0);
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = there && lane + 64 * e < g.list.vocab ? (float)row[lane + 64 * e] : -INFINITY;
        if (lane < kShortDistill / 32) bits[w][lane] = 0;
        if constexpr (LISTED <= 64) {
            bool first;
            const int32_t token = there && lane < K ? token_of(g.list, r, lane) : kNothing, slot = slot_in_wave(token, K, first);
            if (lane < K) {
                slots[w][lane] = slot;
                sorted[w][lane] = kNoToken;
            }
            __syncthreads();
            if (first) sorted[w][slot] = token;
            __syncthreads();
        } else {
            make_list(g.list, r, there, lane, 64, mark[w], sorted[w], slots[w]);
        }
        for (int32_t u = lane; u < K; u += 64) {
            const int32_t j = sorted[w][u];
            if (j == kNoToken) continue;
            listed[w][u] = (float)row[j];
            atomicOr(&bits[w][j >> 5], 1u << (j & 31));
        }
        __syncthreads();
        if (there) {
            Others o;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int32_t j = lane + 64 * e;
                if (bits[w][j >> 5] >> (j & 31) & 1u) x[e] = -INFINITY;
                o.max = fmaxf(o.max, x[e]);
            }
            o.max = wave_max(o.max);
            const float to = fmaxf(o.max, -kTokFltMax);
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) s += exp2_of((x[e] - to) * g.scale);
            o.sum = group_sum<64>(s);
            finish_distill(g.teach, r, K, sorted[w], slots[w], listed[w], o);
            for (int32_t u = lane; u < K; u += 64) g.list.sorted[r * K + u] = sorted[w][u];
        }
        __syncthreads();                    // shared memory is free again
    }
}

// dx_j = A s_j, then the listed tokens' entries.  A workgroup a row part.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) distill_back_kernel(DistillArgs g) {
    constexpr int N = 16 / sizeof(T), U = 4;
    const int32_t tid = threadIdx.x, K = g.list.num_tokens, vocab = g.list.vocab;
    for (int64_t unit = blockIdx.x; unit < g.list.rows * g.parts; unit += gridDim.x) {
        const int64_t r = unit / g.parts;
        const int32_t part = (int32_t)(unit - r * g.parts);
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        T* out = static_cast<T*>(g.dlogits) + r * vocab;
        const int32_t lo = part * g.part, hi = vocab - lo < g.part ? vocab : lo + g.part;
        const Share<N, THREADS> share(out + lo, lo, hi);
        const TeachStats st = reinterpret_cast<const TeachStats*>(g.teach.stats)[r];
        const float d = g.dloss[r] * (float)g.teach.inverse_temperature;
        const bool live = d != 0.0f && st.live;
        const float A = live ? d * st.others : 0.0f, off = st.ref_log * kTokLog2e;
        auto at = [&](float x) { return A * exp2_of(fmaf(x - st.ref, g.scale, -off)); };
        if (A != 0.0f) {
            Raw<T, N> next[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u * THREADS + tid < share.vectors) next[u] = stream_raw<N>(row + share.at(u, tid));
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
                    for (int q = 0; q < N; ++q) x[q] = at(piece<N, T>(now[u], q));
                    stream_elements<N>(out + share.at(i + u, tid), x);
                }
            }
            if (tid < share.head()) out[share.lo + tid] = (T)at((float)row[share.lo + tid]);
            if (tid < share.tail()) out[share.full + tid] = (T)at((float)row[share.full + tid]);
        } else {
            const float zeros[N] = {};
            for (int32_t i = 0; i * THREADS + tid < share.vectors; ++i) stream_elements<N>(out + share.at(i, tid), zeros);
            if (tid < share.head()) out[share.lo + tid] = (T)0.0f;
            if (tid < share.tail()) out[share.full + tid] = (T)0.0f;
        }
        __syncthreads();                    // the listed tokens' entries are written once more
        if (live)
            for (int32_t u = tid; u < K; u += THREADS) {
                const int32_t j = g.list.sorted[r * K + u];
                if (j >= lo && j < hi) out[j] = (T)(d * g.teach.moved[r * K + u]);
            }
    }
}

}  // namespace klay
