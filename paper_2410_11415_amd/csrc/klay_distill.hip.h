// Divergence of rows of logits from a teacher's list, and its gradient (the formulas: klay_lists.hip.h).  Bound: memory, one read of the
// logits forward, a read and a write backward.  A thread runs through its vectors of the row once, with a reference that follows its maximum
// from afar, and leaves out the vectors that hold a listed token (a bit each, set before); those few are read again, element by element.
#pragma once

#include "klay_lists.hip.h"

namespace klay {

struct DistillArgs {
    const void* logits;
    RowMap logit_rows;
    ListArgs list;                          // its sorted, slots: where they are kept, or null
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

constexpr int kChunk = 32;                  // vectors of a thread whose bits are held at a time

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) distill_row_kernel(DistillArgs g) {
    constexpr int N = 16 / sizeof(T), U = 4;
    __shared__ int32_t mark[kMaxListed], sorted[kMaxListed], slots[kMaxListed];
    __shared__ float listed[kMaxListed];
    __shared__ uint32_t skip[THREADS];
    __shared__ float scratch[6 * kScratch];
    const int32_t tid = threadIdx.x, K = g.list.num_tokens, vocab = g.list.vocab;
    for (int64_t r = blockIdx.x; r < g.list.rows; r += gridDim.x) {
        const T* row = static_cast<const T*>(g.logits) + g.logit_rows.at(r);
        make_list(g.list, r, true, tid, THREADS, mark, sorted, slots);
        for (int32_t u = tid; u < K; u += THREADS) listed[u] = sorted[u] < kNoToken ? (float)row[sorted[u]] : 0.0f;
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
            skip[tid] = 0;
            __syncthreads();
            for (int32_t u = tid; u < K; u += THREADS) {
                const int32_t j = sorted[u];
                if (j == kNoToken || !share.in_vector(j)) continue;
                const int32_t v = (j - share.begin) / N - c0 * THREADS;
                if (v >= 0 && v < kChunk * THREADS) atomicOr(&skip[v % THREADS], 1u << (v / THREADS));
            }
            __syncthreads();
            const uint32_t out = skip[tid];
            const int32_t left = share.vectors - c0 * THREADS - tid, count = left <= 0 ? 0 : (left + THREADS - 1) / THREADS < kChunk ? (left + THREADS - 1) / THREADS : kChunk;
            Raw<T, N> next[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < count) next[u] = stream_raw<N>(row + share.at(c0 + u, tid));
            for (int32_t i = 0; i < count; i += U) {
                Raw<T, N> now[U];
#pragma unroll
                for (int u = 0; u < U; ++u) now[u] = next[u];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + U + u < count) next[u] = stream_raw<N>(row + share.at(c0 + i + U + u, tid));
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (i + u >= count || (out >> (i + u) & 1u)) continue;
                    float x[N];
#pragma unroll
                    for (int q = 0; q < N; ++q) x[q] = piece<N, T>(now[u], q);
                    run.take(x, g.scale);
                }
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
            for (int q = 0; q < N; ++q) {
                const int32_t e = share.begin + v * N + q;
                if (at < K && sorted[at] == e) { ++at; continue; }
                const float x[1] = {(float)row[e]};
                run.take(x, g.scale);
            }
        }
        Others o;
        o.max = block_max<THREADS>(run.max, scratch);
        const float to = fmaxf(o.max, -kTokFltMax);
        float s = run.s, none = 0.0f;
        if (s > 0.0f) s *= exp2_of((run.ref - to) * g.scale);
        block_sum2<THREADS>(s, none, scratch + kScratch);
        o.sum = s;
        if (tid < 64) finish_distill(g.teach, r, K, sorted, slots, listed, o);
        if (g.list.sorted)
            for (int32_t u = tid; u < K; u += THREADS) g.list.sorted[r * K + u] = sorted[u];
        __syncthreads();                    // shared memory is free again
    }
}

// Rows of at most 512: a wave each, the logits in its registers.
constexpr int kShortDistill = 512;
template <typename T>
__global__ void __launch_bounds__(256) distill_short_kernel(DistillArgs g) {
    constexpr int E = kShortDistill / 64;
    __shared__ int32_t mark[4][kMaxListed], sorted[4][kMaxListed], slots[4][kMaxListed];
    __shared__ float listed[4][kMaxListed];
    __shared__ uint32_t bits[4][kShortDistill / 32];
    const int w = threadIdx.x >> 6;
    const int32_t lane = threadIdx.x & 63, K = g.list.num_tokens;
    const int64_t r = (int64_t)blockIdx.x * 4 + w;
    const bool there = r < g.list.rows;
    const T* row = static_cast<const T*>(g.logits) + (there ? g.logit_rows.at(r) : 0);
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = there && lane + 64 * e < g.list.vocab ? (float)row[lane + 64 * e] : -INFINITY;
    if (lane < kShortDistill / 32) bits[w][lane] = 0;
    make_list(g.list, r, there, lane, 64, mark[w], sorted[w], slots[w]);
    for (int32_t u = lane; u < K; u += 64) {
        const int32_t j = sorted[w][u];
        if (j == kNoToken) continue;
        listed[w][u] = (float)row[j];
        atomicOr(&bits[w][j >> 5], 1u << (j & 31));
    }
    __syncthreads();
    if (!there) return;
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
    if (g.list.sorted)
        for (int32_t u = lane; u < K; u += 64) g.list.sorted[r * K + u] = sorted[w][u];
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
