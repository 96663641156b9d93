// Log probabilities, and divergences from a teacher's list, straight from a network's hidden states: x_ij = h_i . w_j + b_j is made tile by tile in the
// registers of the matrix cores and never written.  Forward, a tile leaves of each row the sums over its tokens that are not listed (klay_lists.hip.h)
// and the logits of those that are; a wave a row joins them.  Backward, the tiles are made again, a piece of the vocabulary at a time, and turned
// into the adjoint of the logits, which in all of these losses has the form
//   G_ij = s_ij (A_i + B_i ln s_ij),  s_ij = e^((x_ij - ref_i) / T - ln S_i),
// with an entry of its own for a listed token; then dH = G W, dW = G^T H, db = sum_i G_i.  G is rounded to the type of the operands (bf16: 2^-8 of an entry,
// independent from entry to entry, as large as the rounding of the result; fp16: under a power of two taken from the largest entry, so that small
// adjoints stay in its range; fp32: the three parts of all operands).  Sums over tokens and rows are in fp32, in an order that the sizes alone decide.
#pragma once

#include "klay_lists.hip.h"
#include "klay_matrix.hip.h"

namespace klay {

// ---- what the C entry points hand to the kernels of a type -----------------------------------------------------------
struct HeadArgs {
    Operand hidden, weight;                 // [rows, width], [tokens of this launch, width]
    const float* bias;                      // of these tokens, or null
    int32_t first, vocab;                   // the first of these tokens; how many tokens there are in all
    int64_t rows;
    int32_t num_tokens;
    const int32_t* sorted;                  // [rows, num_tokens]
    float scale;                            // log2 e / T
    // forward
    float* values;                          // [rows, num_tokens]: the listed tokens' logits
    float4* partial;                        // [rows, tiles of tokens]: max, rest, weighted
    // backward
    const float4* coefs;                    // [rows]: ref (+inf: the row has no gradient), ln S log2 e, A, B ln 2
    const float* entries;                   // [rows, num_tokens]
    const uint32_t* largest;                // bits of the largest adjoint (fp16), or null
    void *g, *g_across;                     // [rows, g_columns], [g_columns, g_rows], their rows so many elements apart
    int64_t g_columns, g_rows, g_stride, g_across_stride;
    float* bias_partial;                    // [tiles of rows, g_columns], or null
};

// One product of a launch: `splits` runs over its stages, each into fp32 sums of its own or, if it is the only one of all pieces, into `out`.
struct ProductJob {
    Operand a, b;
    int32_t splits;
    int64_t rows, columns;
    void* out;                              // [rows, columns], or null
    float* sums;                            // [splits, rows, columns]
    int32_t add;                            // to what is there
};
struct ProductArgs {
    ProductJob job[2];
    int32_t jobs;
    const uint32_t* largest;
};

// fp16: 2^k with which the largest adjoint comes to 2^13 .. 2^14.
__device__ __forceinline__ float adjoint_scale(const uint32_t* largest) {
    if (!largest) return 1.0f;
    const int e = (int)(*largest >> 23) - 127;
    if (*largest == 0u || e > 120) return 1.0f;
    const int k = 13 - e;
    return exp2_of((float)(k > 100 ? 100 : k));
}

// The tokens of a row that fall into a tile: `first` their first place in the row's sorted list, a bit for each column.
template <int BM, int BN> struct Marks {
    static constexpr int kWords = BN / 32;
    uint32_t bits[BM][kWords];
    int32_t first[BM];
    __device__ __forceinline__ void make(const HeadArgs& g, int64_t m0, int32_t token0, int32_t thread, int32_t threads) {
        for (int i = thread; i < BM; i += threads) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) bits[i][w] = 0;
            if (m0 + i >= g.rows) continue;
            const int32_t* list = g.sorted + (m0 + i) * g.num_tokens;
            int32_t lo = 0, hi = g.num_tokens;
            while (lo < hi) {
                const int32_t mid = (lo + hi) >> 1;
                if (list[mid] < token0) lo = mid + 1;
                else hi = mid;
            }
            first[i] = lo;
            for (; lo < g.num_tokens; ++lo) {
                const uint32_t c = (uint32_t)list[lo] - (uint32_t)token0;
                if (c >= (uint32_t)BN) break;
                bits[i][c >> 5] |= 1u << (c & 31);
            }
        }
    }
    __device__ __forceinline__ int32_t place(int row, int word, int bit) const {
        int32_t p = first[row] + __popc(bits[row][word] & ((1u << bit) - 1u));
        for (int w = 0; w < word; ++w) p += __popc(bits[row][w]);
        return p;
    }
};

// Over the 32 lanes of a half; all of them get the result.
__device__ __forceinline__ float other_row(float x) { return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401f)); }     // lane ^ 16
__device__ __forceinline__ float half_max(float x) {
    x = group_max<16>(x);
    return fmaxf(x, other_row(x));
}
__device__ __forceinline__ float half_sum(float x) {
    x = group_sum<16>(x);
    return x + other_row(x);
}

// ---- forward ---------------------------------------------------------------------------------------------------------
template <typename Tile, bool ENT>
__global__ void __launch_bounds__(Tile::kThreads, Tile::kThreads / 256) head_forward_kernel(HeadArgs g, Tiles tiles) {
    constexpr int BM = Tile::kM, BN = Tile::kN, TM = Tile::TM, TN = Tile::TN, WN = Tile::kWavesN;
    // (one object: of several the compiler would wait for all loads into one before every read of it)
    __shared__ struct {
        typename Tile::Shared stage[Tile::kStages];
        Marks<BM, BN> marks;
        float parts[WN][3][BM];
    } sh;
    auto &marks = sh.marks;
    auto &parts = sh.parts;
    int64_t tm, tn;
    tiles.at(blockIdx.x, tm, tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    Tile t;
    if (g.num_tokens) marks.make(g, m0, g.first + (int32_t)n0, threadIdx.x, Tile::kThreads);
    t.run(g.hidden, g.weight, m0, n0, 0, Tile::stages(g.hidden), sh.stage);           // (its barriers are behind the marks, too)
    float bias[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t c = n0 + t.column(j);
        bias[j] = c < g.weight.rows ? (g.bias ? g.bias[c] : 0.0f) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int row = t.row(i) + (e >> 2) * 8 + (e & 3);
            float x[TN], max = -INFINITY;
#pragma unroll
            for (int j = 0; j < TN; ++j) x[j] = bias[j] == -INFINITY ? -INFINITY : t.acc[i][j][e] + bias[j];
            if (g.num_tokens) {
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int word = t.wn * TN + j, bit = t.lane & 31;
                    if (marks.bits[row][word] >> bit & 1u) {
                        g.values[(m0 + row) * g.num_tokens + marks.place(row, word, bit)] = x[j];
                        x[j] = -INFINITY;
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) max = fmaxf(max, x[j]);
            max = half_max(max);
            const float to = fmaxf(max, -kTokFltMax);
            float s = 0.0f, u = 0.0f;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const float y = (x[j] - to) * g.scale, p = exp2_of(y);
                s += p;
                if constexpr (ENT) u = fmaf(p, fmaxf(y, -200.0f), u);
            }
            s = half_sum(s);
            if constexpr (ENT) u = half_sum(u);
            float rest = s == 0.0f ? 0.0f : s - 1.0f;
            if (s > 0.0f && s < 1.5f) {                           // one holds most of the sum: the others by themselves
                rest = 0.0f;
#pragma unroll
                for (int j = 0; j < TN; ++j) rest += x[j] == max ? 0.0f : exp2_of((x[j] - to) * g.scale);
                rest = half_sum(rest);
            }
            if ((t.lane & 31) == 0) {
                parts[t.wn][0][row] = max;
                parts[t.wn][1][row] = rest;
                parts[t.wn][2][row] = u;
            }
        }
    }
    __syncthreads();
    for (int row = threadIdx.x; row < BM; row += Tile::kThreads) {
        if (m0 + row >= g.rows) break;
        float max = parts[0][0][row], rest = parts[0][1][row], u = parts[0][2][row];
#pragma unroll
        for (int w = 1; w < WN; ++w) {
            // the part with the larger maximum keeps its rest; the other brings its maximum's own term along
            const float m = parts[w][0][row], r = parts[w][1][row], v = parts[w][2][row];
            const bool up = m > max;
            const float big = up ? m : max, small = up ? max : m, r_big = up ? r : rest, r_small = up ? rest : r, u_small = up ? u : v;
            const bool none = small == -INFINITY && r_small == 0.0f;
            const float d = (fmaxf(small, -kTokFltMax) - fmaxf(big, -kTokFltMax)) * g.scale, f = none ? 0.0f : exp2_of(d), whole = 1.0f + r_small;
            rest = r_big + (none ? 0.0f : f * whole);
            u = (up ? v : u) + (f > 0.0f ? f * (u_small + d * whole) : 0.0f);
            max = big;
        }
        g.partial[(m0 + row) * tiles.n + tn] = make_float4(max, rest, u, 0.0f);
    }
}

// ---- backward --------------------------------------------------------------------------------------------------------
template <typename Tile>
__global__ void __launch_bounds__(Tile::kThreads, Tile::kThreads / 256) head_adjoint_kernel(HeadArgs g, Tiles tiles) {
    typedef typename Tile::Element T;
    constexpr int BM = Tile::kM, BN = Tile::kN, TM = Tile::TM, TN = Tile::TN, WM = Tile::kWavesM;
    __shared__ struct {
        typename Tile::Shared stage[Tile::kStages];
        Marks<BM, BN> marks;
        float4 coefs[BM];
        float sums[WM][BN];
    } sh;
    auto &marks = sh.marks;
    auto &coefs = sh.coefs;
    auto &sums = sh.sums;
    int64_t tm, tn;
    tiles.at(blockIdx.x, tm, tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    Tile t;
    if (g.num_tokens) marks.make(g, m0, g.first + (int32_t)n0, threadIdx.x, Tile::kThreads);
    for (int row = threadIdx.x; row < BM; row += Tile::kThreads) coefs[row] = m0 + row < g.rows ? g.coefs[m0 + row] : make_float4(INFINITY, 0, 0, 0);
    t.run(g.hidden, g.weight, m0, n0, 0, Tile::stages(g.hidden), sh.stage);
    const float up = adjoint_scale(g.largest);
    float bias[TN], sum[TN] = {};
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t c = n0 + t.column(j);
        bias[j] = c < g.weight.rows ? (g.bias ? g.bias[c] : 0.0f) : -INFINITY;
    }
    T *out = static_cast<T*>(g.g), *across = static_cast<T*>(g.g_across);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float d[TN][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = t.row(i) + 8 * q + e;
                const float4 c = coefs[row];
                const bool live = c.x < INFINITY;
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const float x = bias[j] == -INFINITY ? -INFINITY : t.acc[i][j][4 * q + e] + bias[j];
                    const float y = fmaf(x - c.x, g.scale, -c.y);
                    d[j][e] = live ? exp2_of(y) * fmaf(c.w, fmaxf(y, -200.0f), c.z) : 0.0f;
                    if (n0 + t.column(j) >= g.weight.rows) d[j][e] = 0.0f;
                    if (g.num_tokens) {
                        const int word = t.wn * TN + j, bit = t.lane & 31;
                        if (marks.bits[row][word] >> bit & 1u) d[j][e] = g.entries[(m0 + row) * g.num_tokens + marks.place(row, word, bit)];
                    }
                    sum[j] += d[j][e];
                }
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t c = n0 + t.column(j), r = m0 + t.row(i) + 8 * q;
                if (c >= g.g_columns) continue;
                float scaled[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    scaled[e] = d[j][e] * up;
                    if (out && r + e < g.rows) out[(r + e) * g.g_stride + c] = (T)scaled[e];
                }
                if (across && r < g.g_rows) store_elements<4>(across + c * g.g_across_stride + r, scaled);      // (g_rows is a multiple of 8)
            }
        }
    }
    if (g.bias_partial) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            sum[j] += __shfl_xor(sum[j], 32);
            if (t.lane < 32) sums[t.wm][t.column(j)] = sum[j];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < BN; c += Tile::kThreads) {
            float s = sums[0][c];
#pragma unroll
            for (int w = 1; w < WM; ++w) s += sums[w][c];
            if (n0 + c < g.g_columns) g.bias_partial[tm * g.g_columns + n0 + c] = s;
        }
    }
}

template <typename Tile>
__global__ void __launch_bounds__(Tile::kThreads, Tile::kThreads / 256) head_product_kernel(ProductArgs g, int64_t first_job) {
    typedef typename Tile::Element T;
    __shared__ typename Tile::Shared sh[Tile::kStages];
    const int which = blockIdx.x >= first_job;
    const ProductJob& job = g.job[which];
    int64_t id = blockIdx.x - (which ? first_job : 0);
    const Tiles tiles{(job.rows + Tile::kM - 1) / Tile::kM, (job.columns + Tile::kN - 1) / Tile::kN};
    const int64_t all = tiles.m * tiles.n;
    const int32_t split = (int32_t)(id / all);
    int64_t tm, tn;
    tiles.at(id - split * all, tm, tn);
    const int64_t m0 = tm * Tile::kM, n0 = tn * Tile::kN;
    const int64_t stages = Tile::stages(job.a);
    const int32_t from = (int32_t)(stages * split / job.splits), to = (int32_t)(stages * (split + 1) / job.splits);
    Tile t;
    t.run(job.a, job.b, m0, n0, from, to, sh);
    const float down = 1.0f / adjoint_scale(g.largest);
#pragma unroll
    for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
        for (int j = 0; j < Tile::TN; ++j) {
            const int64_t c = n0 + t.column(j);
            if (c >= job.columns) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int64_t r = m0 + t.row(i) + (e >> 2) * 8 + (e & 3);
                if (r >= job.rows) continue;
                const float x = t.acc[i][j][e] * down;
                if (job.out) {
                    static_cast<T*>(job.out)[r * job.columns + c] = (T)x;
                } else {
                    float* s = job.sums + ((int64_t)split * job.rows + r) * job.columns + c;
                    *s = job.add ? *s + x : x;
                }
            }
        }
}

// out[i] = sum over parts of from[part][i], in their order
struct SumArgs {
    const float* from;
    int64_t count, apart;
    int32_t parts, typed;                   // typed: out is of the operands' type, otherwise fp32
    void* out;
};
struct SumsArgs {
    SumArgs sum[3];
    int32_t sums;
};
template <typename T>
__global__ void __launch_bounds__(256) head_sums_kernel(SumsArgs g) {
    for (int s = 0; s < g.sums; ++s) {
        const SumArgs& a = g.sum[s];
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.count; i += (int64_t)gridDim.x * 256) {
            float x = a.from[i];
            for (int32_t p = 1; p < a.parts; ++p) x += a.from[p * a.apart + i];
            if (a.typed) static_cast<T*>(a.out)[i] = (T)x;
            else static_cast<float*>(a.out)[i] = x;
        }
    }
}

template <typename T> __global__ void __launch_bounds__(256) head_pack_kernel(PackArgs g) { pack_rows<T>(g, blockIdx.x, gridDim.x); }
template <typename T> __global__ void __launch_bounds__(256) head_pack_across_kernel(PackArgs g) { pack_across<T>(g, blockIdx.x, gridDim.x); }

// ---- launches of a type, each type in a translation unit of its own -------------------------------------------------
enum HeadTile : int { TILE_32, TILE_64, TILE_128, TILE_256 };
struct TileSize {
    int m, n;
};
constexpr TileSize kTileSizes[] = {{32, 128}, {64, 128}, {128, 128}, {256, 256}};

template <typename T> struct HeadLaunch {
    static klay_status forward(HeadTile tile, const HeadArgs& g, bool entropy, void* stream);
    static klay_status adjoint(HeadTile tile, const HeadArgs& g, void* stream);
    static klay_status products(HeadTile tile, const ProductArgs& g, void* stream);
    static klay_status sums(const SumsArgs& g, void* stream);
    static klay_status pack(const PackArgs& g, bool across, void* stream);
};

}  // namespace klay
