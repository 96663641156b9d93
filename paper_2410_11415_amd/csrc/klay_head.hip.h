// Log probabilities, and divergences from a teacher's list, straight from a network's hidden states: x_ij = h_i . w_j + b_j is made tile by tile in the
// registers of the matrix cores and never written.  Forward, a tile leaves of each row the sums over its tokens that are not listed (klay_lists.hip.h)
// and the logits of those that are; a wave a row joins them.  Backward, the tiles are made again, a piece of the vocabulary at a time, and turned
// into the adjoint of the logits, which in all of these losses has the form
//   G_ij = s_ij (A_i + B_i ln s_ij),  s_ij = e^((x_ij - ref_i) / T - ln S_i),
// with an entry of its own for a listed token; then dH = G W, dW = G^T H, db = sum_i G_i, W, H and G^T read across from memory
// that holds their rows.  G goes into the products as two numbers of the type of 16-bit operands, what the first one's rounding leaves in the second (bf16: off by
// 2^-16 of an entry at most; fp16: 2^-22, under a power of two taken from the largest entry, so that small adjoints stay in its range), or as the three parts of all
// operands of fp32.  Sums over tokens and rows are in fp32, in an order that the sizes alone decide.
#pragma once

#include "klay_lists.hip.h"
#include "klay_matrix.hip.h"

namespace klay {

// ---- what the C entry points hand to the kernels of a type -----------------------------------------------------------
struct HeadArgs {
    Operand hidden, weight;                 // [rows, width], [tokens of this launch, width]
    const float* bias;                      // of these tokens, or null
    int32_t first;                          // the first of these tokens
    int64_t rows;
    int32_t tail;                           // elements of a row behind its last whole piece of 16 bytes
    int32_t num_tokens;
    const int32_t* sorted;                  // [rows, num_tokens]; null (num_tokens = 1): `list` as it was given, from its row list_row on
    ListArgs list;
    int64_t list_row;
    float scale;                            // log2 e / T
    // forward
    float* values;                          // [rows, num_tokens]: the listed tokens' logits
    float4* partial;                        // [rows, tiles of tokens]: max, rest, weighted
    // backward
    const float4* coefs;                    // [rows]: ref (+inf: the row has no gradient), ln S log2 e, A, B ln 2
    const float* entries;                   // [rows, num_tokens]
    const uint32_t* largest;                // bits of the largest adjoint (fp16), or null
    uint32_t* odd;                          // made 1 if a token that the bias bars may have weights that are not finite; or null
    void* g;                                // [rows, g_columns], or null
    void* g_low;                            // likewise: what the rounding has left of g (16 bits), or null
    int64_t g_columns;                      // a multiple of 8
    float* bias_partial;                    // [tiles of rows, g_columns], or null
};

// One product of a launch: `splits` runs over its stages, each into fp32 sums of its own or, if it is the only one of all pieces, into `out`.
struct ProductJob {
    Operand a, b;                           // b lies across, a where a_across
    const uint32_t* odd;                    // null, or what decides whether b is rather a copy of it without what is not finite, `clean`, of this stride
    const void* clean;
    int64_t clean_stride;
    int32_t a_across, splits;
    int64_t rows, columns;
    void* out;                              // [rows, columns], or null
    int32_t stream;                         // out past the caches: its rows are whole lines of 128 bytes
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

// The tokens of a row that fall into a tile of ROWS rows and COLUMNS tokens: `first` their first place in the row's sorted list, a bit for each column.
template <int ROWS, int COLUMNS> struct Marks {
    static constexpr int kWords = COLUMNS / 32;
    uint32_t bits[ROWS][kWords];
    int32_t first[ROWS];
    // Short lists entry by entry, all loads at once; long ones row by row, from where a search finds the tile's first.  (Every thread comes here: barriers.)
    __device__ __forceinline__ void make(const HeadArgs& g, int64_t row0, int32_t token0, int32_t thread, int32_t threads) {
        const int32_t K = g.num_tokens;
        for (int i = thread; i < ROWS; i += threads) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) bits[i][w] = 0;
            first[i] = INT32_MAX;
        }
        __syncthreads();
        const int32_t rows = g.rows - row0 < ROWS ? (int32_t)(g.rows - row0) : ROWS;
        const int32_t* lists = g.sorted + row0 * K;
        if (K <= 8) {
#pragma unroll 4
            for (int32_t n = thread; n < rows * K; n += threads) {
                const uint32_t c = (uint32_t)(g.sorted ? lists[n] : token_of(g.list, g.list_row + row0 + n, 0)) - (uint32_t)token0;
                if (c >= (uint32_t)COLUMNS) continue;
                const int32_t i = n / K;
                atomicOr(&bits[i][c >> 5], 1u << (c & 31));
                atomicMin(&first[i], n - i * K);
            }
            return;
        }
        for (int i = thread; i < rows; i += threads) {
            const int32_t* list = lists + (int64_t)i * K;
            int32_t lo = 0, hi = K;
            while (lo < hi) {
                const int32_t mid = (lo + hi) >> 1;
                if (list[mid] < token0) lo = mid + 1;
                else hi = mid;
            }
            first[i] = lo;
            for (; lo < K; ++lo) {
                const uint32_t c = (uint32_t)list[lo] - (uint32_t)token0;
                if (c >= (uint32_t)COLUMNS) break;
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
// f(i, e, place) for a lane's marked columns of its row of block j: element e of its i-th block, and the token's place in the row's list.
template <typename Tile, typename M, typename F>
__device__ __forceinline__ void each_mark(const Tile& t, const M& marks, int j, F&& f) {
#pragma unroll
    for (int i = 0; i < Tile::TM; ++i) {
        const int word = t.columns_from(i) / 32;
        const uint32_t mine = marks.bits[t.row(j)][word] >> (4 * (t.lane >> 5));
        if (__ballot((mine & 0x0f0f0f0fu) != 0) == 0) continue;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (mine >> (8 * (e >> 2) + (e & 3)) & 1u) f(i, e, marks.place(t.row(j), word, 8 * (e >> 2) + (e & 3) + 4 * (t.lane >> 5)));
    }
}
// The bias of a lane's columns, -inf where there are none: `some` is whether it changes anything.
template <typename Tile>
__device__ __forceinline__ bool some_bias(const HeadArgs& g, int64_t column0) { return g.bias != nullptr || column0 + Tile::kM > g.weight.rows; }
template <typename Tile>
__device__ __forceinline__ bool add_bias(Tile& t, const HeadArgs& g, int64_t column0) {
    bool odd = false;                       // (such a token's logits are not finite, whatever the row)
#pragma unroll
    for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int64_t c = column0 + t.column(i) + 8 * (e >> 2) + (e & 3);
            const float b = c < g.weight.rows ? (g.bias ? g.bias[c] : 0.0f) : -INFINITY;
#pragma unroll
            for (int j = 0; j < Tile::TN; ++j) {
                odd |= b == -INFINITY && c < g.weight.rows && !(fabsf(t.acc[i][j][e]) < INFINITY);
                t.acc[i][j][e] = b == -INFINITY ? -INFINITY : t.acc[i][j][e] + b;
            }
        }
    return odd;
}

// What the elements behind the last whole pieces add to the logits: through shared memory (`at`: 32 bytes a row and column), in fp32.
template <typename Tile>
__device__ __forceinline__ void add_tail(Tile& t, const HeadArgs& g, int64_t row0, int64_t column0, char* at) {
    typedef typename Tile::Element T;
    constexpr int ROWS = Tile::kN, COLUMNS = Tile::kM, MOST = 8;
    float(*h)[MOST] = reinterpret_cast<float(*)[MOST]>(at), (*w)[MOST] = h + ROWS;
    for (int i = threadIdx.x; i < (ROWS + COLUMNS) * MOST; i += Tile::kThreads) {
        const int r = i / MOST, d = i % MOST;
        const Operand& o = r < ROWS ? g.hidden : g.weight;
        const int64_t row = r < ROWS ? row0 + r : column0 + r - ROWS;
        const T* from = reinterpret_cast<const T*>(static_cast<const char*>(o.p) + row * o.stride + (int64_t)o.pieces * 16);
        h[r][d] = d < g.tail && row < o.rows ? (float)from[d] : 0.0f;
    }
    __syncthreads();
    for (int d = 0; d < g.tail; ++d) {
        float x[Tile::TN];
#pragma unroll
        for (int j = 0; j < Tile::TN; ++j) x[j] = h[t.row(j)][d];
#pragma unroll
        for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float y = w[t.column(i) + 8 * (e >> 2) + (e & 3)][d];
#pragma unroll
                for (int j = 0; j < Tile::TN; ++j) t.acc[i][j][e] = fmaf(x[j], y, t.acc[i][j][e]);
            }
    }
    __syncthreads();
}

// ---- forward ---------------------------------------------------------------------------------------------------------
// What a lane finds out about its columns of its row of block j, and the other half of the wave about the others': y = x scale - shift with shift = max scale
// rounded by itself is one multiply-add; what that rounding puts into all terms, 2^d, comes out again at the end.  WIDE takes the difference first, for
// maxima so far from 0 that the product would leave the range of fp32 (a row of nothing but the type's lowest value, for one).
struct Part {
    float max, rest, weighted;
};
template <bool ENT, bool WIDE, typename Tile>
__device__ __forceinline__ Part part_of(const Tile& t, int j, float max, float scale) {
    const float to = WIDE ? fmaxf(max, -kTokFltMax) : max == -INFINITY ? 0.0f : max, shift = to * scale;
    auto term = [&](float x) { return WIDE ? (x - to) * scale : fmaf(x, scale, -shift); };
    float s = 0.0f, u = 0.0f;
#pragma unroll
    for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float y = term(t.acc[i][j][e]), p = exp2_of(y);
            s += p;
            if constexpr (ENT) u = fmaf(p, fmaxf(y, -200.0f), u);
        }
    s += __shfl_xor(s, 32);
    if constexpr (ENT) u += __shfl_xor(u, 32);
    if constexpr (!WIDE) {
        const float d = fmaf(to, scale, -shift), f = exp2_of(-d);
        u = f * (u - d * s);
        s *= f;
    }
    float rest = s == 0.0f ? 0.0f : s - 1.0f;
    if (s > 0.0f && s < 1.5f) {                                  // one holds most of the sum: the others by themselves
        rest = 0.0f;
#pragma unroll
        for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) rest += t.acc[i][j][e] == max ? 0.0f : exp2_of((t.acc[i][j][e] - to) * scale);
    }
    const float other = __shfl_xor(rest, 32);                    // (both halves have the same s)
    if (s > 0.0f && s < 1.5f) rest += other;
    return Part{max, rest, u};
}
// The part with the larger maximum keeps its rest; the other brings its maximum's own term along.
__device__ __forceinline__ Part joined(const Part& a, const Part& b, float scale) {
    const bool up = b.max > a.max;
    const Part big = up ? b : a, small = up ? a : b;
    const bool none = small.max == -INFINITY && small.rest == 0.0f;
    const float d = (fmaxf(small.max, -kTokFltMax) - fmaxf(big.max, -kTokFltMax)) * scale, f = none ? 0.0f : exp2_of(d), whole = 1.0f + small.rest;
    return Part{big.max, big.rest + (none ? 0.0f : f * whole), big.weighted + (f > 0.0f ? f * (small.weighted + d * whole) : 0.0f)};
}

template <typename Tile, bool ENT>
__global__ void __launch_bounds__(Tile::kThreads, Tile::kThreads / 256) head_forward_kernel(HeadArgs g, Tiles tiles) {
    constexpr int ROWS = Tile::kN, COLUMNS = Tile::kM, TM = Tile::TM, TN = Tile::TN, PARTS = Tile::kWavesM;
    // (one object: of several the compiler would wait for all loads into one before every read of it)
    __shared__ struct {
        typename Tile::Shared stage[Tile::kStages];
        Marks<ROWS, COLUMNS> marks;
        Part parts[PARTS][ROWS];
    } sh;
    int64_t tr, tc;
    tiles.at(blockIdx.x, tr, tc);
    const int64_t row0 = tr * ROWS, column0 = tc * COLUMNS;
    Tile t;
    t.template run<false, false>(g.weight, g.hidden, column0, row0, 0, Tile::stages(g.hidden), sh.stage, [&] {
        if (g.num_tokens) sh.marks.make(g, row0, g.first + (int32_t)column0, threadIdx.x, Tile::kThreads);
    });
    if (g.tail) add_tail(t, g, row0, column0, reinterpret_cast<char*>(sh.stage));
    if (some_bias<Tile>(g, column0)) add_bias(t, g, column0);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        if (g.num_tokens)
            each_mark(t, sh.marks, j, [&](int i, int e, int32_t place) {
                g.values[(row0 + t.row(j)) * g.num_tokens + place] = t.acc[i][j][e];
                t.acc[i][j][e] = -INFINITY;
            });
        float max = t.acc[0][j][0];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) max = fmaxf(max, t.acc[i][j][e]);
        max = fmaxf(max, __shfl_xor(max, 32));
        Part part = part_of<ENT, false>(t, j, max, g.scale);
        const bool far = fabsf(max) < INFINITY && fabsf(max) * g.scale > 1e37f;
        if (__ballot(far)) {
            const Part wide = part_of<ENT, true>(t, j, max, g.scale);
            if (far) part = wide;                                 // (a row's bits do not depend on its neighbours)
        }
        if (t.lane < 32) sh.parts[t.wm][t.row(j)] = part;
    }
    __syncthreads();
    for (int row = threadIdx.x; row < ROWS; row += Tile::kThreads) {
        if (row0 + row >= g.rows) break;
        Part part = sh.parts[0][row];
#pragma unroll
        for (int w = 1; w < PARTS; ++w) part = joined(part, sh.parts[w][row], g.scale);
        g.partial[(row0 + row) * tiles.n + tc] = make_float4(part.max, part.rest, part.weighted, 0.0f);
    }
}

// Over the 32 lanes of a half of the wave; all of them get the result.
__device__ __forceinline__ float half_sum(float x) {
    x = group_sum<16>(x);
    return x + __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401f));       // (lane ^ 16)
}

// ---- backward --------------------------------------------------------------------------------------------------------
template <typename Tile>
__global__ void __launch_bounds__(Tile::kThreads, Tile::kThreads / 256) head_adjoint_kernel(HeadArgs g, Tiles tiles) {
    typedef typename Tile::Element T;
    constexpr int ROWS = Tile::kN, COLUMNS = Tile::kM, TM = Tile::TM, TN = Tile::TN, WN = Tile::kWavesN;
    __shared__ struct {
        typename Tile::Shared stage[Tile::kStages];
        Marks<ROWS, COLUMNS> marks;
        float sums[WN][COLUMNS];
    } sh;
    int64_t tr, tc;
    tiles.at(blockIdx.x, tr, tc);
    const int64_t row0 = tr * ROWS, column0 = tc * COLUMNS;
    Tile t;
    t.template run<false, false>(g.weight, g.hidden, column0, row0, 0, Tile::stages(g.hidden), sh.stage, [&] {
        if (g.num_tokens) sh.marks.make(g, row0, g.first + (int32_t)column0, threadIdx.x, Tile::kThreads);
    });
    if (g.tail) add_tail(t, g, row0, column0, reinterpret_cast<char*>(sh.stage));
    if (some_bias<Tile>(g, column0) && add_bias(t, g, column0) && g.odd) *g.odd = 1;
    const bool last = column0 + COLUMNS > g.weight.rows;
    const float up = adjoint_scale(g.largest);
    const uint32_t lower = 4 * (t.lane >> 5);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t r = row0 + t.row(j);
        const float4 c = r < g.rows ? g.coefs[r] : make_float4(INFINITY, 0.0f, 0.0f, 0.0f);
        const bool live = c.x < INFINITY;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const uint32_t block = t.columns_from(i);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float y = fmaf(t.acc[i][j][e] - c.x, g.scale, -c.y);
                t.acc[i][j][e] = live ? exp2_of(y) * fmaf(c.w, fmaxf(y, -200.0f), c.z) : 0.0f;
            }
            if (g.num_tokens) {
                const uint32_t mine = sh.marks.bits[t.row(j)][block / 32] >> lower;
                if (__ballot((mine & 0x0f0f0f0fu) != 0)) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int bit = 8 * (e >> 2) + (e & 3);
                        if (mine >> bit & 1u) t.acc[i][j][e] = g.entries[r * g.num_tokens + sh.marks.place(t.row(j), block / 32, bit + lower)];
                    }
                }
            }
            if (last) {                                           // (columns of no token: nothing, whatever the row holds)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (column0 + t.column(i) + 8 * (e >> 2) + (e & 3) >= g.weight.rows) t.acc[i][j][e] = 0.0f;
            }
        }
    }
    const auto write = [&](void* to, float scale) {
        t.template each_line<T>(reinterpret_cast<char*>(sh.stage), scale, [&](int row, int column, const typename Tile::template Line<T>& x) {
            const int64_t r = row0 + row, c = column0 + column;
            if (r < g.rows && c < g.g_columns)                    // (a multiple of 8: whole lines)
                *reinterpret_cast<typename Tile::template Line<T>*>(static_cast<T*>(to) + r * g.g_columns + c) = x;
        });
    };
    if (g.g) write(g.g, up);
    if (g.bias_partial) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float sum = t.acc[i][0][e];
#pragma unroll
                for (int j = 1; j < TN; ++j) sum += t.acc[i][j][e];
                sum = half_sum(sum);
                if ((t.lane & 31) == 0) sh.sums[t.wn][t.column(i) + 8 * (e >> 2) + (e & 3)] = sum;
            }
        __syncthreads();
        for (int c = threadIdx.x; c < COLUMNS; c += Tile::kThreads) {
            float s = sh.sums[0][c];
#pragma unroll
            for (int w = 1; w < WN; ++w) s += sh.sums[w][c];
            if (column0 + c < g.g_columns) g.bias_partial[tr * g.g_columns + column0 + c] = s;
        }
    }
    if constexpr (sizeof(T) == 2)
        if (g.g_low) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float d = t.acc[i][j][e] * up, low = d - (float)(T)d;
                        t.acc[i][j][e] = low == low ? low : 0.0f;          // (of an infinity nothing is left)
                    }
            write(g.g_low, 1.0f);
        }
}

template <typename Tile>
__global__ void __launch_bounds__(Tile::kThreads, Tile::kThreads / 256) head_product_kernel(ProductArgs g, int64_t first_job) {
    typedef typename Tile::Element T;
    __shared__ typename Tile::Shared sh[Tile::kStages];
    const int which = blockIdx.x >= first_job;
    const ProductJob& job = g.job[which];
    int64_t id = blockIdx.x - (which ? first_job : 0);
    const Tiles tiles{(job.rows + Tile::kN - 1) / Tile::kN, (job.columns + Tile::kM - 1) / Tile::kM};
    const int64_t all = tiles.m * tiles.n;
    const int32_t split = (int32_t)(id / all);
    int64_t tr, tc;
    tiles.at(id - split * all, tr, tc);
    const int64_t row0 = tr * Tile::kN, column0 = tc * Tile::kM;
    const int64_t stages = job.a_across ? Tile::stages_across(job.a) : Tile::stages(job.a);
    const int32_t from = (int32_t)(stages * split / job.splits), to = (int32_t)(stages * (split + 1) / job.splits);
    Operand b = job.b;
    if (job.odd && *job.odd) {
        b.p = job.clean;
        b.stride = job.clean_stride;
    }
    Tile t;
    if (job.a_across) t.template run<true, true>(b, job.a, column0, row0, from, to, sh, [] {});
    else t.template run<true, false>(b, job.a, column0, row0, from, to, sh, [] {});
    const float down = 1.0f / adjoint_scale(g.largest);
    char* const lds = reinterpret_cast<char*>(sh);
    if (job.out) {
        auto put = [&](int row, int column, const typename Tile::template Line<T>& x, auto past) {
            const int64_t r = row0 + row, c = column0 + column;
            if (r >= job.rows || c >= job.columns) return;
            constexpr int N = 16 / sizeof(T);
            T* out = static_cast<T*>(job.out) + r * job.columns + c;
            if (c + N <= job.columns) {
                auto* line = reinterpret_cast<typename Pieces<T, N>::Loose*>(out);
                if constexpr (past) __builtin_nontemporal_store(x, line);
                else *line = x;
            } else {
#pragma unroll
                for (int e = 0; e < N - 1; ++e)
                    if (c + e < job.columns) out[e] = x[e];
            }
        };
        if (Tile::kStages == 1 && job.stream)
            t.template each_line<T>(lds, down, [&](int row, int column, const auto& x) { put(row, column, x, std::true_type{}); });
        else
            t.template each_line<T>(lds, down, [&](int row, int column, const auto& x) { put(row, column, x, std::false_type{}); });
        return;
    }
    if constexpr (Tile::kStages > 1)                              // (a single stage: the only sum)
        t.template each_line<float>(lds, down, [&](int row, int column, const typename Tile::template Line<float>& x) {
            const int64_t r = row0 + row, c = column0 + column;
            if (r >= job.rows || c >= job.columns) return;
            float* s = job.sums + ((int64_t)split * job.rows + r) * job.columns + c;
            if (c + 4 <= job.columns) {
                auto* four = reinterpret_cast<typename Pieces<float, 4>::Loose*>(s);
                *four = job.add ? *four + x : x;
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (c + e < job.columns) s[e] = job.add ? s[e] + x[e] : x[e];
            }
        });
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
            for (int32_t p = 1; p < a.parts; p += 8) {
                float y[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) y[q] = p + q < a.parts ? a.from[(p + q) * a.apart + i] : 0.0f;
#pragma unroll
                for (int q = 0; q < 8; ++q) x += y[q];
            }
            if (a.typed) static_cast<T*>(a.out)[i] = (T)x;
            else static_cast<float*>(a.out)[i] = x;
        }
    }
}

// Copies of a launch: workgroups until[i - 1] .. until[i] - 1 make copy i.
struct PacksArgs {
    PackArgs copy[5];
    uint32_t until[5];
    int32_t copies;
    uint32_t* clear;                        // two words that are made 0, or null
    const uint32_t* only;                   // null, or: nothing is copied if this is 0
};
template <typename T> __global__ void __launch_bounds__(256) head_pack_kernel(PacksArgs g) {
    if (g.clear && blockIdx.x == 0 && threadIdx.x < 2) g.clear[threadIdx.x] = 0;
    if (g.only && *g.only == 0) return;
    uint32_t first = 0;
    for (int i = 0; i < g.copies; ++i) {
        if (blockIdx.x < g.until[i]) {
            pack_rows<T>(g.copy[i], blockIdx.x - first, g.until[i] - first);
            return;
        }
        first = g.until[i];
    }
}

// ---- launches of a type, each type in a translation unit of its own -------------------------------------------------
enum HeadTile : int { TILE_32, TILE_64, TILE_128, TILE_256, TILE_ONE };    // (TILE_ONE: weights' gradients of a single stage, 128 x 128)
struct TileSize {
    int rows, columns;
};
constexpr TileSize kTileSizes[] = {{32, 128}, {64, 128}, {128, 128}, {256, 256}, {128, 128}};

template <typename T> struct HeadLaunch {
    static klay_status forward(HeadTile tile, const HeadArgs& g, bool entropy, void* stream);
    static klay_status adjoint(HeadTile tile, const HeadArgs& g, void* stream);
    static klay_status products(HeadTile tile, const ProductArgs& g, void* stream);
    static klay_status sums(const SumsArgs& g, void* stream);
    static klay_status pack(PacksArgs& g, void* stream);      // (copies, copy, clear, only given)
};

}  // namespace klay
