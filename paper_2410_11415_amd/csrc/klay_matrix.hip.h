// Products of matrices for the head of a network: C[m, n] = sum_k A[m, k] B[n, k], both operands with k next to each other, sums in fp32 by
// v_mfma_f32_32x32x16.  fp32 elements are three bf16 each on their way into the registers (a float's 24 bits are three times eight: hi + mid +
// lo = x exactly between 2^-110 and 3.38e38), and of the nine products the six that reach fp32's precision are made; the dropped ones are below 2^-25
// of hi x hi.
#pragma once

#include "klay_typed.hip.h"

namespace klay {

typedef float Acc __attribute__((ext_vector_type(16)));
template <typename T> using Eight = typename Pieces<T, 8>::Vec;

__device__ __forceinline__ Acc mma(Eight<bf16> a, Eight<bf16> b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ Acc mma(Eight<f16> a, Eight<f16> b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

constexpr int kStageBytes = 128;            // a row's share of a stage: 64 k's of 16 bits, 32 of 32
constexpr int kStagePieces = kStageBytes / 16;
constexpr uint32_t kMostStride = 1u << 23;  // bytes from row to row: 256 rows lie within 31 bits

// One side of a product.
struct Operand {
    const void* p;                          // 16-byte aligned
    int64_t stride;                         // bytes from row to row, a multiple of 16, at most kMostStride
    int64_t rows;
    int32_t pieces;                         // 16-byte pieces of a row; what lies behind them reads as zeros
};

// The 16-byte pieces of a stage's row lie permuted by bits 1 .. 3 of the row, so that the rows of a fragment come from all banks.
__device__ __forceinline__ int place_of(int row, int piece) { return piece ^ ((row >> 1) & 7); }

// A wave's part of the loads of ROWS rows by WAVES waves: 1 KB, eight rows, an instruction, straight into shared memory.
template <int ROWS, int WAVES> struct Stage {
    static constexpr int kLoads = ROWS / 8 / WAVES;
    static_assert(ROWS % (8 * WAVES) == 0 && (WAVES % 2 == 0 || kLoads == 1), "whole loads, one permutation a lane");
    Stretch from;
    uint32_t offset[kLoads];
    int32_t piece, pieces;
    __device__ __forceinline__ void init(const Operand& s, int64_t row0, int wave, int lane) {
        from = stretch_at(static_cast<const char*>(s.p) + row0 * s.stride);
        pieces = s.pieces;
        piece = place_of(wave * 8 + (lane >> 3), lane & 7);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = (i * WAVES + wave) * 8 + (lane >> 3);
            offset[i] = row0 + r < s.rows ? (uint32_t)r * (uint32_t)s.stride + (uint32_t)piece * 16u : kNoLane;
        }
    }
    // stage `at` of k; behind the last piece: zeros
    __device__ __forceinline__ void load(int at, char* lds, int wave) const {
        const bool in = at * kStagePieces + piece < pieces;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(lds + (i * WAVES + wave) * 1024), 16,
                                                     in ? offset[i] : kNoLane, at * kStageBytes, 0, 0);
    }
};

// The eight k's of a lane's row that a matrix instruction takes, `half` 0 or 1 of sixteen.
template <typename T> struct Fragment {
    static constexpr int kSixteens = 4;     // of a stage
    Eight<T> x;
    __device__ __forceinline__ void load(const char* lds, int row, int s, int half) {
        x = *reinterpret_cast<const Eight<T>*>(lds + row * kStageBytes + place_of(row, 2 * s + half) * 16);
    }
};
template <> struct Fragment<f32> {
    static constexpr int kSixteens = 2;
    Eight<bf16> hi, mid, lo;
    __device__ __forceinline__ void load(const char* lds, int row, int s, int half) {
        typedef float Four __attribute__((ext_vector_type(4)));
        typedef float Floats __attribute__((ext_vector_type(8)));
        const Four a = *reinterpret_cast<const Four*>(lds + row * kStageBytes + place_of(row, 4 * s + 2 * half) * 16);
        const Four b = *reinterpret_cast<const Four*>(lds + row * kStageBytes + place_of(row, 4 * s + 2 * half + 1) * 16);
        Floats x = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        hi = __builtin_convertvector(x, Eight<bf16>);
        x -= __builtin_convertvector(hi, Floats);
        mid = __builtin_convertvector(x, Eight<bf16>);
        x -= __builtin_convertvector(mid, Floats);
        lo = __builtin_convertvector(x, Eight<bf16>);
    }
};

// A tile of BM x BN by WM x WN waves, S stages of k in shared memory; wave (wm, wn) has TM x TN blocks of 32 x 32 in registers.  Lane l of a block holds
// column l % 32 and of it the rows 8 q + 4 (l / 32) + e as element 4 q + e.
template <typename T, int BM, int BN, int WM, int WN, int S> struct Tile {
    static constexpr int kM = BM, kN = BN, kWavesM = WM, kWavesN = WN, kWaves = WM * WN, kThreads = 64 * kWaves, kStages = S;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    typedef T Element;
    struct Shared {                         // one stage
        char a[BM * kStageBytes], b[BN * kStageBytes];
    };
    Acc acc[TM][TN];
    int wave, lane, wm, wn;
    __device__ __forceinline__ Tile() {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        wm = wave / WN;
        wn = wave % WN;
    }
    // of the tile: a lane's first row of block row i (the others: + 8 q + e), its column of block column j
    __device__ __forceinline__ int row(int i) const { return (wm * TM + i) * 32 + 4 * (lane >> 5); }
    __device__ __forceinline__ int column(int j) const { return (wn * TN + j) * 32 + (lane & 31); }

    __device__ __forceinline__ void step(const char* a, const char* b) {
        const int r = lane & 31, half = lane >> 5;
#pragma unroll
        for (int s = 0; s < Fragment<T>::kSixteens; ++s) {
            Fragment<T> fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i].load(a, (wm * TM + i) * 32 + r, s, half);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j].load(b, (wn * TN + j) * 32 + r, s, half);
            auto all = [&](auto&& one) {
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = one(fa[i], fb[j], acc[i][j]);
            };
            typedef Fragment<T> F;
            if constexpr (std::is_same_v<T, f32>) {          // smallest first
                all([](const F& x, const F& y, Acc c) { return mma(x.lo, y.hi, c); });
                all([](const F& x, const F& y, Acc c) { return mma(x.hi, y.lo, c); });
                all([](const F& x, const F& y, Acc c) { return mma(x.mid, y.mid, c); });
                all([](const F& x, const F& y, Acc c) { return mma(x.mid, y.hi, c); });
                all([](const F& x, const F& y, Acc c) { return mma(x.hi, y.mid, c); });
                all([](const F& x, const F& y, Acc c) { return mma(x.hi, y.hi, c); });
            } else {
                all([](const F& x, const F& y, Acc c) { return mma(x.x, y.x, c); });
            }
        }
    }
    // Stages from .. to - 1 of rows m0 .. of a and n0 .. of b.  Stage s + S - 1 is asked for while stage s is worked on, in the place of stage s - 1, which
    // all waves have left at the barrier between the two.  (Stages behind the last one read zeros, so that always as many loads are on their way.)
    // Ends with a barrier: shared memory is free again.
    __device__ __forceinline__ void run(const Operand& oa, const Operand& ob, int64_t m0, int64_t n0, int from, int to, Shared (&sh)[S]) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = Acc{};
        Stage<BM, kWaves> la;
        Stage<BN, kWaves> lb;
        la.init(oa, m0, wave, lane);
        lb.init(ob, n0, wave, lane);
        constexpr int kInFlight = (S - 2) * (Stage<BM, kWaves>::kLoads + Stage<BN, kWaves>::kLoads);
#pragma unroll
        for (int s = 0; s < S - 1; ++s) {
            la.load(from + s, sh[s].a, wave);
            lb.load(from + s, sh[s].b, wave);
        }
        for (int kt = from; kt < to; kt += S) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                if (kt + s >= to) break;
                asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kInFlight) : "memory");
                la.load(kt + s + S - 1, sh[(s + S - 1) % S].a, wave);
                lb.load(kt + s + S - 1, sh[(s + S - 1) % S].b, wave);
                step(sh[s].a, sh[s].b);
            }
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
};

// Which tile a workgroup takes: the workgroups that an XCD gets (every eighth) take a stretch of the tiles, bands of kBand columns of tiles at a
// time, so that what its L2 holds is read by several.
constexpr int kXcds = 8, kBand = 4;
struct Tiles {
    int64_t m, n;                           // tiles along rows and columns
    __device__ __forceinline__ void at(int64_t id, int64_t& tm, int64_t& tn) const {
        const int64_t total = m * n, each = total / kXcds, more = total - each * kXcds, x = id % kXcds;
        const int64_t t = x * each + (x < more ? x : more) + id / kXcds;
        const int64_t band = t / (m * kBand), first = band * kBand, wide = n - first < kBand ? n - first : kBand;
        const int64_t in = t - band * m * kBand;
        tm = in / wide;
        tn = first + in - tm * wide;
    }
};

// ---- operands as the products take them ----------------------------------------------------------------------------
struct PackArgs {
    const void* from;
    int64_t outer, inner_stride;            // row r: (r / inner) * outer + (r % inner) * inner_stride elements on
    int64_t inner;
    int64_t count, columns;                 // rows and columns taken
    void* to;
    int64_t stride;                         // of the copy, elements
    int64_t padded;                         // elements of a row of the copy; zeros behind what is taken
    const float4* coefs;                    // a row whose x is +inf has no gradient and is zeros; null: none is
    const float* bias;                      // of a row whose entry is -inf only what is finite is taken; null: all is
};
__device__ __forceinline__ int64_t packed_row(const PackArgs& g, int64_t r) { return r / g.inner * g.outer + r % g.inner * g.inner_stride; }
__device__ __forceinline__ bool packed_live(const PackArgs& g, int64_t r) { return !g.coefs || g.coefs[r].x < INFINITY; }

// Rows as they are: a thread takes 16 bytes of the copy.
template <typename T>
__device__ __forceinline__ void pack_rows(const PackArgs& g, int64_t block, int64_t blocks) {
    constexpr int N = 16 / sizeof(T);
    const int64_t across = g.padded / N, all = g.count * across;
    for (int64_t i = block * 256 + threadIdx.x; i < all; i += blocks * 256) {
        const int64_t r = i / across, c = (i - r * across) * N;
        typename Pieces<T, N>::Vec out = {};
        const T* row = static_cast<const T*>(g.from) + packed_row(g, r);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c + e < g.columns) out[e] = row[c + e];
        *reinterpret_cast<typename Pieces<T, N>::Vec*>(static_cast<T*>(g.to) + r * g.stride + c) = out;
    }
}

// Rows and columns exchanged: copy[c][r], `padded` (a multiple of 16 bytes) next to each other, by squares of 64 x 64.
template <typename T>
__device__ __forceinline__ void pack_across(const PackArgs& g, int64_t block, int64_t blocks) {
    constexpr int N = 16 / sizeof(T);
    __shared__ T square[64][65];
    const int64_t across = (g.columns + 63) / 64, all = (g.padded + 63) / 64 * across;
    for (int64_t i = block; i < all; i += blocks) {
        const int64_t r0 = i / across * 64, c0 = (i % across) * 64;
        for (int e = threadIdx.x; e < 64 * 64; e += 256) {
            const int r = e >> 6, c = e & 63;
            T x = (T)0.0f;
            if (r0 + r < g.count && c0 + c < g.columns && packed_live(g, r0 + r)) {
                x = (static_cast<const T*>(g.from) + packed_row(g, r0 + r))[c0 + c];
                if (g.bias && g.bias[r0 + r] == -INFINITY && !(fabsf((float)x) < INFINITY)) x = (T)0.0f;
            }
            square[r][c] = x;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 64 * 64 / N; e += 256) {
            const int c = e / (64 / N), r = e % (64 / N) * N;
            if (c0 + c >= g.columns || r0 + r >= g.padded) continue;
            typename Pieces<T, N>::Vec out;
#pragma unroll
            for (int q = 0; q < N; ++q) out[q] = square[r + q][c];
            *reinterpret_cast<typename Pieces<T, N>::Vec*>(static_cast<T*>(g.to) + (c0 + c) * g.stride + r0 + r) = out;
        }
        __syncthreads();
    }
}

}  // namespace klay
