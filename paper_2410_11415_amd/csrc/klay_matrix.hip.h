// Products of matrices for the head of a network: C[n, m] = sum_k A[m, k] B[n, k], sums in fp32 by
// v_mfma_f32_32x32x16.  fp32 elements are three bf16 each on their way into the registers (a float's 24 bits are three times eight: hi + mid +
// lo = x exactly above 2^-110), and of the nine products the six that reach fp32's precision are made; the dropped ones are below 2^-21 of hi x hi
// each, 2^-24 on average.
#pragma once

#include "klay_typed.hip.h"

namespace klay {

typedef float Acc __attribute__((ext_vector_type(16)));
template <typename T> using Eight = typename Pieces<T, 8>::Vec;

__device__ __forceinline__ Acc mma(Eight<bf16> a, Eight<bf16> b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ Acc mma(Eight<f16> a, Eight<f16> b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// A stage of k: SB bytes of each row, 64 or 128 (32 or 64 k's of 16 bits, half as many of 32).
constexpr int kMostStageBytes = 128;
constexpr uint32_t kMostStride = 1u << 23;  // bytes from row to row: 256 rows lie within 31 bits

// One side of a product: rows with k next to each other; or, `across`, rows of k with the side's own rows next to each other.  Rows start at multiples of 4
// bytes, and nothing is read behind the four bytes that the last one ends in.
struct Operand {
    const void* p;
    int64_t stride;                         // bytes from row to row (across: from k to k), a multiple of 4, as long as a row at least, at most kMostStride
    int64_t rows;
    int32_t pieces;                         // whole pieces of 16 bytes of a row; what lies behind them reads as zeros.  Across: the number of k's
};

// The 16-byte pieces of a stage's row lie permuted by the row's place among sixteen, so that the rows of a fragment come from all banks.
template <int SB> __device__ __forceinline__ int place_of(int row, int piece) { return piece ^ (SB == 128 ? (row >> 1) & 7 : (row >> 2) & 3); }

// `bytes` of memory from p on, which buffer loads do not read beyond (zeros instead).
__device__ __forceinline__ Stretch stretch_of(const void* p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)(bytes < (int64_t)kStretchBytes ? bytes : kStretchBytes), 0x00020000);
}

// x, about which the compiler knows nothing more: what is added to it is added where it is used, and not kept in registers of its own all the loop long.
__device__ __forceinline__ uint32_t fresh(uint32_t x) {
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("" : "+v"(x));
#endif
    return x;
}

// A wave's part of the loads of one side's ROWS rows by WAVES waves, in HALVES halves: 1 KB an instruction, straight into shared memory.
template <int ROWS, int HALVES, int WAVES, int SB> struct Stage {
    static constexpr int kRows = 1024 / SB, kPieces = SB / 16, kLoads = ROWS / HALVES / kRows / WAVES;
    static_assert(ROWS % (HALVES * kRows * WAVES) == 0 && (WAVES * kRows) % 16 == 0, "whole loads, one permutation a lane");
    Stretch from;
    uint32_t stride, offset;                // of the first load; the others' rows are whole strides on
    int32_t piece, pieces;
    static __device__ __forceinline__ int first_row(int half, int i, int wave) { return half * (ROWS / HALVES) + (i * WAVES + wave) * kRows; }
    __device__ __forceinline__ void init(const Operand& s, int64_t row0, int wave, int lane) {
        const int64_t left = s.rows - row0;
        from = stretch_of(static_cast<const char*>(s.p) + row0 * s.stride, (left < ROWS ? left : ROWS) * s.stride);
        pieces = s.pieces;
        stride = (uint32_t)s.stride;
        piece = place_of<SB>(first_row(0, 0, wave) + lane / kPieces, lane % kPieces);
        offset = (uint32_t)(first_row(0, 0, wave) + lane / kPieces) * stride + (uint32_t)piece * 16u;
    }
    // a half, or all, of stage `at` of k; behind the last piece: zeros
    __device__ __forceinline__ void load(int half, int at, char* lds, int wave) const {
        const uint32_t here = fresh(offset);
        const bool in = at * kPieces + piece < pieces;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(lds + first_row(half, i, wave) * SB), 16,
                                                     in ? here + (first_row(half, i, 0) * stride + at * SB) : kNoLane, 0, 0, 0);
    }
};
// Likewise of an operand that lies across.  (Of rows behind the last one comes what lies there, for results that nobody stores.)
template <int ROWS, int HALVES, int WAVES, int SB, int BYTES> struct StageAcross;
// 16 bits: 64 k's of 64 of its rows (128 bytes) after the other.  Every other pair of k's has its 64-byte halves exchanged, so that the four k's of a transposing
// read come from all banks.
template <int ROWS, int HALVES, int WAVES, int SB> struct StageAcross<ROWS, HALVES, WAVES, SB, 2> {
    static constexpr int kAll = ROWS < 64 ? 64 : ROWS, kLoads = kAll / HALVES / 8 / WAVES;
    static_assert(SB == 128 && kAll % (HALVES * 64) == 0 && kAll % (HALVES * 8 * WAVES) == 0, "whole loads");
    const char* from;
    int64_t bytes;                          // from there to the operand's end
    uint32_t stride, offset;
    static __device__ __forceinline__ int first(int half, int i, int wave) { return half * (kAll / HALVES) + (i * WAVES + wave) * 8; }
    __device__ __forceinline__ void init(const Operand& s, int64_t row0, int wave, int lane) {
        from = static_cast<const char*>(s.p) + row0 * 2;
        stride = (uint32_t)s.stride;
        bytes = ((s.pieces - 1) * s.stride + (s.rows - row0) * 2 + 3) & ~(int64_t)3;     // (loads are in or out of range by four bytes)
        const int k = lane >> 3;
        offset = (uint32_t)k * stride + (uint32_t)((lane & 7) ^ (((k >> 1) & 1) << 2)) * 16u;
    }
    __device__ __forceinline__ void load(int half, int at, char* lds, int wave) const {
        const int64_t gone = at * 64 * (int64_t)stride;
        const Stretch stage = stretch_of(from + gone, gone < bytes ? bytes - gone : 0);
        const uint32_t here = fresh(offset);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int place = first(half, i, wave);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(stage, (__attribute__((address_space(3))) void*)(lds + place * 128), 16,
                                                     here + ((uint32_t)(place & 63) * stride + (uint32_t)(place & ~63) * 2u), 0, 0, 0);
        }
    }
};
// 32 bits: the k's of a stage one after the other, a half's rows each.
template <int ROWS, int HALVES, int WAVES, int SB> struct StageAcross<ROWS, HALVES, WAVES, SB, 4> {
    static constexpr int kKs = SB / 4, kLong = ROWS / HALVES * 4, kEach = 1024 / kLong, kLoads = kKs / kEach / WAVES;
    static_assert(kLong <= 1024 && kKs % (kEach * WAVES) == 0, "whole loads");
    const char* from;
    int64_t bytes;
    uint32_t stride, offset;
    __device__ __forceinline__ void init(const Operand& s, int64_t row0, int wave, int lane) {
        from = static_cast<const char*>(s.p) + row0 * 4;
        stride = (uint32_t)s.stride;
        bytes = (s.pieces - 1) * s.stride + (s.rows - row0) * 4;
        offset = (uint32_t)(wave * kEach + lane / (kLong / 16)) * stride + (uint32_t)(lane % (kLong / 16)) * 16u;
    }
    __device__ __forceinline__ void load(int half, int at, char* lds, int wave) const {
        const int64_t gone = at * kKs * (int64_t)stride;
        const Stretch stage = stretch_of(from + gone, gone < bytes ? bytes - gone : 0);
        const uint32_t here = fresh(offset);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(stage, (__attribute__((address_space(3))) void*)(lds + half * kKs * kLong + (i * WAVES + wave) * 1024), 16,
                                                     here + ((uint32_t)(i * WAVES * kEach) * stride + (uint32_t)(half * kLong)), 0, 0, 0);
    }
};

// A transposing read: lane i of sixteen gets the i-th elements of four rows of sixteen that the lanes point to, a quarter of a row each.  (Of a pointer that nothing else
// is said to reach: otherwise the compiler waits for all loads into shared memory before it.)
typedef short FourShorts __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) FourShorts SharedFour;
__device__ __forceinline__ FourShorts read_across(SharedFour* __restrict__ p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }

// The eight k's of a lane's row that a matrix instruction takes.  `at`: where the lane's row (of the first block) starts in a stage's side, its first piece
// (lane_place); `on`: bytes from the first block to this one.
template <typename T> struct Fragment {
    Eight<T> x;
    template <int SB> __device__ __forceinline__ void load(const char* lds, uint32_t at, int on, int s) {
        x = *reinterpret_cast<const Eight<T>*>(lds + (at ^ (uint32_t)(32 * s)) + on);
    }
    // Of an operand that lies across, `block` 32 rows on.
    template <int LONG, int KS> __device__ __forceinline__ void load_across(const char* lds, uint32_t at, int half, int block, int s) {
        const int blocks = half * (LONG / 64) + block, second = blocks & 1, on = blocks / 2 * 8192;      // (LONG: bytes of a k of a half)
        typedef short Shorts __attribute__((ext_vector_type(8)));
        FourShorts part[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
            part[t] = read_across((SharedFour*)(lds + (at ^ (uint32_t)(64 * second)) + on + s * 2048 + t * 512));
        x = __builtin_bit_cast(Eight<T>, (Shorts)__builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
template <typename T, int SB> __device__ __forceinline__ uint32_t lane_place(int lane) {
    const int row = lane & 31, half = lane >> 5;
    return row * SB + place_of<SB>(row, sizeof(T) == 4 ? 2 * half : half) * 16;
}
// ... of an operand that lies across, LONG bytes of a k of a half of the tile, from row `wave0` of it on
template <typename T, int LONG> __device__ __forceinline__ uint32_t lane_place_across(int lane, int wave0) {
    if constexpr (sizeof(T) == 4) return (8 * (lane >> 5)) * LONG + (wave0 + (lane & 31)) * 4;
    const int in = lane & 15, group = lane >> 4;
    const uint32_t at = (8 * (group >> 1) + (in >> 2)) * 128 + ((in >> 3) & 1) * 64 + (group & 1) * 32 + (in & 3) * 8;
    return (at ^ (wave0 & 32) * 2u) + (wave0 >> 6) * 8192u;
}
template <> struct Fragment<f32> {
    typedef float Four __attribute__((ext_vector_type(4)));
    typedef float Floats __attribute__((ext_vector_type(8)));
    Four x[2];
    Eight<bf16> hi, mid, lo;
    template <int SB> __device__ __forceinline__ void load(const char* lds, uint32_t at, int on, int s) {
#pragma unroll
        for (int p = 0; p < 2; ++p) x[p] = *reinterpret_cast<const Four*>(lds + (at ^ (uint32_t)(64 * s + 16 * p)) + on);
    }
    template <int LONG, int KS> __device__ __forceinline__ void load_across(const char* lds, uint32_t at, int half, int block, int s) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e / 4][e % 4] = *reinterpret_cast<const float*>(lds + at + half * KS * LONG + (16 * s + e) * LONG + block * 128);
    }
    // Cut, not rounded: masks, subtractions and moves of bytes only, five and a half a number (with conversions the loop of 4096 x 1024 x 16384 took 743
    // us for 712).
    __device__ __forceinline__ void take_apart() {
        typedef uint32_t Words __attribute__((ext_vector_type(4)));
        Words w[3];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float a = x[e / 4][e % 4], b = x[e / 4][e % 4 + 1];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const uint32_t u = __float_as_uint(a), v = __float_as_uint(b);
                w[p][e / 2] = __builtin_amdgcn_perm(v, u, 0x07060302);          // the upper halves of both
                if (p == 2) break;
                a -= __uint_as_float(u & 0xffff0000u);
                b -= __uint_as_float(v & 0xffff0000u);
            }
        }
        hi = __builtin_bit_cast(Eight<bf16>, w[0]);
        mid = __builtin_bit_cast(Eight<bf16>, w[1]);
        lo = __builtin_bit_cast(Eight<bf16>, w[2]);
    }
};

// The products of a pair of fragments, by `first` and then `all`, which make one of them for all pairs.  fp32: into a sum of their own from the smallest ones on,
// which joins the others' in one addition.  By themselves the small ones are below half a step of a long sum and all of the sign of the terms, as the parts
// are cut: a sum over 4096 loses 5e-6 of itself then, and is 2.4e-7 off so (as by multiply-adds one after the other).  The additions cost: 4096 x 1024 x 16384
// 690 us without them, 812 so.
template <typename T, typename First, typename All> __device__ __forceinline__ void products(First&& first, All&& all) {
    typedef Fragment<T> F;
    if constexpr (std::is_same_v<T, f32>) {
        first([](const F& x, const F& y, Acc c) { return mma(x.lo, y.hi, c); });
        all([](const F& x, const F& y, Acc c) { return mma(x.hi, y.lo, c); });
        all([](const F& x, const F& y, Acc c) { return mma(x.mid, y.mid, c); });
        all([](const F& x, const F& y, Acc c) { return mma(x.mid, y.hi, c); });
        all([](const F& x, const F& y, Acc c) { return mma(x.hi, y.mid, c); });
        all([](const F& x, const F& y, Acc c) { return mma(x.hi, y.hi, c); });
    } else {
        first([](const F& x, const F& y, Acc c) { return mma(x.x, y.x, c); });
    }
}

// A tile of BM columns x BN rows of the result by WM x WN waves, S stages of SB bytes of k in shared memory; wave (wm, wn) has TM x TN blocks of 32 x 32 in
// registers.  Lane l of a block holds row l % 32 of the result and of it the columns 8 q + 4 (l / 32) + e as element 4 q + e, so that what is summed or
// looked for along a row stays within a lane but for the other half of the wave.
template <typename T, int BM, int BN, int WM, int WN, int S, int SB> struct Tile {
    static constexpr int kM = BM, kN = BN, kWavesM = WM, kWavesN = WN, kWaves = WM * WN, kThreads = 64 * kWaves, kStages = S, kStageBytes = SB;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    static constexpr int kParts = SB / (16 * sizeof(T));        // sixteen k's each
    static constexpr bool kQuarters = TM % 2 == 0 && TN % 2 == 0 && S == 2;
    static constexpr int kHalves = kQuarters ? 2 : 1, HA = TM / kHalves, HB = TN / kHalves;      // of the tile's columns and rows; blocks of a wave in each
    template <bool ACROSS> using LoadsA = std::conditional_t<ACROSS, StageAcross<BM, kHalves, kWaves, SB, sizeof(T)>, Stage<BM, kHalves, kWaves, SB>>;
    template <bool ACROSS> using LoadsB = std::conditional_t<ACROSS, StageAcross<BN, kHalves, kWaves, SB, sizeof(T)>, Stage<BN, kHalves, kWaves, SB>>;
    typedef T Element;
    struct Shared {                         // one stage
        char a[BM * SB], b[(sizeof(T) == 2 && BN < 64 ? 64 : BN) * SB];
    };
    static __device__ __forceinline__ int stages(const Operand& o) { return o.pieces > 0 ? (o.pieces * 16 + SB - 1) / SB : 1; }
    static __device__ __forceinline__ int stages_across(const Operand& o) { return (o.pieces + SB / (int)sizeof(T) - 1) / (SB / (int)sizeof(T)); }
    Acc acc[TM][TN];
    int wave, lane, wm, wn;
    uint32_t lane_along;
    __device__ __forceinline__ Tile() {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        wm = wave / WN;
        wn = wave % WN;
        lane_along = lane_place<T, SB>(lane);
    }
    // of the tile: a lane's first column of the i-th blocks (the others: + 8 q + e), its row of the j-th
    __device__ __forceinline__ int column(int i) const { return columns_from(i) + 4 * (lane >> 5); }
    __device__ __forceinline__ int row(int j) const { return rows_from(j) + (lane & 31); }
    // where a wave's i-th blocks of columns, its j-th of rows start
    __device__ __forceinline__ int columns_from(int i) const { return i / HA * (BM / kHalves) + (wm * HA + i % HA) * 32; }
    __device__ __forceinline__ int rows_from(int j) const { return j / HB * (BN / kHalves) + (wn * HB + j % HB) * 32; }

    // The tile's elements, times `scale`, as U: put(row, column, x), x sixteen bytes of a row of the tile, neighbouring lanes next to each other.  Through the
    // wave's own part of shared memory, which nothing else may be in: a lane's own elements are 8 or 16 bytes of 32 rows each, which costs a store of them as
    // many cycles (the product of 16 rows' adjoints into 131072 x 4096 bf16: 522 us so, 378 through shared memory).
    template <typename U> using Line = typename Pieces<U, 16 / sizeof(U)>::Vec;
    template <typename U, typename F> __device__ __forceinline__ void each_line(char* lds, float scale, F&& put) const {
        constexpr int N = 16 / sizeof(U), LINES = HA * 32 / N, LONG = LINES * 16, SAME = LONG < 256 ? 256 / LONG : 1;        // (SAME: rows in all banks)
        static_assert(32 * LONG * kWaves <= S * sizeof(Shared), "rows of a block fit");
        char* const mine = lds + wave * (32 * LONG);
        const auto place = [](int row, int line) { return row * LONG + (line ^ ((row / SAME) & (LINES - 1))) * 16; };
        const int to = lane & 31;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
#pragma unroll
                for (int i = 0; i < HA; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float x[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = acc[h * HA + i][j][4 * q + e] * scale;
                        const int at = 32 * i + 8 * q + 4 * (lane >> 5);
                        *reinterpret_cast<typename Pieces<U, 4>::Vec*>(mine + place(to, at / N) + at % N * sizeof(U)) = rounded<U, 4>(x);
                    }
                written();
#pragma unroll
                for (int k = 0; k < LINES / 2; ++k) {
                    const int row = (64 * k + lane) / LINES, line = lane % LINES;
                    put(rows_from(j) + row, columns_from(h * HA) + line * N, *reinterpret_cast<const Line<U>*>(mine + place(row, line)));
                }
                written();
            }
    }
    // (a wave's accesses to shared memory keep their order: the compiler must, too)
    static __device__ __forceinline__ void written() {
#ifdef __HIP_DEVICE_COMPILE__
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
#endif
    }

    static constexpr bool kApartSums = std::is_same_v<T, f32>;      // (products)
    // What a matrix instruction of each block takes: sixteen k's.
    struct Fragments {
        Fragment<T> a[TM], b[TN];
    };
    // The fragment of block `block` of a half of a side of ROWS rows; `at`: the lane's place in the wave's first block.
    template <bool ACROSS, int ROWS> __device__ __forceinline__ void fetch(Fragment<T>& f, const char* lds, uint32_t at, int half, int block, int s) const {
        if constexpr (ACROSS) f.template load_across<ROWS / kHalves * (int)sizeof(T), SB / (int)sizeof(T)>(lds, at, half, block, s);
        else f.template load<SB>(lds, at, (half * (ROWS / kHalves) + block * 32) * SB, s);
    }
    template <bool ACROSS, int ROWS> __device__ __forceinline__ uint32_t place(int wave0) const {
        if constexpr (ACROSS) return lane_place_across<T, ROWS / kHalves * (int)sizeof(T)>(lane, wave0);
        else return fresh(lane_along) + wave0 * SB;
    }
    template <bool AA, bool BA> __device__ __forceinline__ void fetch(Fragments& f, const Shared& sh, int s) const {
        const uint32_t a = place<AA, BM>(wm * HA * 32), b = place<BA, BN>(wn * HB * 32);
#pragma unroll
        for (int j = 0; j < TN; ++j) fetch<BA, BN>(f.b[j], sh.b, b, 0, j, s);
#pragma unroll
        for (int i = 0; i < TM; ++i) fetch<AA, BM>(f.a[i], sh.a, a, 0, i, s);
    }
    __device__ __forceinline__ void multiply(Fragments& f, Acc (&sum)[TM][TN], bool begins) {
        const auto all = [&](auto&& one) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) sum[i][j] = one(f.a[i], f.b[j], sum[i][j]);
        };
        const auto first = [&](auto&& one) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) sum[i][j] = one(f.a[i], f.b[j], begins ? Acc{} : sum[i][j]);
        };
        if constexpr (std::is_same_v<T, f32>) {
#pragma unroll
            for (int i = 0; i < TM; ++i) f.a[i].take_apart();
#pragma unroll
            for (int j = 0; j < TN; ++j) f.b[j].take_apart();
        }
        products<T>(first, all);
    }
    // Stages from .. to - 1 (one at least) of rows m0 .. of a and n0 .. of b (AA, BA: which of them lie across).  `meanwhile` is done while the first loads are on
    // their way.  Ends with a barrier: shared memory is free again.
    template <bool AA, bool BA, typename F> __device__ __forceinline__ void run(const Operand& oa, const Operand& ob, int64_t m0, int64_t n0, int from, int to, Shared (&sh)[S],
                                                              F&& meanwhile) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = Acc{};
        LoadsA<AA> la;
        LoadsB<BA> lb;
        la.init(oa, m0, wave, lane);
        lb.init(ob, n0, wave, lane);
        if constexpr (kQuarters) run_quarters<AA, BA>(la, lb, from, to, sh, meanwhile);
        else run_stages<AA, BA>(la, lb, from, to, sh, meanwhile);
        arrived<0>();
    }

    // All but the `left` youngest of this wave's loads have come, and its reads of shared memory; then those of all waves.
    template <int LEFT> static __device__ __forceinline__ void arrived() {
#ifdef __HIP_DEVICE_COMPILE__
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
#endif
    }

    // A stage at a time: stage s + S is asked for when all waves have left stage s.  (Stages behind the last one read zeros, so that always as many
    // loads are on their way.)
    template <bool AA, bool BA, typename F>
    __device__ __forceinline__ void run_stages(const LoadsA<AA>& la, const LoadsB<BA>& lb, int from, int to, Shared (&sh)[S], F&& meanwhile) {
        constexpr int kLoads = LoadsA<AA>::kLoads + LoadsB<BA>::kLoads;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            la.load(0, from + s, sh[s].a, wave);
            lb.load(0, from + s, sh[s].b, wave);
        }
        meanwhile();
        arrived<(S - 1) * kLoads>();
        for (int kt = from; kt < to; kt += S) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                Fragments f;
                Acc sum[TM][TN];                    // of the stage: as many roundings fewer in the long sum, and nothing waits for these
#pragma unroll
                for (int part = 0; part < kParts; ++part) {
                    fetch<AA, BA>(f, sh[s], part);
                    if (part == kParts - 1 && kt + s + 1 < to) {
                        arrived<(S > 1 ? S - 2 : 0) * kLoads>();
                        la.load(0, kt + s + S, sh[s].a, wave);
                        lb.load(0, kt + s + S, sh[s].b, wave);
                    }
                    multiply(f, sum, part == 0);
                }
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] += sum[i][j];
                if (kt + s + 1 >= to) break;
                if constexpr (S == 1) arrived<0>();
            }
        }
    }

    // A stage in four phases, a quarter of the blocks each: A0 B0, A0 B1, A1 B0, A1 B1, of halves of the wave's rows and columns.  A phase's fragments are in
    // registers when it begins; while its matrix instructions run, the half that a later phase needs is read: B1, A1, the next stage's A0, its B0.  A half that
    // all waves have read (the barrier behind each phase) is filled again at once, for the stage after next: seven phases before it is read, so that six
    // halves are on their way at every barrier and the loads never pause.  (Loading whole stages, one ahead: 3790 us for the loop of 4096 x 131072 x 4096.)
    struct HalfA { Fragment<T> x[HA][kParts]; };
    struct HalfB { Fragment<T> x[HB][kParts]; };
    template <bool ACROSS> __device__ __forceinline__ void fetch(HalfA& f, const Shared& sh, int half) const {
        const uint32_t at = place<ACROSS, BM>(wm * HA * 32);
#pragma unroll
        for (int i = 0; i < HA; ++i)
#pragma unroll
            for (int s = 0; s < kParts; ++s) fetch<ACROSS, BM>(f.x[i][s], sh.a, at, half, i, s);
    }
    template <bool ACROSS> __device__ __forceinline__ void fetch(HalfB& f, const Shared& sh, int half) const {
        const uint32_t at = place<ACROSS, BN>(wn * HB * 32);
#pragma unroll
        for (int j = 0; j < HB; ++j)
#pragma unroll
            for (int s = 0; s < kParts; ++s) fetch<ACROSS, BN>(f.x[j][s], sh.b, at, half, j, s);
    }
    template <typename Half> static __device__ __forceinline__ void take_apart(Half& f) {
        if constexpr (std::is_same_v<T, f32>)
            for (auto& row : f.x)
                for (auto& x : row) x.take_apart();
    }
    template <int FROM, int TO> __device__ __forceinline__ void multiply(const HalfA& a, const HalfB& b, int ha, int hb) {
        Acc sum[HA][HB];
        const auto at = [&](int i, int j) -> Acc& { return kApartSums ? sum[i][j] : acc[ha * HA + i][hb * HB + j]; };
#pragma unroll
        for (int s = FROM; s < TO; ++s) {
            const auto all = [&](auto&& one) {
#pragma unroll
                for (int i = 0; i < HA; ++i)
#pragma unroll
                    for (int j = 0; j < HB; ++j) at(i, j) = one(a.x[i][s], b.x[j][s], at(i, j));
            };
            const auto first = [&](auto&& one) {
#pragma unroll
                for (int i = 0; i < HA; ++i)
#pragma unroll
                    for (int j = 0; j < HB; ++j) at(i, j) = one(a.x[i][s], b.x[j][s], kApartSums && s == FROM ? Acc{} : at(i, j));
            };
            products<T>(first, all);
        }
        if constexpr (kApartSums) {
#pragma unroll
            for (int i = 0; i < HA; ++i)
#pragma unroll
                for (int j = 0; j < HB; ++j) acc[ha * HA + i][hb * HB + j] += sum[i][j];
        }
    }
    // One phase; `others` asks for the half that is free now and reads `next`, the one that is needed later.  fp32: which is taken apart between the matrix
    // instructions, at most kApart vector instructions behind each, while they run.
    static constexpr int kApart = 8;
    template <int LEFT, typename Half, typename F>
    __device__ __forceinline__ void phase(const HalfA& a, const HalfB& b, int ha, int hb, Half& next, F&& others) {
        if constexpr (std::is_same_v<T, f32>) {
            others();
            __builtin_amdgcn_sched_barrier(0);
            multiply<0, kParts>(a, b, ha, hb);
            take_apart(next);
#pragma unroll
            for (int m = 0; m < 6 * HA * HB * kParts; ++m) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x2, kApart, 0);
            }
        } else {
            multiply<0, 1>(a, b, ha, hb);                 // (the matrix cores have work at once)
            __builtin_amdgcn_sched_barrier(0);
            others();
            __builtin_amdgcn_sched_barrier(0);
            multiply<1, kParts>(a, b, ha, hb);
        }
        __builtin_amdgcn_sched_barrier(0);
        arrived<LEFT>();
    }
    template <bool AA, bool BA, typename F>
    __device__ __forceinline__ void run_quarters(const LoadsA<AA>& la, const LoadsB<BA>& lb, int from, int to, Shared (&sh)[S], F&& meanwhile) {
        constexpr int kLeft = 3 * (LoadsA<AA>::kLoads + LoadsB<BA>::kLoads);
        HalfA a0, a1;
        HalfB b0, b1;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            la.load(0, from + s, sh[s].a, wave);
            lb.load(0, from + s, sh[s].b, wave);
            lb.load(1, from + s, sh[s].b, wave);
            la.load(1, from + s, sh[s].a, wave);
        }
        meanwhile();
        arrived<kLeft>();
        fetch<AA>(a0, sh[0], 0);
        fetch<BA>(b0, sh[0], 0);
        arrived<kLeft>();
        take_apart(a0);
        take_apart(b0);
        la.load(0, from + 2, sh[0].a, wave);
        arrived<kLeft>();
        for (int kt = from; kt < to; kt += 2) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Shared &now = sh[s], &next = sh[s ^ 1];
                phase<kLeft>(a0, b0, 0, 0, b1, [&] {
                    lb.load(0, kt + s + 2, now.b, wave);
                    fetch<BA>(b1, now, 1);
                });
                phase<kLeft>(a0, b1, 0, 1, a1, [&] {
                    lb.load(1, kt + s + 2, now.b, wave);
                    fetch<AA>(a1, now, 1);
                });
                phase<kLeft>(a1, b0, 1, 0, a0, [&] {
                    la.load(1, kt + s + 2, now.a, wave);
                    fetch<AA>(a0, next, 0);
                });
                phase<kLeft>(a1, b1, 1, 1, b0, [&] {
                    la.load(0, kt + s + 3, next.a, wave);
                    fetch<BA>(b0, next, 0);
                });
                if (kt + s + 1 >= to) break;
            }
        }
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
    int64_t padded;                         // elements of a row of the copy; zeros behind what is taken
    int32_t finite;                         // 1: only what is finite is taken, zeros for the rest
    const float* bias;                      // of a row whose entry is -inf likewise; null: of none
};
__device__ __forceinline__ int64_t packed_row(const PackArgs& g, int64_t r) { return r / g.inner * g.outer + r % g.inner * g.inner_stride; }

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
        if (g.finite || (g.bias && g.bias[r] == -INFINITY)) {
#pragma unroll
            for (int e = 0; e < N; ++e) out[e] = fabsf((float)out[e]) < INFINITY ? out[e] : (T)0.0f;
        }
        *reinterpret_cast<typename Pieces<T, N>::Vec*>(static_cast<T*>(g.to) + r * g.padded + c) = out;
    }
}

}  // namespace klay
