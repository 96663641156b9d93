// Gated recurrence over long sequences in the library's semirings, its reverse sweep and its single step:
//   h_t = a_t (x) h_{t-1} (+) x_t      REAL: a h + x    LOG: log(exp(a + h) + exp(x))    MAXLOG: max(a + h, x)
// A chain of T AND / OR gates, which as a circuit would be 2 T layers one after the other (paper Section 3.1).  The maps
// h -> a (x) h (+) x compose associatively, (A, H) after (A', H') = (A (x) A', A (x) H' (+) H), so the time axis is cut
// into pieces whose maps are found independently and then joined.
//
// Bound: memory.  A forward pass has to read a and x and write h once, a reverse sweep reads a, h (LOG: x too) and dh and writes two
// arrays.  A lane owns VC neighbouring channels.  A workgroup of W waves takes W * kSteps time steps at a time: every wave keeps its
// kSteps steps in registers, finds their map, the maps meet in LDS, and the wave goes through its steps again from the registers,
// so that memory is read once.  Where batch x channels give workgroups enough to fill the chip, one goes through all tiles of its channels.
// Otherwise every tile is a workgroup of its own (scan_chain_kernel), which publishes its map and takes the state in front of it from what
// the tiles before it have published.  (Two launches, the first of them for the maps alone, read the inputs twice: 65536 x 512 fp32
// forward 134 us, reverse 191 us, for 100 and 130.)
// Measured: 16 x 4096 x 4096 fp32 forward 563 us = 5.7 TB/s, reverse 1012 us = 5.3 TB/s (a copy of 1 GiB reaches 5.2 to 6.1); 8 x 4096 x 2048 bf16,
// a workgroup per CU, 93 us = 4.3 TB/s and 170 us = 4.0 TB/s; 65536 x 512 fp32, chained, 100 us and 130 us = 5.4 TB/s.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "klay_typed.hip.h"

namespace klay {

enum Semi : int { SEMI_REAL = 0, SEMI_LOG = 1, SEMI_MAX = 2 };

constexpr int kSteps = 16;          // time steps that a wave holds in registers
constexpr uint32_t kAllSteps = (1u << kSteps) - 1;
constexpr float kScanLog2e = 1.4426950408889634f, kScanLn2 = 0.6931471805599453f;

// log(exp(p) + exp(q)): the larger one plus log1p of a number in [0, 1].  u = 1 + e rounds away up to 2^-24 of e; the exact
// remainder e - (u - 1) comes back through the derivative 1 / u, so that a chain next to log 1 = 0 keeps its relative accuracy.
__device__ __forceinline__ float log_add(float p, float q) {
    const float top = fmaxf(p, q);
    const float e = __builtin_amdgcn_exp2f(p == q ? 0.0f : -fabsf(p - q) * kScanLog2e);   // (equal infinities have no difference)
    const float u = 1.0f + e;
    const float l = __builtin_amdgcn_logf(u) * kScanLn2;
    return top + fmaf(e - (u - 1.0f), __builtin_amdgcn_rcpf(u), l);
}

template <int S> struct Ring {
    static constexpr float one = S == SEMI_REAL ? 1.0f : 0.0f;
    static __device__ __forceinline__ float zero() { return S == SEMI_REAL ? 0.0f : -INFINITY; }
    static __device__ __forceinline__ float times(float a, float b) { return S == SEMI_REAL ? a * b : a + b; }
    static __device__ __forceinline__ float step(float a, float h, float x) {
        if constexpr (S == SEMI_REAL) return fmaf(a, h, x);
        if constexpr (S == SEMI_LOG) return log_add(a + h, x);
        const float y = a + h;
        return y > x || y != y ? y : x;      // a NaN passes on
    }
};

// A map's factor A may leave the range of its type where the states do not (gates above 1 behind a state of 0; a large state that falls by 2^-150 and
// rises again).  So in the real ring it is a * 2^e: for the steps of a wave e = 0 and a is A itself unless that is out of range, from
// there on 1/2 <= |a| < 1 or a = 0.  (The sums of a log-domain ring need no such thing.)
template <int S> __device__ __forceinline__ void times_scaled(float& a, int32_t& e, float by, int32_t by_e) {
    a = Ring<S>::times(by, a);
    if constexpr (S == SEMI_REAL) {
        e += by_e + __builtin_amdgcn_frexp_expf(a);
        a = __builtin_amdgcn_frexp_mantf(a);
    }
}
template <int S> __device__ __forceinline__ float step_scaled(float a, int32_t e, float h, float x) {
    if constexpr (S == SEMI_REAL) return __builtin_ldexpf(a * h, e) + x;
    return Ring<S>::step(a, h, x);
}
constexpr float kLeastFactor = 0x1p-100f;        // (with room above the smallest number for the products it goes into)

// What a row of the time axis is to its sequence.
enum : int { ROW_FIRST = 1, ROW_LAST = 2 };
constexpr int kDeadRow = -1;        // behind the last sequence (or before the first)

struct ScanArgs {
    const void *a, *x, *h, *dh;     // [batch, time, channels], channels contiguous, elements of type T
    void *out, *da, *dx;
    const float *initial, *dfinal;  // [sequences, channels] or null
    float *final, *dinitial;
    const int32_t* rows;            // packed: 4 * sequence + ROW_FIRST + ROW_LAST of every row, or kDeadRow; null: dense
    uint64_t *words, *state_words;  // chained: [chains, tiles, 2, 64 VC], [chains, groups of tiles, 64 VC], published; all 0 at the start
    uint32_t* ticket;               // chained: tiles that have been taken up; 0 at the start
    int64_t a_batch, a_time, x_batch, x_time;       // strides in elements; h, dh, out, da, dx are contiguous
    int64_t time;
    int32_t channels;
    int32_t blocks_c;               // workgroups along the channels
    int32_t chains, tiles;          // chained: workgroups along channels and batch, tiles of each
};

// The kSteps rows from t on, as a wave sees them: bit i = row t + i.
struct Rows {
    uint32_t first, last, live;
    int32_t info;           // packed, lane i: what row t + i is;  dense: the sequence
    __device__ __forceinline__ void load(const ScanArgs& g, int64_t t, int64_t end, int32_t batch) {
        info = batch;
        if (g.rows) {
            const int64_t r = t + (threadIdx.x & (kSteps - 1));
            info = g.rows[r < end ? r : end - 1];
        }
    }
    __device__ __forceinline__ void resolve(const ScanArgs& g, int64_t t, int64_t end) {
        const int64_t left = end - t;
        live = left >= kSteps ? kAllSteps : left > 0 ? (1u << left) - 1 : 0;
        if (g.rows) {
            first = (uint32_t)__ballot(info >= 0 && (info & ROW_FIRST)) & live;
            last = (uint32_t)__ballot(info >= 0 && (info & ROW_LAST)) & live;
            live &= (uint32_t)__ballot(info >= 0);
        } else {
            first = t == 0 ? 1u & live : 0;
            const int64_t behind = g.time - 1 - t;
            last = behind >= 0 && behind < kSteps ? (1u << behind) & live : 0;
        }
    }
    // all rows in the middle of one sequence: the waves' steps are straight-line code, in which loads of the tile behind stay in flight
    __device__ __forceinline__ bool plain() const { return live == kAllSteps && (first | last) == 0; }
    __device__ __forceinline__ int64_t sequence(const ScanArgs& g, int i) const {
        return g.rows ? __builtin_amdgcn_readlane(info, i) >> 2 : __builtin_amdgcn_readfirstlane(info);
    }
};

// Where a lane's channels are.
struct Place {
    int32_t batch, c;
    bool in;
    uint32_t lane;          // the first one, 0 past the channels
};

// The rows from t on of an array whose row 0 is at `base`.  Rows past `end` stand for the last one before it (they are not live, and
// what they load is not used).
template <int VC, typename T>
__device__ __forceinline__ void load_rows(Raw<T, VC> (&to)[kSteps], const T* base, int64_t stride, int64_t t, int64_t end, const Place& at) {
    const int64_t t0 = t < end ? t : end - 1;
    const uint32_t left = (uint32_t)(end - 1 - t0 < kSteps ? end - 1 - t0 : kSteps), bytes = (uint32_t)stride * sizeof(T);
    const Stretch from = stretch_at(base + t0 * stride);
    const uint32_t lane = at.in ? at.lane * (uint32_t)sizeof(T) : kNoLane;
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i) to[i] = load_raw<VC, T>(from, lane, (i < left ? i : left) * bytes);
}

template <int VC>
__device__ __forceinline__ void load_state(float (&h)[VC], const float* states, int64_t seq, const ScanArgs& g, const Place& at, float none) {
#pragma unroll
    for (int v = 0; v < VC; ++v) h[v] = none;
    if (states && at.in) load_elements<VC>(h, states + seq * g.channels + at.c);
}

// The place of chain number `chain`: channels, then the batch.
template <int VC>
__device__ __forceinline__ Place place_of(const ScanArgs& g, uint32_t chain) {
    Place at;
    const uint32_t batch = chain / (uint32_t)g.blocks_c;
    at.c = (int32_t)((chain - batch * (uint32_t)g.blocks_c) * 64 + threadIdx.x) * VC;
    at.batch = (int32_t)batch;
    at.in = at.c < g.channels;
    at.lane = at.in ? (uint32_t)at.c : 0;
    return at;
}

// A workgroup barrier for what the waves exchange in LDS: loads from memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The map of a wave's steps.
enum Kind : int32_t { PLAIN, CUT, SCALED };     // CUT: h does not depend on what comes in (a sequence starts in the steps);  SCALED: some e != 0
template <int VC> struct Map {
    float a[VC], h[VC], least[VC];              // least: the smallest |product| on the way to a
    int32_t e[VC];
    Kind kind;
    // From the product as it was multiplied: is it right?  If not, by mantissas and exponents.
    template <typename T>
    __device__ __forceinline__ void scale(const Raw<T, VC> (&gates)[kSteps]) {
        bool right = true;
#pragma unroll
        for (int v = 0; v < VC; ++v) right = right && least[v] >= kLeastFactor && fabsf(a[v]) < INFINITY;
        if (__ballot(!right) == 0) return;
        bool fits = true;
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            a[v] = 1.0f;
            e[v] = 0;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const float gate = piece<VC, T>(gates[i], v);
                a[v] *= __builtin_amdgcn_frexp_mantf(gate);
                e[v] += __builtin_amdgcn_frexp_expf(gate);
            }
            int32_t zero = 0;
            times_scaled<SEMI_REAL>(a[v], zero, 1.0f, 0);
            e[v] = a[v] == 0.0f ? 0 : e[v] + zero;
            fits = fits && e[v] > -100 && e[v] <= 128;
        }
        if (__ballot(!fits) == 0) {             // (gates of 0, most of the time)
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                a[v] = __builtin_ldexpf(a[v], e[v]);
                e[v] = 0;
            }
        } else {
            kind = SCALED;
        }
    }
};

// The maps of the W waves of a tile.  Two sets in turn: a wave may write the next tile's while another still reads these.
template <int VC, int W> struct Maps {
    float a[2][W][64][VC], h[2][W][64][VC];
    int32_t e[2][W][64][VC], kind[2][W];        // e is written and read where some map of the tile is SCALED
    __device__ __forceinline__ void put(int turn, int wave, const Map<VC>& m) {
        const int lane = threadIdx.x;
#pragma unroll
        for (int v = 0; v < VC; ++v) { a[turn][wave][lane][v] = m.a[v]; h[turn][wave][lane][v] = m.h[v]; }
        if (m.kind == SCALED)
#pragma unroll
            for (int v = 0; v < VC; ++v) e[turn][wave][lane][v] = m.e[v];
        if (lane == 0) kind[turn][wave] = m.kind;
    }
    // bit w: wave w's map is of that kind
    __device__ __forceinline__ uint64_t are(int turn, Kind which) const {
        const int lane = threadIdx.x;
        return __ballot(lane < W && kind[turn][lane < W ? lane : 0] == which);
    }
    // The state behind wave w's steps, from the one in front of them.
    template <int S>
    __device__ __forceinline__ void pass(float (&state)[VC], int turn, int w, uint64_t cuts, uint64_t scaled) const {
        const int lane = threadIdx.x;
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            const float A = a[turn][w][lane][v], H = h[turn][w][lane][v];
            const float h0 = state[v];
            state[v] = Ring<S>::step(A, h0, H);
            if ((cuts | scaled) != 0) {
                if (scaled >> w & 1) state[v] = step_scaled<S>(A, e[turn][w][lane][v], h0, H);
                if (cuts >> w & 1) state[v] = H;
            }
        }
    }
};

// ---- tiles that are workgroups of their own -----------------------------------------------------------------------
// The tiles of a chain come in groups of kGroup.  A tile publishes its map, joins the maps of the tiles before it in its group, and waits for the state
// in front of the group, which the last tile of the group before publishes: one wait after the other for every kGroup tiles.  Which
// maps are joined in which order depends on nothing but the tile's number, so the same inputs give the same bits.
// A published word is a value and a tag in one 64-bit store, and needs no other word to be ordered before or behind it.  Every wait ends: tiles are
// taken up by ticket, a tile waits only for words of tiles with lower tickets, whose workgroups are running then, and a workgroup
// publishes its map before it waits for anything.
constexpr int kGroup = 16;
// (tags: of an H, kMap, or kCut where it does not depend on what comes in; of an A, kMap + its exponent)
constexpr uint32_t kMap = 1u << 30, kCut = 2u << 30;
__device__ __forceinline__ void publish(uint64_t* word, float value, uint32_t tag) {
    __hip_atomic_store(word, (uint64_t)tag << 32 | __float_as_uint(value), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t published(const uint64_t* word) { return __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float value_of(uint64_t word) { return __uint_as_float((uint32_t)word); }
__device__ __forceinline__ uint32_t tag_of(uint64_t word) { return (uint32_t)(word >> 32); }

// A lane's words: H (word 0) and A (1) of tile number q of a chain, in the order in which the tiles follow each other; the state in front of a group.
template <int VC>
__device__ __forceinline__ uint64_t* map_word(const ScanArgs& g, uint32_t chain, int32_t q, int word) {
    return g.words + (((int64_t)chain * g.tiles + q) * 2 + word) * (64 * VC) + threadIdx.x * VC;
}
template <int VC>
__device__ __forceinline__ uint64_t* state_word(const ScanArgs& g, uint32_t chain, int32_t group) {
    return g.state_words + ((int64_t)chain * ((g.tiles + kGroup - 1) / kGroup) + group) * (64 * VC) + threadIdx.x * VC;
}

// Takes up the next tile: its chain, and its number in the chain's order.
__device__ __forceinline__ uint32_t take_tile(const ScanArgs& g, uint32_t* shared, int32_t& q) {
    if (threadIdx.x == 0 && threadIdx.y == 0) *shared = __hip_atomic_fetch_add(g.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const uint32_t ticket = __builtin_amdgcn_readfirstlane(*shared);
    q = (int32_t)(ticket / (uint32_t)g.chains);
    return ticket - (uint32_t)q * (uint32_t)g.chains;
}

// What the waves of a tile share besides their own maps: those of the tiles before it in the group, and the state in front of the tile.
template <int VC> struct Before {
    float a[kGroup - 1][64][VC], h[kGroup - 1][64][VC], state[64][VC];
    int32_t e[kGroup - 1][64][VC], cut[kGroup - 1];
    uint32_t ticket;
};

// The state in front of a wave's steps, from the maps of the tile's W waves (set 0), in rising (BACK: falling) order, and what is published of the
// chain.
template <int S, int VC, int W, bool BACK>
__device__ __forceinline__ void state_of_wave(float (&h)[VC], Maps<VC, W>& maps, Before<VC>& before, const ScanArgs& g, uint32_t chain, int32_t q) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y), lane = threadIdx.x;
    const int32_t group = q / kGroup, inside = q - group * kGroup;
    lds_barrier();
    const uint64_t cuts = maps.are(0, CUT), scaled = S == SEMI_REAL ? maps.are(0, SCALED) : 0;
    float A[VC], H[VC];                     // wave 0: the tile's map
    int32_t E[VC];
    if (wave == 0) {
#pragma unroll
        for (int v = 0; v < VC; ++v) { A[v] = Ring<S>::one; H[v] = Ring<S>::zero(); E[v] = 0; }
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const int w = BACK ? W - 1 - k : k;
            maps.template pass<S>(H, 0, w, cuts, scaled);
#pragma unroll
            for (int v = 0; v < VC; ++v) times_scaled<S>(A[v], E[v], maps.a[0][w][lane][v], scaled >> w & 1 ? maps.e[0][w][lane][v] : 0);
        }
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            publish(map_word<VC>(g, chain, q, 1) + v, A[v], kMap + (uint32_t)E[v]);
            publish(map_word<VC>(g, chain, q, 0) + v, H[v], cuts ? kCut : kMap);
        }
    }
    for (int32_t j = W - 1 - wave; j < inside; j += W) {          // (wave 0, which has published, last)
        uint64_t w0[VC], w1[VC];
        for (;;) {
            bool there = true;
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                w0[v] = published(map_word<VC>(g, chain, q - inside + j, 0) + v);
                w1[v] = published(map_word<VC>(g, chain, q - inside + j, 1) + v);
                there = there && tag_of(w0[v]) != 0 && tag_of(w1[v]) != 0;
            }
            if (__ballot(!there) == 0) break;
            __builtin_amdgcn_s_sleep(2);
        }
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            before.h[j][lane][v] = value_of(w0[v]);
            before.a[j][lane][v] = value_of(w1[v]);
            before.e[j][lane][v] = (int32_t)(tag_of(w1[v]) - kMap);
        }
        if (lane == 0) before.cut[j] = tag_of(w0[0]) == kCut;
    }
    lds_barrier();
    if (wave == 0) {
        const uint64_t cut_before = __ballot(lane < inside && before.cut[lane < inside ? lane : 0] != 0);
        float a[VC], b[VC];
        int32_t e[VC];
#pragma unroll
        for (int v = 0; v < VC; ++v) { a[v] = Ring<S>::one; b[v] = Ring<S>::zero(); e[v] = 0; }
#pragma unroll 5
        for (int32_t j = 0; j < inside; ++j)
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                const float aj = before.a[j][lane][v], hj = before.h[j][lane][v];
                const int32_t ej = before.e[j][lane][v];
                b[v] = cut_before >> j & 1 ? hj : step_scaled<S>(aj, ej, b[v], hj);
                times_scaled<S>(a[v], e[v], aj, ej);
            }
        if (cut_before == 0) {
            float front[VC];
#pragma unroll
            for (int v = 0; v < VC; ++v) front[v] = Ring<S>::zero();
            while (group > 0) {
                bool there = true;
#pragma unroll
                for (int v = 0; v < VC; ++v) {
                    const uint64_t w = published(state_word<VC>(g, chain, group) + v);
                    there = there && tag_of(w) != 0;
                    front[v] = value_of(w);
                }
                if (__ballot(!there) == 0) break;
                __builtin_amdgcn_s_sleep(1);
            }
#pragma unroll
            for (int v = 0; v < VC; ++v) b[v] = step_scaled<S>(a[v], e[v], front[v], b[v]);
        }
        if (inside == kGroup - 1 && q + 1 < g.tiles)
#pragma unroll
            for (int v = 0; v < VC; ++v) publish(state_word<VC>(g, chain, group + 1) + v, cuts ? H[v] : step_scaled<S>(A[v], E[v], b[v], H[v]), kMap);
#pragma unroll
        for (int v = 0; v < VC; ++v) before.state[lane][v] = b[v];
    }
    lds_barrier();
#pragma unroll
    for (int v = 0; v < VC; ++v) h[v] = before.state[lane][v];
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const int w = BACK ? W - 1 - k : k;
        if (BACK ? w <= wave : w >= wave) break;
        maps.template pass<S>(h, 0, w, cuts, scaled);
    }
}

// ---- forward ----------------------------------------------------------------------------------------------------
template <int S, typename T, int VC> struct Tile {
    Raw<T, VC> a[kSteps], x[kSteps];
    Rows rows;
    __device__ __forceinline__ void load(const ScanArgs& g, int64_t t, int64_t end, const Place& at) {
        rows.load(g, t, end, at.batch);
        load_rows<VC, T>(a, static_cast<const T*>(g.a) + at.batch * g.a_batch, g.a_time, t, end, at);
        load_rows<VC, T>(x, static_cast<const T*>(g.x) + at.batch * g.x_batch, g.x_time, t, end, at);
    }
    // rows that are not live become steps that change nothing
    __device__ __forceinline__ void resolve(const ScanArgs& g, int64_t t, int64_t end) {
        rows.resolve(g, t, end);
        if (rows.live == kAllSteps) return;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            if (!(rows.live >> i & 1)) {
                a[i] = all_pieces<VC, T>(Ring<S>::one);
                x[i] = all_pieces<VC, T>(Ring<S>::zero());
            }
    }
    __device__ __forceinline__ void map(Map<VC>& m, const ScanArgs& g, const Place& at) const {
        if (rows.plain()) map_steps<true>(m, g, at);
        else map_steps<false>(m, g, at);
        if (S == SEMI_REAL && m.kind != CUT) m.template scale<T>(a);
    }
    template <bool PLAIN> __device__ __forceinline__ void map_steps(Map<VC>& m, const ScanArgs& g, const Place& at) const {
        m.kind = !PLAIN && rows.first != 0 ? CUT : Kind::PLAIN;
#pragma unroll
        for (int v = 0; v < VC; ++v) { m.a[v] = Ring<S>::one; m.h[v] = Ring<S>::zero(); m.least[v] = INFINITY; m.e[v] = 0; }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (!PLAIN && (rows.first >> i & 1)) load_state<VC>(m.h, g.initial, rows.sequence(g, i), g, at, Ring<S>::zero());
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                const float av = piece<VC, T>(a[i], v);
                m.h[v] = Ring<S>::step(av, m.h[v], piece<VC, T>(x[i], v));
                m.a[v] = Ring<S>::times(av, m.a[v]);
                if constexpr (S == SEMI_REAL) m.least[v] = fminf(m.least[v], fabsf(m.a[v]));
            }
        }
    }
    // the steps themselves, from the state h
    template <bool PLAIN> __device__ __forceinline__ void walk(float (&h)[VC], const ScanArgs& g, int64_t t, int64_t end, const Place& at) const {
        const Stretch out = stretch_at(static_cast<T*>(g.out) + ((int64_t)at.batch * g.time + t) * g.channels);
        const uint32_t lane = at.in ? at.lane * (uint32_t)sizeof(T) : kNoLane, row = (uint32_t)g.channels * sizeof(T);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (!PLAIN && (rows.first >> i & 1)) load_state<VC>(h, g.initial, rows.sequence(g, i), g, at, Ring<S>::zero());
#pragma unroll
            for (int v = 0; v < VC; ++v) h[v] = Ring<S>::step(piece<VC, T>(a[i], v), h[v], piece<VC, T>(x[i], v));
            if (PLAIN || t + i < end) {
                float y[VC];
#pragma unroll
                for (int v = 0; v < VC; ++v) y[v] = PLAIN || (rows.live >> i & 1) ? h[v] : 0.0f;
                store_row<VC, T>(out, lane, i * row, y);
            }
            if (!PLAIN && g.final && (rows.last >> i & 1) && at.in)
                store_elements<VC>(g.final + rows.sequence(g, i) * g.channels + at.lane, h);
        }
    }
};

// A workgroup goes through all tiles of its channels.
template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_kernel(ScanArgs g) {
    __shared__ Maps<VC, W> maps;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const Place at = place_of<VC>(g, blockIdx.x);
    const int64_t end = g.time;
    Tile<S, T, VC> next;
    next.load(g, wave * kSteps, end, at);
    float carry[VC];
#pragma unroll
    for (int v = 0; v < VC; ++v) carry[v] = Ring<S>::zero();
    int turn = 0;
    for (int64_t tile = 0; tile < end; tile += W * kSteps, turn ^= 1) {
        const int64_t t = tile + wave * kSteps;
        Tile<S, T, VC> now = next;
        if (tile + W * kSteps < end) next.load(g, t + W * kSteps, end, at);
        now.resolve(g, t, end);
        float h[VC];
#pragma unroll
        for (int v = 0; v < VC; ++v) h[v] = carry[v];
        if constexpr (W > 1) {
            Map<VC> m;
            now.map(m, g, at);
            maps.put(turn, wave, m);
            lds_barrier();
            const uint64_t cuts = maps.are(turn, CUT), scaled = S == SEMI_REAL ? maps.are(turn, SCALED) : 0;
#pragma unroll
            for (int w = 0; w < W; ++w) {
#pragma unroll
                for (int v = 0; v < VC; ++v)
                    if (w == wave) h[v] = carry[v];
                maps.template pass<S>(carry, turn, w, cuts, scaled);
            }
        }
        if (now.rows.plain()) now.template walk<true>(h, g, t, end, at);
        else now.template walk<false>(h, g, t, end, at);
        if constexpr (W == 1)
#pragma unroll
            for (int v = 0; v < VC; ++v) carry[v] = h[v];
    }
}

// A tile a workgroup.
template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_chain_kernel(ScanArgs g) {
    __shared__ Maps<VC, W> maps;
    __shared__ Before<VC> before;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
    int32_t q;
    const uint32_t chain = take_tile(g, &before.ticket, q);
    const Place at = place_of<VC>(g, chain);
    const int64_t t = (int64_t)q * (W * kSteps) + wave * kSteps, end = g.time;
    Tile<S, T, VC> now;
    now.load(g, t, end, at);
    now.resolve(g, t, end);
    float h[VC];
    {
        Map<VC> m;
        now.map(m, g, at);
        maps.put(0, wave, m);
    }
    state_of_wave<S, VC, W, false>(h, maps, before, g, chain, q);
    if (now.rows.plain()) now.template walk<true>(h, g, t, end, at);
    else now.template walk<false>(h, g, t, end, at);
}

// ---- reverse sweep ------------------------------------------------------------------------------------------------
// c_t is the adjoint of the state that step t reads, g_t = dh_t + c_{t+1} that of h_t (c behind the last row: dfinal):
//   REAL: dx_t = g_t, da_t = g_t h_{t-1}, c_t = a_t g_t
//   LOG:  dx_t = g_t v_t, da_t = c_t = g_t w_t with the shares w = exp(a + h_{t-1} - h_t), v = exp(x - h_t) = 1 - w of the two
//         children, taken from the difference z = a + h_{t-1} - x, in which the rounding of h_t does not enter.  A step both of whose
//         children are impossible passes nothing down, as an OR gate of value log 0 does.
// Linear in c with the factors w (REAL: a): the same kind of map, joined from the last step to the first.
// REAL with 16-bit tensors takes h_{t-1} as the forward pass returned it: one rounding of up to 2^-8 (bf16) or 2^-11 (fp16) relative in
// da, which is rounded as much itself; keeping the states in 32 bits for it would cost 2 N C more bytes in each direction.
__device__ __forceinline__ void shares(float& w, float& v, float a, float h, float x) {
    const float p = a + h;
    const float z = p - x;
    const float e = __builtin_amdgcn_exp2f(-fabsf(z) * kScanLog2e);
    const float large = __builtin_amdgcn_rcpf(1.0f + e), small = e * large;
    w = z >= 0.0f ? large : small;
    v = z >= 0.0f ? small : large;
    if (p == x) w = v = p == -INFINITY ? 0.0f : 0.5f;
    if (z != z && p != x) w = v = z;
}

template <int S, typename T, int VC> struct BackTile {
    static constexpr bool kLog = S == SEMI_LOG;
    Raw<T, VC> a[kSteps], d[kSteps], h[kSteps], x[kLog ? kSteps : 1];      // h: the states before the steps;  LOG, resolved: a = w, x = v
    Rows rows;
    // gates_too: h is needed (LOG: for the shares)
    __device__ __forceinline__ void load(const ScanArgs& g, int64_t t, int64_t end, const Place& at, bool need_h) {
        rows.load(g, t, end, at.batch);
        const int64_t states = (int64_t)at.batch * g.time * g.channels;
        load_rows<VC, T>(a, static_cast<const T*>(g.a) + at.batch * g.a_batch, g.a_time, t, end, at);
        if (g.dh) load_rows<VC, T>(d, static_cast<const T*>(g.dh) + states, g.channels, t, end, at);
        if constexpr (kLog) load_rows<VC, T>(x, static_cast<const T*>(g.x) + at.batch * g.x_batch, g.x_time, t, end, at);
        if (need_h) {
            // rows t - 1 ..;  row 0 starts a sequence: what is loaded for it is not used
            const int64_t t0 = t < end ? t : end - 1;
            const uint32_t left = (uint32_t)(end - 1 - t0 < kSteps ? end - 1 - t0 : kSteps), bytes = (uint32_t)g.channels * sizeof(T);
            const uint32_t back = t0 > 0 ? 1 : 0, lane = at.in ? at.lane * (uint32_t)sizeof(T) : kNoLane;
            const Stretch from = stretch_at(static_cast<const T*>(g.h) + states + (t0 - back) * g.channels);
#pragma unroll
            for (uint32_t i = 0; i < kSteps; ++i) {
                const uint32_t row = (i < left ? i : left) + back;
                h[i] = load_raw<VC, T>(from, lane, (row > 0 ? row - 1 : 0) * bytes);
            }
        }
    }
    __device__ __forceinline__ void resolve(const ScanArgs& g, int64_t t, int64_t end, const Place& at) {
        rows.resolve(g, t, end);
        if (!g.dh) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) d[i] = all_pieces<VC, T>(0.0f);
        }
        if (kLog && !rows.plain()) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                if (rows.first >> i & 1) {
                    float before[VC];
                    load_state<VC>(before, g.initial, rows.sequence(g, i), g, at, Ring<S>::zero());
                    h[i] = all_pieces<VC, T>(before[0]);
                }
        }
        if constexpr (kLog) {
            static_assert(VC == 1, "the log-domain semirings take one channel a lane");
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                float w, v;
                shares(w, v, a[i], h[i], x[i]);
                a[i] = w;
                x[i] = v;
            }
        }
        if (rows.live != kAllSteps) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                if (!(rows.live >> i & 1)) {
                    a[i] = all_pieces<VC, T>(1.0f);
                    d[i] = all_pieces<VC, T>(0.0f);
                }
        }
    }
    __device__ __forceinline__ void map(Map<VC>& m, const ScanArgs& g, const Place& at) const {
        if (rows.plain()) map_steps<true>(m, g, at);
        else map_steps<false>(m, g, at);
        if (m.kind != CUT) m.template scale<T>(a);
    }
    template <bool PLAIN> __device__ __forceinline__ void map_steps(Map<VC>& m, const ScanArgs& g, const Place& at) const {
        m.kind = !PLAIN && rows.last != 0 ? CUT : Kind::PLAIN;
#pragma unroll
        for (int v = 0; v < VC; ++v) { m.a[v] = 1.0f; m.h[v] = 0.0f; m.least[v] = INFINITY; m.e[v] = 0; }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            if (!PLAIN && (rows.last >> i & 1)) load_state<VC>(m.h, g.dfinal, rows.sequence(g, i), g, at, 0.0f);
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                const float w = piece<VC, T>(a[i], v);
                m.h[v] = w * (piece<VC, T>(d[i], v) + m.h[v]);
                m.a[v] *= w;
                m.least[v] = fminf(m.least[v], fabsf(m.a[v]));
            }
        }
    }
    // the steps themselves, from the last to the first, from the adjoint c of the state behind them
    template <bool PLAIN> __device__ __forceinline__ void walk(float (&c)[VC], const ScanArgs& g, int64_t t, int64_t end, const Place& at) const {
        const int64_t to = ((int64_t)at.batch * g.time + t) * g.channels;
        const Stretch da = stretch_at(static_cast<T*>(g.da) + to), dx = stretch_at(static_cast<T*>(g.dx) + to);
        const uint32_t lane = at.in ? at.lane * (uint32_t)sizeof(T) : kNoLane, row = (uint32_t)g.channels * sizeof(T);
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            if (!PLAIN && (rows.last >> i & 1)) load_state<VC>(c, g.dfinal, rows.sequence(g, i), g, at, 0.0f);
            float ya[VC], yx[VC], before[VC];
            const bool live = PLAIN || (rows.live >> i & 1);
            if constexpr (!kLog) {
#pragma unroll
                for (int v = 0; v < VC; ++v) before[v] = piece<VC, T>(h[i], v);
                if (!PLAIN && (rows.first >> i & 1)) load_state<VC>(before, g.initial, rows.sequence(g, i), g, at, Ring<S>::zero());
            }
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                const float gt = piece<VC, T>(d[i], v) + c[v];
                c[v] = piece<VC, T>(a[i], v) * gt;
                if constexpr (!kLog) {
                    ya[v] = live ? gt * before[v] : 0.0f;
                    yx[v] = live ? gt : 0.0f;
                } else {
                    ya[v] = live ? c[v] : 0.0f;
                    yx[v] = live ? gt * piece<VC, T>(x[i], v) : 0.0f;
                }
            }
            if (PLAIN || t + i < end) {
                if (g.da) store_row<VC, T>(da, lane, i * row, ya);
                if (g.dx) store_row<VC, T>(dx, lane, i * row, yx);
            }
            if (!PLAIN && g.dinitial && (rows.first >> i & 1) && at.in)
                store_elements<VC>(g.dinitial + rows.sequence(g, i) * g.channels + at.lane, c);
        }
    }
};

template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_back_kernel(ScanArgs g) {
    __shared__ Maps<VC, W> maps;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const Place at = place_of<VC>(g, blockIdx.x);
    const int64_t end = g.time;
    const bool need_h = S == SEMI_LOG || g.da;
    const int64_t tiles = (end + W * kSteps - 1) / (W * kSteps);
    BackTile<S, T, VC> next;
    next.load(g, (tiles - 1) * (W * kSteps) + wave * kSteps, end, at, need_h);
    float carry[VC];
#pragma unroll
    for (int v = 0; v < VC; ++v) carry[v] = 0.0f;
    int turn = 0;
    for (int64_t n = tiles - 1; n >= 0; --n, turn ^= 1) {
        const int64_t t = n * (W * kSteps) + wave * kSteps;
        BackTile<S, T, VC> now = next;
        if (n > 0) next.load(g, t - W * kSteps, end, at, need_h);
        now.resolve(g, t, end, at);
        float c[VC];
#pragma unroll
        for (int v = 0; v < VC; ++v) c[v] = carry[v];
        if constexpr (W > 1) {
            Map<VC> m;
            now.map(m, g, at);
            maps.put(turn, wave, m);
            lds_barrier();
            const uint64_t cuts = maps.are(turn, CUT), scaled = maps.are(turn, SCALED);
#pragma unroll
            for (int w = W - 1; w >= 0; --w) {
#pragma unroll
                for (int v = 0; v < VC; ++v)
                    if (w == wave) c[v] = carry[v];
                maps.template pass<SEMI_REAL>(carry, turn, w, cuts, scaled);
            }
        }
        if (now.rows.plain()) now.template walk<true>(c, g, t, end, at);
        else now.template walk<false>(c, g, t, end, at);
        if constexpr (W == 1)
#pragma unroll
            for (int v = 0; v < VC; ++v) carry[v] = c[v];
    }
}

template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(4))) scan_back_chain_kernel(ScanArgs g) {
    __shared__ Maps<VC, W> maps;
    __shared__ Before<VC> before;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
    int32_t q;
    const uint32_t chain = take_tile(g, &before.ticket, q);
    const Place at = place_of<VC>(g, chain);
    const int64_t t = (int64_t)(g.tiles - 1 - q) * (W * kSteps) + wave * kSteps, end = g.time;
    BackTile<S, T, VC> now;
    now.load(g, t, end, at, S == SEMI_LOG || g.da);
    now.resolve(g, t, end, at);
    float c[VC];
    {
        Map<VC> m;
        now.map(m, g, at);
        maps.put(0, wave, m);
    }
    state_of_wave<SEMI_REAL, VC, W, true>(c, maps, before, g, chain, q);
    if (now.rows.plain()) now.template walk<true>(c, g, t, end, at);
    else now.template walk<false>(c, g, t, end, at);
}

// ---- packed sequences: what each row is, and the states of sequences without rows -----------------------------------
// Thread n < rows: row n belongs to the first sequence s with offsets[s + 1] > n.  Offsets that are not what they should be (descending,
// past the rows, negative) give other results, never an access out of range: s is found in [0, sequences], and row 0 reads no row
// before it.
struct PrepareArgs {
    int32_t* rows;                  // [count], of the packed sequences of `offsets`
    const int64_t* offsets;
    int64_t count;
    int32_t sequences;
    float none;
    float* states;                  // [states_count] = from, or `none`: what the sequences without rows end with
    const float* from;
    int64_t states_count;
    uint64_t* words;                // [words_count] = 0
    int64_t words_count;
};
__global__ void __launch_bounds__(256) scan_prepare_kernel(PrepareArgs g) {
    const int64_t all = g.count > g.states_count ? g.count : g.states_count;
    for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < all || n < g.words_count; n += (int64_t)gridDim.x * 256) {
        if (n < g.words_count) g.words[n] = 0;
        if (n < g.states_count) g.states[n] = g.from ? g.from[n] : g.none;
        if (n >= g.count) continue;
        int32_t lo = 0, hi = g.sequences;
        while (lo < hi) {
            const int32_t mid = lo + (hi - lo) / 2;
            if (g.offsets[mid + 1] > n) hi = mid;
            else lo = mid + 1;
        }
        int32_t r = kDeadRow;
        if (lo < g.sequences && g.offsets[lo] <= n)
            r = 4 * lo + (g.offsets[lo] == n || n == 0 ? ROW_FIRST : 0) + (g.offsets[lo + 1] == n + 1 ? ROW_LAST : 0);
        g.rows[n] = r;
    }
}

// ---- one step -----------------------------------------------------------------------------------------------------
struct StepArgs {
    const void *a, *x;
    void* out;
    float* state;
    int64_t a_row, x_row, out_row, state_row;
    int32_t batch, channels;
};

// grid: x over the channels, y over the batch (in strides of the grid)
template <int S, typename T, int VC>
__global__ void __launch_bounds__(256) step_kernel(StepArgs g) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VC;
    if (c >= g.channels) return;
    for (int64_t b = blockIdx.y; b < g.batch; b += gridDim.y) {
        float a[VC], x[VC], h[VC];
        load_elements<VC>(a, static_cast<const T*>(g.a) + b * g.a_row + c);
        load_elements<VC>(x, static_cast<const T*>(g.x) + b * g.x_row + c);
        float* state = g.state + b * g.state_row + c;
        load_elements<VC>(h, state);
#pragma unroll
        for (int v = 0; v < VC; ++v) h[v] = Ring<S>::step(a[v], h[v], x[v]);
        store_elements<VC>(state, h);
        if (g.out) store_elements<VC>(static_cast<T*>(g.out) + b * g.out_row + c, h);
    }
}

}  // namespace klay
