// Gated recurrence over long sequences in the library's semirings, its reverse sweep and its single step:
//   h_t = a_t (x) h_{t-1} (+) x_t      REAL: a h + x    LOG: log(exp(a + h) + exp(x))    MAXLOG: max(a + h, x)
// A chain of T AND / OR gates, which as a circuit would be 2 T layers one after the other (paper Section 3.1).  The maps
// h -> a (x) h (+) x compose associatively, (A, H) after (A', H') = (A (x) A', A (x) H' (+) H), so the time axis is cut
// into pieces whose maps are found independently and then joined.
//
// Bound: memory.  A forward pass has to read a and x and write h once, a reverse sweep reads a, h (LOG: x too) and dh and writes two
// arrays.  A lane owns VC neighbouring channels.  A workgroup of W waves takes W * kSteps time steps at a time: every wave keeps its
// kSteps steps in registers, finds their map, the maps meet in LDS, and the wave goes through its steps again from the registers,
// so that memory is read once.  Where batch x channels give too few workgroups to fill the chip, the time axis is cut into chunks:
// a first launch finds the maps of the chunks, the second starts from the maps of the chunks before its own.
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

// What a row of the time axis is to its sequence.
enum : int { ROW_FIRST = 1, ROW_LAST = 2 };
constexpr int kDeadRow = -1;        // behind the last sequence (or before the first)

struct ScanArgs {
    const void *a, *x, *h, *dh;     // [batch, time, channels], channels contiguous, elements of type T
    void *out, *da, *dx;
    const float *initial, *dfinal;  // [sequences, channels] or null
    float *final, *dinitial;
    const int32_t* rows;            // packed: 4 * sequence + ROW_FIRST + ROW_LAST of every row, or kDeadRow; null: dense
    float *map_a, *map_h;           // [batch, chunks, channels]: maps of the chunks
    int32_t* map_cut;               // [batch, chunks]: the map does not depend on what comes in
    int64_t a_batch, a_time, x_batch, x_time;       // strides in elements; h, dh, out, da, dx are contiguous
    int64_t time;
    int32_t channels, chunks, chunk;    // chunk: time steps, a multiple of W * kSteps unless it is the only one
    int32_t blocks_c;                   // workgroups along the channels
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

// The workgroup's place: x = channels, then chunks, then the batch.
template <int VC>
__device__ __forceinline__ Place place_of(const ScanArgs& g, int32_t chunks, int32_t& chunk) {
    Place at;
    const uint32_t rest = blockIdx.x / (uint32_t)g.blocks_c;
    at.c = (int32_t)((blockIdx.x - rest * (uint32_t)g.blocks_c) * 64 + threadIdx.x) * VC;
    at.batch = (int32_t)(rest / (uint32_t)chunks);
    chunk = (int32_t)(rest - (uint32_t)at.batch * (uint32_t)chunks);
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

// The maps of the W waves of a tile.  Two sets in turn: a wave may write the next tile's while another still reads these.
template <int VC, int W> struct Maps {
    float a[2][W][64][VC], h[2][W][64][VC];
    int32_t cut[2][W];
    __device__ __forceinline__ void put(int turn, int wave, const float (&A)[VC], const float (&H)[VC], bool is_cut) {
        const int lane = threadIdx.x;
#pragma unroll
        for (int v = 0; v < VC; ++v) { a[turn][wave][lane][v] = A[v]; h[turn][wave][lane][v] = H[v]; }
        if (lane == 0) cut[turn][wave] = is_cut;
    }
    __device__ __forceinline__ uint64_t cuts(int turn) const {
        const int lane = threadIdx.x;
        return __ballot(lane < W && cut[turn][lane < W ? lane : 0] != 0);
    }
};

// The state that comes out of the chunks first .. first + count - 1 of a batch entry, taken in rising (BACK: falling) order, from
// nothing.  Every wave joins a part of their maps, eight loaded at a time; the parts meet in LDS, in set 1 of `maps`.
template <int S, int VC, int W, bool BACK>
__device__ __forceinline__ void state_of_chunks(float (&carry)[VC], Maps<VC, W>& maps, const ScanArgs& g, const Place& at, int32_t first, int32_t count) {
    constexpr int kAtOnce = 8;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y), lane = threadIdx.x;
#pragma unroll
    for (int v = 0; v < VC; ++v) carry[v] = Ring<S>::zero();
    if (count <= 0) return;
    const int32_t each = (count + W - 1) / W;
    const int32_t from = wave * each, to = from + each < count ? from + each : count;
    float A[VC], H[VC];
    bool cut = false;
#pragma unroll
    for (int v = 0; v < VC; ++v) { A[v] = Ring<S>::one; H[v] = Ring<S>::zero(); }
    for (int32_t n = from; n < to; n += kAtOnce) {
        float a[kAtOnce][VC], h[kAtOnce][VC];
        int32_t c[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int32_t i = n + j < to ? n + j : to - 1;          // (one past the part: again the last one, which is then not taken)
            const int64_t k = (int64_t)at.batch * g.chunks + first + (BACK ? count - 1 - i : i);
            load_elements<VC>(a[j], g.map_a + k * g.channels + at.lane);
            load_elements<VC>(h[j], g.map_h + k * g.channels + at.lane);
            c[j] = g.map_cut[k];
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (n + j >= to) break;
            cut |= c[j] != 0;
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                H[v] = c[j] ? h[j][v] : Ring<S>::step(a[j][v], H[v], h[j][v]);
                A[v] = Ring<S>::times(a[j][v], A[v]);
            }
        }
    }
    maps.put(1, wave, A, H, cut);
    lds_barrier();
    const uint64_t cuts = maps.cuts(1);
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
        for (int v = 0; v < VC; ++v)
            carry[v] = cuts >> w & 1 ? maps.h[1][w][lane][v] : Ring<S>::step(maps.a[1][w][lane][v], carry[v], maps.h[1][w][lane][v]);
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
    // the map of the steps, (A, H) before them; whether a sequence starts in them
    __device__ __forceinline__ bool map(float (&A)[VC], float (&H)[VC], const ScanArgs& g, const Place& at) const {
        return rows.plain() ? map_steps<true>(A, H, g, at) : map_steps<false>(A, H, g, at);
    }
    template <bool PLAIN> __device__ __forceinline__ bool map_steps(float (&A)[VC], float (&H)[VC], const ScanArgs& g, const Place& at) const {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (!PLAIN && (rows.first >> i & 1)) load_state<VC>(H, g.initial, rows.sequence(g, i), g, at, Ring<S>::zero());
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                const float av = piece<VC, T>(a[i], v);
                H[v] = Ring<S>::step(av, H[v], piece<VC, T>(x[i], v));
                A[v] = Ring<S>::times(av, A[v]);
            }
        }
        return !PLAIN && rows.first != 0;
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

// Maps of the chunks (those before the last one): every wave a run of its own, joined at the end.
template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_map_kernel(ScanArgs g) {
    __shared__ Maps<VC, W> maps;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y), lane = threadIdx.x;
    int32_t chunk;
    const Place at = place_of<VC>(g, g.chunks - 1, chunk);
    const int per_wave = g.chunk / W;
    const int64_t begin = (int64_t)chunk * g.chunk + (int64_t)wave * per_wave, end = begin + per_wave;
    float A[VC], H[VC];
    bool cut = false;
#pragma unroll
    for (int v = 0; v < VC; ++v) { A[v] = Ring<S>::one; H[v] = Ring<S>::zero(); }
    Tile<S, T, VC> next;
    next.load(g, begin, end, at);
    for (int64_t t = begin; t < end; t += kSteps) {
        Tile<S, T, VC> now = next;
        if (t + kSteps < end) next.load(g, t + kSteps, end, at);
        now.resolve(g, t, end);
        cut |= now.map(A, H, g, at);
    }
    maps.put(0, wave, A, H, cut);
    __syncthreads();
    if (wave != 0) return;
    const uint64_t cuts = maps.cuts(0);
    for (int w = 1; w < W; ++w)
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            H[v] = cuts >> w & 1 ? maps.h[0][w][lane][v] : Ring<S>::step(maps.a[0][w][lane][v], H[v], maps.h[0][w][lane][v]);
            A[v] = Ring<S>::times(maps.a[0][w][lane][v], A[v]);
        }
    const int64_t to = (int64_t)at.batch * g.chunks + chunk;
    if (at.in) {
        store_elements<VC>(g.map_a + to * g.channels + at.c, A);
        store_elements<VC>(g.map_h + to * g.channels + at.c, H);
    }
    if (at.c == 0) g.map_cut[to] = cuts != 0;
}

template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_kernel(ScanArgs g) {
    __shared__ Maps<VC, W> maps;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y), lane = threadIdx.x;
    int32_t chunk;
    const Place at = place_of<VC>(g, g.chunks, chunk);
    const int64_t begin = (int64_t)chunk * g.chunk, end = g.time < begin + g.chunk ? g.time : begin + g.chunk;
    Tile<S, T, VC> next;
    next.load(g, begin + wave * kSteps, end, at);
    float carry[VC];
    state_of_chunks<S, VC, W, false>(carry, maps, g, at, 0, chunk);
    int turn = 0;
    for (int64_t tile = begin; tile < end; tile += W * kSteps, turn ^= 1) {
        const int64_t t = tile + wave * kSteps;
        Tile<S, T, VC> now = next;
        if (tile + W * kSteps < end) next.load(g, t + W * kSteps, end, at);
        now.resolve(g, t, end);
        float A[VC], H[VC], h[VC];
#pragma unroll
        for (int v = 0; v < VC; ++v) { A[v] = Ring<S>::one; H[v] = Ring<S>::zero(); h[v] = carry[v]; }
        if constexpr (W > 1) {
            const bool cut = now.map(A, H, g, at);
            maps.put(turn, wave, A, H, cut);
            lds_barrier();
            const uint64_t cuts = maps.cuts(turn);
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int v = 0; v < VC; ++v) {
                    if (w == wave) h[v] = carry[v];
                    carry[v] = Ring<S>::step(maps.a[turn][w][lane][v], carry[v], maps.h[turn][w][lane][v]);
                    if (cuts != 0 && (cuts >> w & 1)) carry[v] = maps.h[turn][w][lane][v];
                }
        }
        if (now.rows.plain()) now.template walk<true>(h, g, t, end, at);
        else now.template walk<false>(h, g, t, end, at);
        if constexpr (W == 1)
#pragma unroll
            for (int v = 0; v < VC; ++v) carry[v] = h[v];
    }
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
    __device__ __forceinline__ bool map(float (&A)[VC], float (&C)[VC], const ScanArgs& g, const Place& at) const {
        return rows.plain() ? map_steps<true>(A, C, g, at) : map_steps<false>(A, C, g, at);
    }
    template <bool PLAIN> __device__ __forceinline__ bool map_steps(float (&A)[VC], float (&C)[VC], const ScanArgs& g, const Place& at) const {
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            if (!PLAIN && (rows.last >> i & 1)) load_state<VC>(C, g.dfinal, rows.sequence(g, i), g, at, 0.0f);
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                const float w = piece<VC, T>(a[i], v);
                C[v] = w * (piece<VC, T>(d[i], v) + C[v]);
                A[v] *= w;
            }
        }
        return !PLAIN && rows.last != 0;
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

// Maps of the chunks (those behind the first one), each from its last step to its first.
template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_back_map_kernel(ScanArgs g) {
    __shared__ Maps<VC, W> maps;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y), lane = threadIdx.x;
    int32_t chunk;
    const Place at = place_of<VC>(g, g.chunks - 1, chunk);
    ++chunk;
    const int per_wave = g.chunk / W;
    const int64_t begin = (int64_t)chunk * g.chunk + (int64_t)wave * per_wave;
    const int64_t end = g.time < begin + per_wave ? g.time : begin + per_wave;
    float A[VC], C[VC];
    bool cut = false;
#pragma unroll
    for (int v = 0; v < VC; ++v) { A[v] = 1.0f; C[v] = 0.0f; }
    if (begin < end) {
        int64_t t = begin + (end - 1 - begin) / kSteps * kSteps;
        BackTile<S, T, VC> next;
        next.load(g, t, end, at, S == SEMI_LOG);
        for (; t >= begin; t -= kSteps) {
            BackTile<S, T, VC> now = next;
            if (t - kSteps >= begin) next.load(g, t - kSteps, end, at, S == SEMI_LOG);
            now.resolve(g, t, end, at);
            cut |= now.map(A, C, g, at);
        }
    }
    maps.put(0, wave, A, C, cut);
    __syncthreads();
    if (wave != W - 1) return;
    const uint64_t cuts = maps.cuts(0);
    for (int w = W - 2; w >= 0; --w)
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            C[v] = cuts >> w & 1 ? maps.h[0][w][lane][v] : fmaf(maps.a[0][w][lane][v], C[v], maps.h[0][w][lane][v]);
            A[v] *= maps.a[0][w][lane][v];
        }
    const int64_t to = (int64_t)at.batch * g.chunks + chunk;
    if (at.in) {
        store_elements<VC>(g.map_a + to * g.channels + at.c, A);
        store_elements<VC>(g.map_h + to * g.channels + at.c, C);
    }
    if (at.c == 0) g.map_cut[to] = cuts != 0;
}

template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_back_kernel(ScanArgs g) {
    __shared__ Maps<VC, W> maps;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y), lane = threadIdx.x;
    int32_t chunk;
    const Place at = place_of<VC>(g, g.chunks, chunk);
    const int64_t begin = (int64_t)chunk * g.chunk, end = g.time < begin + g.chunk ? g.time : begin + g.chunk;
    const bool need_h = S == SEMI_LOG || g.da;
    const int64_t tiles = (end - begin + W * kSteps - 1) / (W * kSteps);
    BackTile<S, T, VC> next;
    next.load(g, begin + (tiles - 1) * (W * kSteps) + wave * kSteps, end, at, need_h);
    float carry[VC];
    state_of_chunks<SEMI_REAL, VC, W, true>(carry, maps, g, at, chunk + 1, g.chunks - 1 - chunk);
    int turn = 0;
    for (int64_t n = tiles - 1; n >= 0; --n, turn ^= 1) {
        const int64_t t = begin + n * (W * kSteps) + wave * kSteps;
        BackTile<S, T, VC> now = next;
        if (n > 0) next.load(g, t - W * kSteps, end, at, need_h);
        now.resolve(g, t, end, at);
        float A[VC], C[VC], c[VC];
#pragma unroll
        for (int v = 0; v < VC; ++v) { A[v] = 1.0f; C[v] = 0.0f; c[v] = carry[v]; }
        if constexpr (W > 1) {
            const bool cut = now.map(A, C, g, at);
            maps.put(turn, wave, A, C, cut);
            lds_barrier();
            const uint64_t cuts = maps.cuts(turn);
#pragma unroll
            for (int w = W - 1; w >= 0; --w)
#pragma unroll
                for (int v = 0; v < VC; ++v) {
                    if (w == wave) c[v] = carry[v];
                    carry[v] = fmaf(maps.a[turn][w][lane][v], carry[v], maps.h[turn][w][lane][v]);
                    if (cuts != 0 && (cuts >> w & 1)) carry[v] = maps.h[turn][w][lane][v];
                }
        }
        if (now.rows.plain()) now.template walk<true>(c, g, t, end, at);
        else now.template walk<false>(c, g, t, end, at);
        if constexpr (W == 1)
#pragma unroll
            for (int v = 0; v < VC; ++v) carry[v] = c[v];
    }
}

// ---- packed sequences: what each row is, and the states of sequences without rows -----------------------------------
// Thread n < rows: row n belongs to the first sequence s with offsets[s + 1] > n.  Offsets that are not what they should be (descending,
// past the rows, negative) give other results, never an access out of range: s is found in [0, sequences], and row 0 reads no row
// before it.
// Thread n < states_count: states[n] = from[n], or `none`: what the sequences without rows end with.
__global__ void __launch_bounds__(256) scan_rows_kernel(int32_t* rows, const int64_t* offsets, int64_t count, int32_t sequences, float* states,
                                                        const float* from, float none, int64_t states_count) {
    for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < count || n < states_count; n += (int64_t)gridDim.x * 256) {
        if (n < states_count) states[n] = from ? from[n] : none;
        if (n >= count) continue;
        int32_t lo = 0, hi = sequences;
        while (lo < hi) {
            const int32_t mid = lo + (hi - lo) / 2;
            if (offsets[mid + 1] > n) hi = mid;
            else lo = mid + 1;
        }
        int32_t r = kDeadRow;
        if (lo < sequences && offsets[lo] <= n)
            r = 4 * lo + (offsets[lo] == n || n == 0 ? ROW_FIRST : 0) + (offsets[lo + 1] == n + 1 ? ROW_LAST : 0);
        rows[n] = r;
    }
}

// states[i] = from[i], or `none`
__global__ void __launch_bounds__(256) scan_fill_kernel(float* states, const float* from, float none, int64_t count) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) states[i] = from ? from[i] : none;
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
