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
    int32_t seq;            // lane i: sequence of row t + i
    __device__ __forceinline__ Rows(const ScanArgs& g, int64_t t, int64_t end, int batch) {
        const int lane = threadIdx.x;
        int32_t r = kDeadRow;
        if (lane < kSteps && t + lane < end) {
            if (g.rows) r = g.rows[t + lane];
            else r = 4 * batch + (t + lane == 0 ? ROW_FIRST : 0) + (t + lane == g.time - 1 ? ROW_LAST : 0);
        }
        seq = r >> 2;
        live = (uint32_t)__ballot(r >= 0);
        first = (uint32_t)__ballot(r >= 0 && (r & ROW_FIRST));
        last = (uint32_t)__ballot(r >= 0 && (r & ROW_LAST));
    }
    __device__ __forceinline__ int64_t sequence(int i) const { return __builtin_amdgcn_readlane(seq, i); }
};

template <int VC>
__device__ __forceinline__ void load_state(float (&h)[VC], const float* states, int64_t seq, const ScanArgs& g, int c, bool in, float none) {
#pragma unroll
    for (int v = 0; v < VC; ++v) h[v] = none;
    if (states && in) load_elements<VC>(h, states + seq * g.channels + c);
}

// ---- forward ----------------------------------------------------------------------------------------------------
template <int S, typename T, int VC>
__device__ __forceinline__ void load_steps(float (&a)[kSteps][VC], float (&x)[kSteps][VC], const ScanArgs& g, int64_t batch, int64_t t,
                                           int c, bool in, uint32_t live) {
    const int cs = in ? c : 0;          // lanes past the channels read channel 0: no branch around the loads
    const T* pa = static_cast<const T*>(g.a) + batch * g.a_batch + t * g.a_time + cs;
    const T* px = static_cast<const T*>(g.x) + batch * g.x_batch + t * g.x_time + cs;
    if (live == kAllSteps) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            load_elements<VC>(a[i], pa + i * g.a_time);
            load_elements<VC>(x[i], px + i * g.x_time);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
#pragma unroll
        for (int v = 0; v < VC; ++v) { a[i][v] = Ring<S>::one; x[i][v] = Ring<S>::zero(); }
        if (live >> i & 1) {
            load_elements<VC>(a[i], pa + i * g.a_time);
            load_elements<VC>(x[i], px + i * g.x_time);
        }
    }
}

// The map of the steps in registers: (A, H), and whether a sequence starts in them.
template <int S, int VC>
__device__ __forceinline__ bool map_of(float (&A)[VC], float (&H)[VC], const float (&a)[kSteps][VC], const float (&x)[kSteps][VC],
                                       const Rows& rows, const ScanArgs& g, int c, bool in) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (rows.first >> i & 1) load_state<VC>(H, g.initial, rows.sequence(i), g, c, in, Ring<S>::zero());
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            H[v] = Ring<S>::step(a[i][v], H[v], x[i][v]);
            A[v] = Ring<S>::times(a[i][v], A[v]);
        }
    }
    return rows.first != 0;
}

// Maps of the chunks (those before the last one): every wave a run of its own, joined at the end.
template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_map_kernel(ScanArgs g) {
    __shared__ float sa[W][64][VC], sh[W][64][VC];
    __shared__ int scut[W];
    const int lane = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const int bc = blockIdx.x % g.blocks_c;
    const int64_t rest = blockIdx.x / g.blocks_c;
    const int chunk = (int)(rest % (g.chunks - 1));
    const int64_t batch = rest / (g.chunks - 1);
    const int c = (bc * 64 + lane) * VC;
    const bool in = c < g.channels;
    const int per_wave = g.chunk / W;
    const int64_t begin = (int64_t)chunk * g.chunk + (int64_t)wave * per_wave, end = begin + per_wave;
    float A[VC], H[VC];
    bool cut = false;
#pragma unroll
    for (int v = 0; v < VC; ++v) { A[v] = Ring<S>::one; H[v] = Ring<S>::zero(); }
    for (int64_t t = begin; t < end; t += kSteps) {
        float a[kSteps][VC], x[kSteps][VC];
        const Rows rows(g, t, end, (int)batch);
        load_steps<S, T, VC>(a, x, g, batch, t, c, in, rows.live);
        cut |= map_of<S, VC>(A, H, a, x, rows, g, c, in);
    }
#pragma unroll
    for (int v = 0; v < VC; ++v) { sa[wave][lane][v] = A[v]; sh[wave][lane][v] = H[v]; }
    if (lane == 0) scut[wave] = cut;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < W; ++w) {
        const bool wcut = scut[w];
        cut |= wcut;
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            H[v] = wcut ? sh[w][lane][v] : Ring<S>::step(sa[w][lane][v], H[v], sh[w][lane][v]);
            A[v] = Ring<S>::times(sa[w][lane][v], A[v]);
        }
    }
    const int64_t at = batch * g.chunks + chunk;
    if (in) {
        store_elements<VC>(g.map_a + at * g.channels + c, A);
        store_elements<VC>(g.map_h + at * g.channels + c, H);
    }
    if (bc == 0 && lane == 0) g.map_cut[at] = cut;
}

template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_kernel(ScanArgs g) {
    __shared__ float sa[2][W][64][VC], sh[2][W][64][VC];
    __shared__ int scut[2][W];
    const int lane = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const int bc = blockIdx.x % g.blocks_c;
    const int64_t rest = blockIdx.x / g.blocks_c;
    const int chunk = (int)(rest % g.chunks);
    const int64_t batch = rest / g.chunks;
    const int c = (bc * 64 + lane) * VC;
    const bool in = c < g.channels;
    float carry[VC];
#pragma unroll
    for (int v = 0; v < VC; ++v) carry[v] = Ring<S>::zero();
    for (int k = 0; k < chunk; ++k) {
        const int64_t at = batch * g.chunks + k;
        float A[VC] = {}, H[VC] = {};
        if (in) {
            load_elements<VC>(A, g.map_a + at * g.channels + c);
            load_elements<VC>(H, g.map_h + at * g.channels + c);
        }
        const bool cut = g.map_cut[at];
#pragma unroll
        for (int v = 0; v < VC; ++v) carry[v] = cut ? H[v] : Ring<S>::step(A[v], carry[v], H[v]);
    }
    const int64_t begin = (int64_t)chunk * g.chunk, end = g.time < begin + g.chunk ? g.time : begin + g.chunk;
    int turn = 0;
    for (int64_t tile = begin; tile < end; tile += W * kSteps, turn ^= 1) {
        const int64_t t = tile + wave * kSteps;
        float a[kSteps][VC], x[kSteps][VC], A[VC], H[VC];
        const Rows rows(g, t, end, (int)batch);
        load_steps<S, T, VC>(a, x, g, batch, t, c, in, rows.live);
#pragma unroll
        for (int v = 0; v < VC; ++v) { A[v] = Ring<S>::one; H[v] = Ring<S>::zero(); }
        const bool cut = map_of<S, VC>(A, H, a, x, rows, g, c, in);
        // two sets of maps in turn: a wave may write the next tile's while another still reads these
#pragma unroll
        for (int v = 0; v < VC; ++v) { sa[turn][wave][lane][v] = A[v]; sh[turn][wave][lane][v] = H[v]; }
        if (lane == 0) scut[turn][wave] = cut;
        __syncthreads();
        float h[VC];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const bool wcut = scut[turn][w];
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                if (w == wave) h[v] = carry[v];
                carry[v] = wcut ? sh[turn][w][lane][v] : Ring<S>::step(sa[turn][w][lane][v], carry[v], sh[turn][w][lane][v]);
            }
        }
        T* out = static_cast<T*>(g.out) + (batch * g.time + t) * g.channels + c;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (rows.first >> i & 1) load_state<VC>(h, g.initial, rows.sequence(i), g, c, in, Ring<S>::zero());
#pragma unroll
            for (int v = 0; v < VC; ++v) h[v] = Ring<S>::step(a[i][v], h[v], x[i][v]);
            if (t + i < end && in) {
                const bool live = rows.live >> i & 1;
                float y[VC];
#pragma unroll
                for (int v = 0; v < VC; ++v) y[v] = live ? h[v] : 0.0f;
                store_elements<VC>(out + (int64_t)i * g.channels, y);
                if (g.final && (rows.last >> i & 1)) store_elements<VC>(g.final + rows.sequence(i) * g.channels + c, h);
            }
        }
    }
}

// ---- reverse sweep ------------------------------------------------------------------------------------------------
// c_t is the adjoint of the state that step t reads, g_t = dh_t + c_{t+1} that of h_t (c behind the last row: dfinal):
//   REAL: dx_t = g_t, da_t = g_t h_{t-1}, c_t = a_t g_t
//   LOG:  dx_t = g_t v_t, da_t = c_t = g_t w_t with the shares w = exp(a + h_{t-1} - h_t), v = exp(x - h_t) = 1 - w of the two
//         children, taken from the difference z = a + h_{t-1} - x, in which the rounding of h_t does not enter.  A step both of whose
//         children are impossible passes nothing down, as an OR gate of value log 0 does.
// Linear in c with the factors w (REAL: a): the same kind of map, joined from the last step to the first.
// REAL with 16-bit tensors takes h_{t-1} as the forward pass returned it: one rounding of up to 2^-8 (bf16) or 2^-11 (fp16) relative in da,
// which is rounded as much itself; keeping the states in 32 bits for it would cost 2 N C more bytes in each direction.
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

// a, w: factors of the steps; b: h_{t-1} (REAL), shares of x (LOG); d: dh
template <int S, typename T, int VC>
__device__ __forceinline__ void load_steps_back(float (&w)[kSteps][VC], float (&b)[kSteps][VC], float (&d)[kSteps][VC], const ScanArgs& g,
                                                int64_t batch, int64_t t, int c, bool in, const Rows& rows, bool need_b) {
    const int cs = in ? c : 0;
    const T* pa = static_cast<const T*>(g.a) + batch * g.a_batch + t * g.a_time + cs;
    const T* px = static_cast<const T*>(g.x) + batch * g.x_batch + t * g.x_time + cs;
    const int64_t at = (batch * g.time + t) * g.channels + cs;
    const T* ph = static_cast<const T*>(g.h) + at;
    const T* pd = static_cast<const T*>(g.dh) + at;
    float x[S == SEMI_LOG ? kSteps : 1][VC];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const bool live = rows.live >> i & 1;
#pragma unroll
        for (int v = 0; v < VC; ++v) { w[i][v] = S == SEMI_REAL ? 1.0f : 0.0f; b[i][v] = 0.0f; d[i][v] = 0.0f; }
        if (live) {
            load_elements<VC>(w[i], pa + i * g.a_time);
            if (g.dh) load_elements<VC>(d[i], pd + (int64_t)i * g.channels);
            if constexpr (S == SEMI_LOG) load_elements<VC>(x[i], px + i * g.x_time);
        }
        if (need_b) {
            if (rows.first >> i & 1) load_state<VC>(b[i], g.initial, rows.sequence(i), g, c, in, Ring<S>::zero());
            else if (live) load_elements<VC>(b[i], ph + (int64_t)(i - 1) * g.channels);
        }
    }
    if constexpr (S == SEMI_LOG) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool live = rows.live >> i & 1;
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                float ws = 1.0f, vs = 0.0f;
                if (live) shares(ws, vs, w[i][v], b[i][v], x[i][v]);
                w[i][v] = ws;
                b[i][v] = vs;
            }
        }
    }
}

template <int VC>
__device__ __forceinline__ bool map_of_back(float (&A)[VC], float (&C)[VC], const float (&w)[kSteps][VC], const float (&d)[kSteps][VC],
                                            const Rows& rows, const ScanArgs& g, int c, bool in) {
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
        if (rows.last >> i & 1) load_state<VC>(C, g.dfinal, rows.sequence(i), g, c, in, 0.0f);
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            C[v] = w[i][v] * (d[i][v] + C[v]);
            A[v] *= w[i][v];
        }
    }
    return rows.last != 0;
}

// Maps of the chunks (those behind the first one), each from its last step to its first.
template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_back_map_kernel(ScanArgs g) {
    __shared__ float sa[W][64][VC], sc[W][64][VC];
    __shared__ int scut[W];
    const int lane = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const int bc = blockIdx.x % g.blocks_c;
    const int64_t rest = blockIdx.x / g.blocks_c;
    const int chunk = 1 + (int)(rest % (g.chunks - 1));
    const int64_t batch = rest / (g.chunks - 1);
    const int c = (bc * 64 + lane) * VC;
    const bool in = c < g.channels;
    const int per_wave = g.chunk / W;
    const int64_t begin = (int64_t)chunk * g.chunk + (int64_t)wave * per_wave;
    const int64_t end = g.time < begin + per_wave ? g.time : begin + per_wave;
    float A[VC], C[VC];
    bool cut = false;
#pragma unroll
    for (int v = 0; v < VC; ++v) { A[v] = 1.0f; C[v] = 0.0f; }
    for (int64_t t = begin + per_wave - kSteps; t >= begin; t -= kSteps) {
        if (t >= end) continue;
        float w[kSteps][VC], b[kSteps][VC], d[kSteps][VC];
        const Rows rows(g, t, end, (int)batch);
        load_steps_back<S, T, VC>(w, b, d, g, batch, t, c, in, rows, S == SEMI_LOG);
        cut |= map_of_back<VC>(A, C, w, d, rows, g, c, in);
    }
#pragma unroll
    for (int v = 0; v < VC; ++v) { sa[wave][lane][v] = A[v]; sc[wave][lane][v] = C[v]; }
    if (lane == 0) scut[wave] = cut;
    __syncthreads();
    if (wave != W - 1) return;
    for (int k = W - 2; k >= 0; --k) {
        const bool wcut = scut[k];
        cut |= wcut;
#pragma unroll
        for (int v = 0; v < VC; ++v) {
            C[v] = wcut ? sc[k][lane][v] : fmaf(sa[k][lane][v], C[v], sc[k][lane][v]);
            A[v] *= sa[k][lane][v];
        }
    }
    const int64_t at = batch * g.chunks + chunk;
    if (in) {
        store_elements<VC>(g.map_a + at * g.channels + c, A);
        store_elements<VC>(g.map_h + at * g.channels + c, C);
    }
    if (bc == 0 && lane == 0) g.map_cut[at] = cut;
}

template <int S, typename T, int VC, int W>
__global__ void __launch_bounds__(64 * W) scan_back_kernel(ScanArgs g) {
    __shared__ float sa[2][W][64][VC], sc[2][W][64][VC];
    __shared__ int scut[2][W];
    const int lane = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const int bc = blockIdx.x % g.blocks_c;
    const int64_t rest = blockIdx.x / g.blocks_c;
    const int chunk = (int)(rest % g.chunks);
    const int64_t batch = rest / g.chunks;
    const int c = (bc * 64 + lane) * VC;
    const bool in = c < g.channels;
    float carry[VC];
#pragma unroll
    for (int v = 0; v < VC; ++v) carry[v] = 0.0f;
    for (int k = g.chunks - 1; k > chunk; --k) {
        const int64_t at = batch * g.chunks + k;
        float A[VC] = {}, C[VC] = {};
        if (in) {
            load_elements<VC>(A, g.map_a + at * g.channels + c);
            load_elements<VC>(C, g.map_h + at * g.channels + c);
        }
        const bool cut = g.map_cut[at];
#pragma unroll
        for (int v = 0; v < VC; ++v) carry[v] = cut ? C[v] : fmaf(A[v], carry[v], C[v]);
    }
    const int64_t begin = (int64_t)chunk * g.chunk, end = g.time < begin + g.chunk ? g.time : begin + g.chunk;
    const int64_t tiles = (end - begin + W * kSteps - 1) / (W * kSteps);
    int turn = 0;
    for (int64_t n = tiles - 1; n >= 0; --n, turn ^= 1) {
        const int64_t t = begin + n * (W * kSteps) + wave * kSteps;
        float w[kSteps][VC], b[kSteps][VC], d[kSteps][VC], A[VC], C[VC];
        const Rows rows(g, t, end, (int)batch);
        load_steps_back<S, T, VC>(w, b, d, g, batch, t, c, in, rows, S == SEMI_LOG || g.da);
#pragma unroll
        for (int v = 0; v < VC; ++v) { A[v] = 1.0f; C[v] = 0.0f; }
        const bool cut = map_of_back<VC>(A, C, w, d, rows, g, c, in);
#pragma unroll
        for (int v = 0; v < VC; ++v) { sa[turn][wave][lane][v] = A[v]; sc[turn][wave][lane][v] = C[v]; }
        if (lane == 0) scut[turn][wave] = cut;
        __syncthreads();
        float cc[VC];
#pragma unroll
        for (int k = W - 1; k >= 0; --k) {
            const bool wcut = scut[turn][k];
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                if (k == wave) cc[v] = carry[v];
                carry[v] = wcut ? sc[turn][k][lane][v] : fmaf(sa[turn][k][lane][v], carry[v], sc[turn][k][lane][v]);
            }
        }
        const int64_t at = (batch * g.time + t) * g.channels + c;
        T* da = static_cast<T*>(g.da) + at;
        T* dx = static_cast<T*>(g.dx) + at;
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            if (rows.last >> i & 1) load_state<VC>(cc, g.dfinal, rows.sequence(i), g, c, in, 0.0f);
            float ya[VC], yx[VC];
            const bool live = rows.live >> i & 1;
#pragma unroll
            for (int v = 0; v < VC; ++v) {
                const float gt = d[i][v] + cc[v];
                cc[v] = w[i][v] * gt;
                ya[v] = live ? (S == SEMI_LOG ? cc[v] : gt * b[i][v]) : 0.0f;
                yx[v] = live ? (S == SEMI_LOG ? gt * b[i][v] : gt) : 0.0f;
            }
            if (t + i < end && in) {
                if (g.da) store_elements<VC>(da + (int64_t)i * g.channels, ya);
                if (g.dx) store_elements<VC>(dx + (int64_t)i * g.channels, yx);
                if (g.dinitial && (rows.first >> i & 1)) store_elements<VC>(g.dinitial + rows.sequence(i) * g.channels + c, cc);
            }
        }
    }
}

// ---- packed sequences: what each row is, and the states of sequences without rows -----------------------------------
// Thread n < rows: row n belongs to the first sequence s with offsets[s + 1] > n.  Offsets that are not what they should be (descending,
// past the rows, negative) give other results, never an access out of range: s is found in [0, sequences], and row 0 reads no row
// before it.
__global__ void __launch_bounds__(256) scan_rows_kernel(int32_t* rows, const int64_t* offsets, int64_t count, int32_t sequences) {
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= count) return;
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
