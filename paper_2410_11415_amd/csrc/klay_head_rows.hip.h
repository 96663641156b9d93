// What is done with a row of a head before and after its tiles: its list of tokens, the join of its tiles, the adjoints that it sends back.  A wave a row.
#pragma once

#include "klay_head.hip.h"

namespace klay {

// The tiles' sums of a row, by a wave: a lane's tiles one after the other, four loads on their way, then the lanes pair by pair.  `scale` = log2 e / T.
__device__ __forceinline__ Others join_tiles(const float4* partial, int64_t tiles, float scale) {
    const int32_t lane = threadIdx.x & 63;
    Part mine{-INFINITY, 0.0f, 0.0f};
    for (int64_t i = lane; i < tiles; i += 256) {
        float4 p[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) p[u] = i + 64 * u < tiles ? partial[i + 64 * u] : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int u = 0; u < 4; ++u) mine = joined(mine, Part{p[u].x, p[u].y, p[u].z}, scale);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        mine = joined(mine, Part{__shfl_xor(mine.max, d), __shfl_xor(mine.rest, d), __shfl_xor(mine.weighted, d)}, scale);
    Others o;
    o.max = lane_of(mine.max, 0);                                // (lanes that joined equal maxima in another order may differ in the last bit)
    const double rest = lane_of(mine.rest, 0);
    o.sum = o.max == -INFINITY && rest == 0.0 ? 0.0 : 1.0 + rest;
    o.rest = rest;
    o.weighted = lane_of(mine.weighted, 0) * 0.693147180559945309;       // (the tiles' are in powers of two)
    return o;
}

struct FinishArgs {
    const float4* partial;
    int64_t tiles, rows;
    int32_t num_tokens;
    float scale;
    int32_t *sorted, *slots;
    const float* values;
    ListArgs list;                          // num_tokens = 1: no list has been made; it is the token, of row list_row + r, and is written here
    int64_t list_row;
};
// A row's one token as its list.
struct One {
    int32_t sorted, slot;
};
__device__ __forceinline__ bool list_of_one(const FinishArgs& g, int64_t r, One* one) {
    if (g.num_tokens != 1) return false;
    if ((threadIdx.x & 63) == 0) {
        const int32_t t = token_of(g.list, g.list_row + r, 0);
        *one = One{t >= 0 ? t : kNoToken, t >= 0 ? 0 : t};
        g.sorted[r] = one->sorted;
        g.slots[r] = one->slot;
    }
    wave_ordered();
    return true;
}
__global__ void __launch_bounds__(256) head_logprobs_finish_kernel(FinishArgs g, RowOut out) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= g.rows) return;
    __shared__ One one[4];
    One* mine = one + (threadIdx.x >> 6);
    const int64_t at = r * g.num_tokens;
    const bool single = list_of_one(g, r, mine);
    finish_logprobs(out, r, g.num_tokens, single ? &mine->sorted : g.sorted + at, single ? &mine->slot : g.slots + at, g.values + at,
                    join_tiles(g.partial + r * g.tiles, g.tiles, g.scale));
}
__global__ void __launch_bounds__(256) head_distill_finish_kernel(FinishArgs g, TeachArgs t) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= g.rows) return;
    __shared__ One one[4];
    One* mine = one + (threadIdx.x >> 6);
    const int64_t at = r * g.num_tokens;
    const bool single = list_of_one(g, r, mine);
    finish_distill(t, r, g.num_tokens, single ? &mine->sorted : g.sorted + at, single ? &mine->slot : g.slots + at, g.values + at,
                   join_tiles(g.partial + r * g.tiles, g.tiles, g.scale));
}

// The lists of rows: a wave a row.
__global__ void __launch_bounds__(256) head_lists_kernel(ListArgs g) {
    __shared__ int32_t mark[4][kMaxListed], sorted[4][kMaxListed], slots[4][kMaxListed];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + w;
    if (g.num_tokens <= 64) {
        if (r >= g.rows) return;
        const int64_t at = r * g.num_tokens;
        bool first;
        const int32_t token = lane < g.num_tokens ? token_of(g, r, lane) : kNothing, slot = slot_in_wave(token, g.num_tokens, first);
        const int32_t many = __popcll(__ballot(first));
        if (lane < g.num_tokens) {
            g.slots[at + lane] = slot;
            if (first) g.sorted[at + slot] = token;
            if (lane >= many) g.sorted[at + lane] = kNoToken;
        }
        return;
    }
    make_list(g, r, r < g.rows, lane, 64, mark[w], sorted[w], slots[w]);
    if (r >= g.rows) return;
    for (int32_t k = lane; k < g.num_tokens; k += 64) {
        g.sorted[r * g.num_tokens + k] = sorted[w][k];
        g.slots[r * g.num_tokens + k] = slots[w][k];
    }
}

// ---- the adjoints of a row -------------------------------------------------------------------------------------------
struct AdjointArgs {
    const float* stats;                     // [rows, kRowFloats]
    const int32_t *sorted, *slots;
    const float* values;                    // forward's: logits of the listed tokens; of a distillation Q p - q
    const float *dlogp, *dneg, *dentropy;   // or null
    const float* dloss;
    float inverse_temperature;
    int64_t rows;
    int32_t num_tokens;
    float4* coefs;
    float* entries;
    uint32_t* largest;                      // or null
};
// Atomic maxima of non-negative numbers' bits: no order changes the result.
__device__ __forceinline__ void note_largest(uint32_t* largest, float x) {
    if (!largest) return;
    x = wave_max(x);
    if ((threadIdx.x & 63) == 0 && x > 0.0f && x < INFINITY) atomicMax(largest, __float_as_uint(x));
}

//   dx_j = s_j (away (sum_k w_k) + n_o p_o) - h p_j (ln p_j + H),  w_k = n_k p_k / (1 - p_k) - g_k,  p_j = away s_j
// with g, n, h the adjoints of logp, neg, H.  Where the largest asked token o is the row's maximum, `away` = 1 - p_o, s_j is the share of j in it, and
// w_o = -g_o: its n_o p_o / (1 - p_o) p_j is n_o p_o s_j, finite however small 1 - p_o is.  Otherwise away = 1 and s = p.
__global__ void __launch_bounds__(256) head_logprobs_adjoint_kernel(AdjointArgs g) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= g.rows) return;
    const int32_t lane = threadIdx.x & 63, K = g.num_tokens;
    const PickStats st = reinterpret_cast<const PickStats*>(g.stats)[r];
    const int32_t *sorted = g.sorted + r * K, *slots = g.slots + r * K;
    const float *x = g.values + r * K, *dlogp = g.dlogp ? g.dlogp + r * K : nullptr, *dneg = g.dneg ? g.dneg + r * K : nullptr;
    float* entries = g.entries + r * K;
    const double h = g.dentropy ? g.dentropy[r] : 0.0f, H = st.entropy;
    float asked = h != 0.0 ? 1.0f : 0.0f, bad = 0.0f;
    for (int32_t k = lane; k < K; k += 64) {
        if (slots[k] == kNothing || !((dlogp && dlogp[k] != 0.0f) || (dneg && dneg[k] != 0.0f))) continue;
        asked = 1.0f;
        if (slots[k] == kOutside) bad = 1.0f;
    }
    asked = wave_max(asked);
    bad = wave_max(bad);
    if (asked == 0.0f || st.empty) {
        for (int32_t u = lane; u < K; u += 64) entries[u] = 0.0f;
        if (lane == 0) g.coefs[r] = make_float4(INFINITY, 0.0f, 0.0f, 0.0f);
        return;
    }
    // the entries of a token added up; of at most 64 entries from the lanes that hold them (all lanes ask together)
    const int32_t slot0 = lane < K ? slots[lane] : kNothing;
    const float g0 = dlogp && lane < K ? dlogp[lane] : 0.0f, n0 = dneg && lane < K ? dneg[lane] : 0.0f;
    auto adjoints = [&](int32_t u, double& gu, double& nu) {
        gu = nu = 0.0;
        if (K <= 64) {
            for (int32_t k = 0; k < K; ++k) {
                const bool this_one = __builtin_amdgcn_readlane(slot0, k) == u;
                gu += this_one ? lane_of(g0, k) : 0.0f;
                nu += this_one ? lane_of(n0, k) : 0.0f;
            }
            return;
        }
        for (int32_t k = 0; k < K; ++k) {
            if (slots[k] != u) continue;
            if (dlogp) gu += dlogp[k];
            if (dneg) nu += dneg[k];
        }
    };
    auto logp = [&](int32_t u) { return ((double)x[u] - st.max) - st.log_sum; };
    auto weight = [&](int32_t u, double gu, double nu) {
        const double lp = logp(u), away = -expm1(lp);
        return (u != st.owner && nu != 0.0 && away > 0.0 ? nu * exp(lp) / away : 0.0) - gu;
    };
    const double away = st.owner >= 0 ? (double)st.away : 1.0;
    double all = 0.0, sure = 0.0, gu0 = 0.0, nu0 = 0.0;           // gu0, nu0: those of token `lane`
    for (int32_t u0 = 0; u0 < K; u0 += 64) {
        const int32_t u = u0 + lane;
        double gu, nu;
        adjoints(u, gu, nu);
        if (u0 == 0) { gu0 = gu; nu0 = nu; }
        if (u >= K || sorted[u] == kNoToken) continue;
        all += weight(u, gu, nu);
        if (u == st.owner) sure = nu * exp(logp(u));
    }
    all = wave_sum(all);
    sure = wave_sum(sure);
    const bool nan = bad > 0.0f || st.log_sum != st.log_sum;
    const double A = nan ? NAN : away * all + sure - (away > 0.0 ? h * away * (log(away) + H) : 0.0), B = -h * away;
    float most = fabsf((float)A) + 0.37f * fabsf((float)B);         // (|s ln s| <= 1 / e)
    for (int32_t u = lane; u < K; u += 64) {
        float entry = 0.0f;
        if (sorted[u] < kNoToken) {
            double gu = gu0, nu = nu0;
            if (u >= 64) adjoints(u, gu, nu);
            const double lp = logp(u), p = exp(lp), others = all - weight(u, gu, nu);
            double d = (u == st.owner ? gu * away : gu * -expm1(lp)) - nu * p + p * others;
            if (u != st.owner && sure != 0.0) d += sure * exp(((double)x[u] - st.ref) - st.ref_log);
            if (p > 0.0) d -= h * p * (lp + H);
            entry = nan ? NAN : (float)d;
        }
        entries[u] = entry;
        most = fmaxf(most, fabsf(entry));
    }
    note_largest(g.largest, most);
    if (lane == 0) g.coefs[r] = make_float4(nan ? 0.0f : st.ref, st.ref_log * kTokLog2e, (float)A, (float)B * kTokLn2);
}

__global__ void __launch_bounds__(256) head_distill_adjoint_kernel(AdjointArgs g) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= g.rows) return;
    const int32_t lane = threadIdx.x & 63, K = g.num_tokens;
    const TeachStats st = reinterpret_cast<const TeachStats*>(g.stats)[r];
    const float d = g.dloss[r] * g.inverse_temperature;
    const bool live = d != 0.0f && st.live;
    const float A = live ? d * st.others : 0.0f;
    float most = fabsf(A);
    for (int32_t u = lane; u < K; u += 64) {
        const float entry = live ? d * g.values[r * K + u] : 0.0f;
        g.entries[r * K + u] = entry;
        most = fmaxf(most, fabsf(entry));
    }
    note_largest(g.largest, most);
    if (lane == 0) g.coefs[r] = make_float4(!live ? INFINITY : A == A ? st.ref : 0.0f, st.ref_log * kTokLog2e, A, 0.0f);
}

}  // namespace klay
