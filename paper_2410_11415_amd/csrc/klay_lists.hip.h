// Rows of tokens that are asked for, or listed by a teacher, and what is said of a row once the tokens' logits and the sums over all
// OTHER tokens are known:  others = {M_o, O = sum e^(x_j - M_o), R_o = O - 1 (its largest term apart), U_o = sum e^(x_j - M_o)(x_j - M_o)}.
// Kept apart like this, the mass of "not t_k" and of "none of the listed" is a sum of positive terms, exact relative to itself however small it
// is, where 1 - p would have lost it.  A row's few numbers are put together in 64 bits (a wave a row; the sums over the vocabulary are in
// 32), since a divergence near 0 and the logarithm of a sum next to 1 are differences of nearly equal numbers.
#pragma once

#include "klay_tokens.hip.h"

namespace klay {

constexpr int kMaxListed = kMaxTokens;
constexpr int32_t kNothing = -1, kOutside = -2;     // of a row's entries: nothing asked; no token of the vocabulary
constexpr int32_t kNoToken = INT32_MAX;             // behind a row's last token
constexpr int kRowFloats = 8;                       // what a forward pass leaves of a row for the gradient

// A row's entries: `slots[k]` is kNothing, kOutside, or the place of entry k's token among the row's different tokens, `sorted[0 ..]`, ascending.
struct ListArgs {
    const int64_t* tokens;
    RowMap token_rows;
    int64_t token_stride;
    int64_t rows;
    int32_t num_tokens, vocab;
    int32_t *sorted, *slots;                // [rows, num_tokens]
};

__device__ __forceinline__ int32_t token_of(const ListArgs& g, int64_t r, int32_t k) {
    const int64_t t = g.tokens[g.token_rows.at(r) + k * g.token_stride];
    return t < 0 ? kNothing : t >= g.vocab ? kOutside : (int32_t)t;
}

// A row's list in shared memory, made by `threads` threads (`thread` is one of them); `mark` is scratch, all are [num_tokens].  Every thread of the
// workgroup has to come here: barriers.
__device__ __forceinline__ void make_list(const ListArgs& g, int64_t r, bool there, int32_t thread, int32_t threads, int32_t* mark, int32_t* sorted,
                                          int32_t* slots) {
    const int32_t K = g.num_tokens;
    for (int32_t k = thread; k < K; k += threads) {
        slots[k] = there ? token_of(g, r, k) : kNothing;
        sorted[k] = kNoToken;
    }
    __syncthreads();
    for (int32_t k = thread; k < K; k += threads) {          // mark: a token where it is mentioned first
        const int32_t t = slots[k];
        bool again = t < 0;
        for (int32_t o = 0; o < k && !again; ++o) again = slots[o] == t;
        mark[k] = again ? kNoToken : t;
    }
    __syncthreads();
    for (int32_t k = thread; k < K; k += threads) {
        const int32_t t = slots[k];
        if (t < 0) continue;
        int32_t place = 0;
        for (int32_t o = 0; o < K; ++o) place += mark[o] < t;
        if (mark[k] == t) sorted[place] = t;
        slots[k] = place;                                     // (read as a token by nobody any more)
    }
    __syncthreads();
}
// Of at most 64 entries, by a wave whose lanes hold them (`token`: kNothing behind the last): lane k gets the slot of entry k, and whether it is its
// token's first mention.
__device__ __forceinline__ int32_t slot_in_wave(int32_t token, int32_t K, bool& first) {
    const int32_t lane = threadIdx.x & 63;
    bool again = token < 0;
    for (int32_t o = 0; o < K; ++o) again |= o < lane && __builtin_amdgcn_readlane(token, o) == token;
    first = !again;
    const int32_t mark = again ? kNoToken : token;
    int32_t place = 0;
    for (int32_t o = 0; o < K; ++o) place += __builtin_amdgcn_readlane(mark, o) < token;
    return token < 0 ? token : place;
}

// What a wave's lanes have written into shared memory before is there for all of them.
__device__ __forceinline__ void wave_ordered() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---- sums over a wave ---------------------------------------------------------------------------------------------
__device__ __forceinline__ double lane_of(double x, int lane) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane), __builtin_amdgcn_readlane(__double2loint(x), lane));
}
__device__ __forceinline__ float lane_of(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }
template <int CONTROL> __device__ __forceinline__ double with_lane_sum(double x) {
    return x + __hiloint2double(from_lane<CONTROL>(0, __double2hiint(x)), from_lane<CONTROL>(0, __double2loint(x)));
}
__device__ __forceinline__ double wave_sum(double x) {
    x = with_lane_sum<LANES_MIRROR>(with_lane_sum<LANES_HALF_MIRROR>(with_lane_sum<LANES_XOR2>(with_lane_sum<LANES_XOR1>(x))));
    return lane_of(with_lane_sum<LANES_NEXT_HALF>(with_lane_sum<LANES_NEXT_ROW>(x)), 63);
}
__device__ __forceinline__ float wave_max(float x) { return group_max<64>(x); }
__device__ __forceinline__ int32_t wave_min(int32_t x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) { const int32_t y = __shfl_xor(x, d); x = y < x ? y : x; }
    return x;
}

struct Others {
    float max = -INFINITY;
    double sum = 0.0, rest = 0.0, weighted = 0.0;
};

// ---- log probabilities --------------------------------------------------------------------------------------------
struct RowOut {
    float *logp, *neg, *entropy;            // [rows, num_tokens], the same, [rows]; null: not asked
    float* stats;                           // [rows, kRowFloats], or null
};
// Of a row: the reference that its gradient is made with (the whole row; or, where an asked token is the row's largest, everything but it), its
// entropy, and the largest asked token.
struct PickStats {
    float ref, ref_log, entropy, max, log_sum, away;     // away: 1 - p of the largest asked token
    int32_t owner, empty;
};
static_assert(sizeof(PickStats) == kRowFloats * sizeof(float), "what a row keeps");

// A wave's: `sorted`, `slots` and the logits `x` of the sorted tokens, [num_tokens].
__device__ __forceinline__ void finish_logprobs(const RowOut& out, int64_t r, int32_t K, const int32_t* sorted, const int32_t* slots, const float* x,
                                                const Others& o) {
    const int32_t lane = threadIdx.x & 63;
    float most = -INFINITY;
    int32_t owner = 1 << 30;
    for (int32_t u = lane; u < K; u += 64)
        if (sorted[u] < kNoToken && x[u] > most) { most = x[u]; owner = u; }
    const float mine = most;
    most = wave_max(most);
    owner = wave_min(mine == most && most > -INFINITY ? owner : 1 << 30);
    const bool asked = owner < (1 << 30) && most >= o.max;
    if (!asked) owner = -1;
    const float M = fmaxf(most, o.max);
    const double at = fmaxf(M, -kTokFltMax);
    float second = -INFINITY;
    double rest = 0.0, weighted = 0.0;
    for (int32_t u = lane; u < K; u += 64) {
        if (sorted[u] == kNoToken || u == owner) continue;
        second = fmaxf(second, x[u]);
        const double d = (double)x[u] - at, e = exp(d);
        rest += e;
        if (d > -1e30) weighted += e * d;
    }
    second = fmaxf(wave_max(second), asked ? o.max : -INFINITY);
    const double o_at = fmaxf(o.max, -kTokFltMax), shift = o_at - at, f = exp(shift);
    rest = wave_sum(rest) + (asked ? o.sum * f : o.max > -INFINITY ? o.rest : o.sum);
    weighted = wave_sum(weighted) + (f > 0.0 ? f * (o.weighted + shift * o.sum) : 0.0);
    const bool bad = M == INFINITY;
    if (bad) rest = NAN;
    // what is left beside the largest asked token, from its own largest on (a gap that no exponential bridges is a finite logarithm all the same)
    double ref_log = 0.0;
    if (asked && second > -INFINITY) {
        const double two = second;
        double s = 0.0;
        for (int32_t u = lane; u < K; u += 64)
            if (sorted[u] < kNoToken && u != owner) s += exp((double)x[u] - two);
        ref_log = log(wave_sum(s) + o.sum * exp(o_at - two));
    }
    const bool empty = M == -INFINITY && rest == 0.0;
    const double log_sum = empty ? 0.0 : log1p(rest);
    const double log_away = second > -INFINITY ? ((double)second - at) + ref_log - log_sum : -INFINITY;
    const float h = empty ? 0.0f : (float)(log_sum - weighted / (1.0 + rest));
    for (int32_t k = lane; k < K; k += 64) {
        const int32_t u = slots[k];
        double lp = 0.0, neg = 0.0;
        if (u == kOutside) {
            lp = neg = NAN;
        } else if (u >= 0) {
            lp = (M == -INFINITY ? -INFINITY : (double)x[u] - at) - log_sum;
            if (bad || log_sum != log_sum) lp = NAN;
            neg = lp != lp ? lp : empty ? 0.0 : u == owner ? log_away : log1p(-exp(lp));
        }
        out.logp[r * K + k] = (float)lp;
        if (out.neg) out.neg[r * K + k] = (float)neg;
    }
    if (lane == 0) {
        if (out.entropy) out.entropy[r] = h;
        if (out.stats) {
            PickStats s;
            const bool apart = asked && second > -INFINITY;
            s.ref = apart ? second : (float)at;
            s.ref_log = (float)(apart ? ref_log : log_sum);
            if (log_sum != log_sum) s.ref_log = NAN;
            s.entropy = h;
            s.max = (float)at;
            s.log_sum = (float)log_sum;
            s.away = asked ? (float)exp(log_away) : 1.0f;
            s.owner = owner;
            s.empty = empty;
            reinterpret_cast<PickStats*>(out.stats)[r] = s;
        }
    }
}

// ---- divergence from a teacher's list ------------------------------------------------------------------------------
//   q = softmax of the listed teacher logits / T (rest: e^teacher, and q_r = 1 - sum q for all other tokens together), p = softmax(x / T)
//   loss = sum q_k (ln q_k - ln p_k) + q_r (ln q_r - ln (1 - P)),  P = sum of p over the listed tokens
//   T dx_j = Q p_j - sum_{k: t_k = j} q_k for a listed token, p_j (Q - q_r / (1 - P)) for the others, Q the sum of all q: 1 but with `rest` where the
//   list has more than 1, or has less and no other token is allowed (q_r is 0 then)
struct TeachArgs {
    const float* teacher;                   // placed by these; row r of the call is its row first + r
    RowMap teacher_rows;
    int64_t first;
    int64_t teacher_stride;
    double inverse_temperature;
    int32_t rest;
    float* loss;                            // [rows]
    float* stats;                           // [rows, kRowFloats], or null
    float* moved;                           // [rows, num_tokens]: of a sorted token its entry of the gradient, Q p - q; or null
};
struct TeachStats {
    float ref, ref_log, others;             // others: Q (1 - P) - q_r, which the tokens that are not listed have by their shares of 1 - P
    int32_t live;                           // 0: nothing is listed, or nothing allowed: no gradient
    float unused[4];
};
static_assert(sizeof(TeachStats) == kRowFloats * sizeof(float), "what a row keeps");

// A wave's, as finish_logprobs.  `moved` may be x (a token's logit is read before its entry is written).
__device__ __forceinline__ void finish_distill(const TeachArgs& t, int64_t r, int32_t K, const int32_t* sorted, const int32_t* slots, const float* x,
                                               const Others& o) {
    const int32_t lane = threadIdx.x & 63;
    const float* teacher = t.teacher + t.teacher_rows.at(t.first + r);
    const double inv = t.inverse_temperature;
    float most = -INFINITY;
    float z_top = -INFINITY, any = 0.0f, bad = 0.0f;
    for (int32_t k = lane; k < K; k += 64) {
        if (sorted[k] < kNoToken) most = fmaxf(most, x[k]);
        if (slots[k] == kNothing) continue;
        if (slots[k] == kOutside) bad = 1.0f;
        const float z = teacher[k * t.teacher_stride];
        if (z != z || z == INFINITY) bad = 1.0f;
        z_top = fmaxf(z_top, z);
        any = 1.0f;
    }
    most = wave_max(most);
    const double z_most = wave_max(z_top);
    any = wave_max(any);
    bad = wave_max(bad);
    const float M = fmaxf(most, o.max);
    const double at = fmaxf(M, -kTokFltMax), o_at = fmaxf(o.max, -kTokFltMax);
    double s = 0.0, zs = 0.0;
    for (int32_t k = lane; k < K; k += 64) {
        if (sorted[k] < kNoToken) s += exp(((double)x[k] - at) * inv);
        if (slots[k] == kNothing) continue;
        const double z = teacher[k * t.teacher_stride];
        if (z > -INFINITY) zs += t.rest ? exp(z) : exp((z - z_most) * inv);
    }
    const double o_mass = o.sum * exp((o_at - at) * inv);
    s = wave_sum(s) + o_mass;
    zs = wave_sum(zs);
    const bool teaches = any > 0.0f && (t.rest || z_most > -INFINITY || bad > 0.0f);
    const double log_s = log(s), log_z = t.rest ? 0.0 : log(zs);
    const bool others = o.max > -INFINITY;
    const double q_rest = t.rest && others ? fmax(0.0, 1.0 - zs) : 0.0;
    const double q_all = t.rest && !(q_rest > 0.0) ? zs : 1.0;
    const bool empty = M == -INFINITY && s == 0.0, nan = bad > 0.0f || M == INFINITY || s != s;
    double loss = 0.0, q0 = 0.0;                              // q0: of entry `lane`
    for (int32_t k = lane; k < K; k += 64) {
        const int32_t u = slots[k];
        if (u < 0) continue;
        const double z = teacher[k * t.teacher_stride];
        const double lq = t.rest ? z : (z - z_most) * inv - log_z, q = z > -INFINITY ? exp(lq) : 0.0;
        const double lp = x[u] > -INFINITY || x[u] != x[u] ? ((double)x[u] - at) * inv - log_s : -INFINITY;
        if (q > 0.0) loss += q * (lq - lp);
        if (k == lane) q0 = q;
    }
    if (t.moved) {
        for (int32_t u0 = 0; u0 < K; u0 += 64) {             // (all lanes together: every x of these 64 is read before one is written)
            const int32_t u = u0 + lane;
            const bool there = u < K && sorted[u] < kNoToken && !empty && teaches;
            double taken = 0.0;
            if (K <= 64) {
                const int32_t slot = lane < K ? slots[lane] : kNothing;
                for (int32_t k = 0; k < K; ++k) taken += __builtin_amdgcn_readlane(slot, k) == u ? lane_of(q0, k) : 0.0;
            } else if (there) {
                for (int32_t k = 0; k < K; ++k) {
                    if (slots[k] != u) continue;
                    const double z = teacher[k * t.teacher_stride];
                    if (z > -INFINITY) taken += t.rest ? exp(z) : exp((z - z_most) * inv - log_z);
                }
            }
            const double lp = there && x[u] > -INFINITY ? ((double)x[u] - at) * inv - log_s : -INFINITY;
            if (u < K) t.moved[r * K + u] = !there ? 0.0f : nan ? NAN : (float)(q_all * exp(lp) - taken);
        }
    }
    loss = wave_sum(loss);
    const double log_o = others ? log(o.sum) : 0.0;
    if (q_rest > 0.0) loss += q_rest * (log(q_rest) - (log_o + (o_at - at) * inv - log_s));
    if (nan) loss = NAN;
    if (!teaches) loss = 0.0;
    if (lane != 0) return;
    t.loss[r] = (float)loss;
    if (t.stats) {
        TeachStats st = {};
        st.ref = others ? o.max : 0.0f;
        st.ref_log = (float)log_o;
        st.live = teaches && !empty;
        st.others = !st.live ? 0.0f : nan ? NAN : (float)(q_all * (o_mass / s) - q_rest);
        reinterpret_cast<TeachStats*>(t.stats)[r] = st;
    }
}

}  // namespace klay
