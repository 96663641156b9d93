// The library's device code: the circuit evaluator (klay_api.hip) and the operators that need no handle, whose entry points are here.
// One translation unit, so that all entry points report through the same thread-local message.
#include "klay_api.hip"

#include "klay_scan.hip.h"
#include "klay_tokens.hip.h"

#include <initializer_list>

namespace {

// Makes `device` current for a call, and the earlier one again afterwards.
struct OnDevice {
    int before = -1;
    bool changed = false;
    hipError_t status;
    explicit OnDevice(int device) {
        status = hipGetDevice(&before);
        if (status == hipSuccess && before != device) {
            status = hipSetDevice(device);
            changed = status == hipSuccess;
        }
    }
    ~OnDevice() {
        if (changed) (void)hipSetDevice(before);
    }
};

// Launch errors come as the launch's own status; what an earlier call has left is none of ours.
#define KLAY_LAUNCH(kernel, grid, block, stream, ...)                                                    \
    do {                                                                                                 \
        (void)hipGetLastError();                                                                         \
        hipLaunchKernelGGL(kernel, grid, block, 0, static_cast<hipStream_t>(stream), __VA_ARGS__);       \
        KLAY_HIP(hipGetLastError());                                                                     \
    } while (0)

constexpr int kComputeUnits = 256;
constexpr int32_t kMostChannels = 1 << 25;      // and the most elements from one time step to the next: a wave's rows lie within 32-bit offsets
bool known_dtype(int32_t t) { return t == KLAY_F32 || t == KLAY_BF16 || t == KLAY_F16; }
int dtype_bytes(int32_t t) { return t == KLAY_F32 ? 4 : 2; }

// ---- tokens ---------------------------------------------------------------------------------------------------------
// Rows in the registers of a wave, of a quarter of one (us, forward and reverse: 65536 x 64 bf16 by quarters / whole waves 13.8 / 50.4, 11.8 / 35.8;
// 65536 x 512 fp32 by a wave's registers / by a wave that goes through vectors 53.6 / 57.7, 94.6 / 102.5; 65536 x 257 bf16 58 / 58, 50 / 110; 65536 x 512
// bf16 77.5 / 56.0, 83.4 / 91.9).
constexpr int32_t kShortRow = 512, kShortestRow = 64;
// Up to this many bytes a row is a single wave's where there are rows enough (us, four waves / one: 8192 x 8192 bf16 forward 38 / 30,
// 16384 x 1000 bf16 45 / 19; 4096 x 32768 bf16 48 / 51, backward 112 / 150).
constexpr int64_t kWaveRow = 16384;
// Workgroups that keep the chip busy by themselves (us, forward, as few rows / as many: 256 x 32771 bf16 7.5 / 9.5, 511 rows 13.1 / 11.6, 768 rows 18.7 / 14.2;
// 256 x 131072 16.6 / 16.6; 511 x 8191 7.3 / 7.8, 1024 rows 8.2 / 9.2, 2000 rows 13.4 / 11.7).
constexpr int64_t kManyRows = 2 * kComputeUnits;

klay_status check_tokens(const klay_tokens_args* a, const char* who) {
    auto refused = [who](const std::string& why) { return fail(KLAY_EINVAL, who + (": " + why)); };
    if (!a) return refused("null argument");
    if (!known_dtype(a->dtype)) return refused("unknown dtype");
    if (a->vocab < 1 || a->num_tokens < 0 || a->num_tokens > klay::kMaxTokens)
        return refused("vocab must be >= 1 and num_tokens 0 .. " + std::to_string(klay::kMaxTokens));
    if (a->top < 0 || a->top > klay::kMaxTop || a->top > a->vocab)
        return refused("top must be 0 .. min(vocab, " + std::to_string(klay::kMaxTop) + ")");
    if (a->rows < 0 || a->rows > INT32_MAX) return refused("rows must be 0 .. 2^31 - 1");
    if (a->rows == 0) return KLAY_OK;
    if (!a->logits || (a->num_tokens > 0 && !a->tokens)) return refused("null argument");
    if (a->logit_rows.inner < 1 || a->logit_rows.inner > INT32_MAX ||
        (a->num_tokens > 0 && (a->token_rows.inner < 1 || a->token_rows.inner > INT32_MAX)))
        return refused("the inner axis of rows must be 1 .. 2^31 - 1");
    return KLAY_OK;
}

// How rows longer than kShortRow are shared out: threads of a workgroup, workgroups per row, elements of each.
struct TokenPlan {
    int threads = 256;
    int32_t parts = 1, part = 0;
};

TokenPlan in_parts(const klay_tokens_args* a, int threads, int64_t parts) {
    TokenPlan p;
    p.threads = threads;
    const int64_t round = (int64_t)threads * (16 / dtype_bytes(a->dtype));       // elements that a workgroup takes at a time
    int64_t size = (a->vocab + parts - 1) / parts;
    if (parts > 1) size = (size + round - 1) / round * round;
    p.part = (int32_t)std::min<int64_t>(size, INT32_MAX);
    p.parts = (int32_t)((a->vocab + size - 1) / size);
    return p;
}

// Many rows: a workgroup each.  Few: sixteen waves each, and several workgroups only where a row is so long that what they save is more
// than the second launch that joins them costs (a workgroup takes in some 55 GB/s; the join is about 8 us.  Whole / in parts, us: 1 x 200000 bf16
// 15.2 / 13.1, 1 x 262144 18.5 / 14.4, 64 x 262144 19.6 / 15.7; 1 x 300000 20.6 / 13.1, 64 x 300000 21.8 / 15.7, 120 x 300000 22.1 / 25.1, 120 x 1000000 62 / 52).
TokenPlan forward_plan(const klay_tokens_args* a) {
    const int64_t bytes = (int64_t)a->vocab * dtype_bytes(a->dtype);
    if (a->rows >= kManyRows) return in_parts(a, bytes <= kWaveRow ? 64 : 256, 1);
    if (bytes <= kWaveRow) return in_parts(a, 256, 1);
    return in_parts(a, 1024, bytes <= 512 * 1024 ? 1 : std::min<int64_t>((bytes + 262143) / 262144, klay::kMaxParts));
}

// The gradient's parts need no joining: workgroups of kBackPart bytes, or less where there would be fewer than four per CU.  (Reads and
// writes together go faster the smaller the stretch that all workgroups are on: 4096 x 131072 bf16, whole rows / 64 / 32 / 16 KB, 416 / 382 / 352 /
// 361 us; a plain copy, 256 / 16 KB, 5.3 / 6.1 TB/s.)
constexpr int64_t kBackPart = 32768;
TokenPlan backward_plan(const klay_tokens_args* a) {
    const int64_t bytes = (int64_t)a->vocab * dtype_bytes(a->dtype);
    if (a->rows >= kManyRows && bytes <= kWaveRow) return in_parts(a, 64, 1);
    const int64_t few = std::min<int64_t>((4 * kComputeUnits + a->rows - 1) / a->rows, (bytes + 8191) / 8192);
    return in_parts(a, 256, std::max<int64_t>(few, (bytes + kBackPart - 1) / kBackPart));
}

size_t token_lists_at(int64_t rows, int32_t parts) { return (size_t)rows * parts * klay::kPartial * sizeof(float); }

klay::TokenArgs token_args(const klay_tokens_args* a) {
    klay::TokenArgs g{};
    g.logits = a->logits;
    g.logit_rows = klay::RowMap{a->logit_rows.outer_stride, a->logit_rows.inner_stride, (int32_t)a->logit_rows.inner};
    g.tokens = a->tokens;
    g.token_rows = klay::RowMap{a->token_rows.outer_stride, a->token_rows.inner_stride, (int32_t)std::max<int64_t>(a->token_rows.inner, 1)};
    g.token_stride = a->token_stride;
    g.rows = a->rows;
    g.vocab = a->vocab;
    g.num_tokens = a->num_tokens;
    g.top = a->top;
    return g;
}

int32_t capped_grid(int64_t units) { return (int32_t)std::min<int64_t>(units, 1 << 20); }

template <typename T, bool ENT, bool TOP>
klay_status run_tokens(const klay::TokenArgs& g, int threads, void* stream) {
    const dim3 block(klay::kTokBlock);
    if (g.vocab <= kShortRow) {
        const int lanes = g.vocab <= kShortestRow ? 16 : 64, per_block = klay::kTokBlock / lanes;
        const dim3 grid(capped_grid((g.rows + per_block - 1) / per_block));
        if (lanes == 16) KLAY_LAUNCH((klay::token_short_kernel<T, 16, 4, ENT, TOP>), grid, block, stream, g);
        else KLAY_LAUNCH((klay::token_short_kernel<T, 64, 8, ENT, TOP>), grid, block, stream, g);
        return KLAY_OK;
    }
    const dim3 grid(capped_grid(g.rows * g.parts));
    if (threads == 64) KLAY_LAUNCH((klay::token_row_kernel<T, ENT, TOP, 64>), grid, dim3(64), stream, g);
    else if (threads == 256) KLAY_LAUNCH((klay::token_row_kernel<T, ENT, TOP, 256>), grid, dim3(256), stream, g);
    else KLAY_LAUNCH((klay::token_row_kernel<T, ENT, TOP, 1024>), grid, dim3(1024), stream, g);
    if (g.parts > 1) KLAY_LAUNCH((klay::token_join_kernel<T, TOP>), dim3((uint32_t)g.rows), block, stream, g);
    return KLAY_OK;
}

template <typename T>
klay_status run_tokens(const klay::TokenArgs& g, int threads, void* stream) {
    if (g.entropy) return g.top ? run_tokens<T, true, true>(g, threads, stream) : run_tokens<T, true, false>(g, threads, stream);
    return g.top ? run_tokens<T, false, true>(g, threads, stream) : run_tokens<T, false, false>(g, threads, stream);
}

template <typename T>
klay_status run_tokens_back(const klay::TokenArgs& g, int threads, void* stream) {
    const dim3 block(klay::kTokBlock);
    if (g.vocab <= kShortRow) {
        const int lanes = g.vocab <= kShortestRow ? 16 : 64, per_block = klay::kTokBlock / lanes;
        const dim3 grid(capped_grid((g.rows + per_block - 1) / per_block));
        if (lanes == 16) KLAY_LAUNCH((klay::token_back_short_kernel<T, 16, 4>), grid, block, stream, g);
        else KLAY_LAUNCH((klay::token_back_short_kernel<T, 64, 8>), grid, block, stream, g);
        return KLAY_OK;
    }
    const dim3 grid(capped_grid(g.rows * g.parts));
    if (threads == 64) KLAY_LAUNCH((klay::token_back_kernel<T, 64>), grid, dim3(64), stream, g);
    else KLAY_LAUNCH((klay::token_back_kernel<T, 256>), grid, dim3(256), stream, g);
    return KLAY_OK;
}

// ---- recurrence -----------------------------------------------------------------------------------------------------
constexpr int64_t kFewChains = kComputeUnits / 2;
constexpr int64_t kMostTiles = (1ll << 32) / 512 - 1;  // a launch has less than 2^32 threads;  beyond (2^30 steps of 64 channels) one workgroup takes all tiles of its channels

struct ScanPlan {
    int vec = 1, waves = 4;         // channels per lane; waves per workgroup
    int32_t blocks_c = 1;
    int64_t chains = 1, tiles = 0;  // tiles > 0: a workgroup a tile
};

klay_status check_scan(const klay_scan_args* a, bool inputs, const char* who) {
    auto refused = [who](const std::string& why) { return fail(KLAY_EINVAL, who + (": " + why)); };
    if (!a) return refused("null argument");
    if (!known_dtype(a->dtype)) return refused("unknown dtype");
    if (a->semiring != KLAY_REAL && a->semiring != KLAY_LOG && a->semiring != KLAY_MAXLOG) return refused("unknown semiring");
    if (a->semiring != KLAY_REAL && a->dtype != KLAY_F32) return refused("the log-domain semirings take KLAY_F32 only");
    if (a->channels < 1 || a->channels > kMostChannels || a->batch < 0 || a->time < 0 || a->time > INT32_MAX || a->batch > INT32_MAX / 8)
        return refused("channels must be 1 .. 2^25, time 0 .. 2^31 - 1, batch 0 .. 2^28 - 1");
    if (a->gates_time_stride < 0 || a->gates_time_stride > kMostChannels || a->inputs_time_stride < 0 || a->inputs_time_stride > kMostChannels)
        return refused("the time strides must be 0 .. 2^25");
    if (a->offsets) {
        if (a->batch != 1) return refused("packed sequences have batch = 1");
        if (a->sequences < 0 || a->sequences > INT32_MAX / 8) return refused("sequences must be 0 .. 2^28 - 1");
        if (a->time > 0 && !a->row_info) return refused("packed sequences need row_info");
    }
    if (a->batch > 0 && a->time > 0 && (!a->gates || (inputs && !a->inputs))) return refused("null argument");
    return KLAY_OK;
}

// All of them multiples of `bytes`?
bool aligned_to(size_t bytes, std::initializer_list<const void*> all) {
    uintptr_t bits = 0;
    for (const void* p : all) bits |= reinterpret_cast<uintptr_t>(p);
    return bits % bytes == 0;
}

// Waves as many as the time steps give work to, eight at most (sixteen: within 5% either way, and the log semiring's reverse sweep runs out of
// registers).  A workgroup a tile where batch and channels give less than one workgroup per two CUs (us, one for all tiles / one a tile, forward
// and reverse: 8 x 4096 x 512 LOG 143 / 56, 227 / 97; at the border, 8 x 2048 x 1024 fp32, 56 / 52, 92 / 79; 8 x 4096 x 2048 bf16 94 / 103,
// 176 / 180).  Two channels a lane, where addresses and strides let a lane take both at once: there, for 16-bit types (one / two: 4 x 4096 x 2048
// bf16 70 / 59, 92 / 96; 65536 x 512 fp32 93 / 105, 139 / 155); with one workgroup for all tiles, where two workgroups per CU are left (16 x
// 4096 x 4096 fp32 653 / 554, 1113 / 964; 32 x 1024 x 4096 bf16 181 / 169, 329 / 278; 8 x 4096 x 2048 bf16, where half of the CUs would be without
// one, 101 / 126, 175 / 182).
ScanPlan scan_plan(const klay_scan_args* a) {
    ScanPlan p;
    const int64_t size = dtype_bytes(a->dtype);
    auto blocks = [&](int vec) { return (a->channels + 64 * vec - 1) / (64 * vec); };
    const bool pairs = a->channels % 2 == 0 && aligned_to(2 * size, {a->gates, a->inputs}) && (a->gates_batch_stride | a->gates_time_stride |
                       a->inputs_batch_stride | a->inputs_time_stride) % 2 == 0;
    p.waves = a->time <= klay::kSteps ? 1 : a->time <= 4 * klay::kSteps ? 4 : 8;
    const int64_t tiles = (a->time + p.waves * klay::kSteps - 1) / (p.waves * klay::kSteps);
    const bool few = p.waves == 8 && blocks(1) * a->batch <= kFewChains && blocks(1) * a->batch * tiles <= kMostTiles;
    p.vec = a->semiring == KLAY_REAL && pairs && (few ? size == 2 : blocks(2) * a->batch >= 2 * kComputeUnits) ? 2 : 1;
    p.blocks_c = blocks(p.vec);
    p.chains = p.blocks_c * a->batch;
    if (few) p.tiles = tiles;
    return p;
}

// 64-bit words of the workspace: the ticket's, then two per tile and channel, then one per group of tiles and channel
int64_t map_words(const ScanPlan& p) { return p.chains * p.tiles * 2 * 64 * p.vec; }
int64_t scan_words(const ScanPlan& p) {
    return p.tiles == 0 ? 0 : 2 + map_words(p) + p.chains * ((p.tiles + klay::kGroup - 1) / klay::kGroup) * 64 * p.vec;
}

// One channel a lane after all, for arrays that two at once do not fit.
void narrow(ScanPlan* p, const klay_scan_args* a) {
    p->vec = 1;
    p->blocks_c = (a->channels + 63) / 64;
    p->chains = p->blocks_c * a->batch;
}

klay::ScanArgs scan_args(const klay_scan_args* a, const ScanPlan& p, void* workspace) {
    klay::ScanArgs g{};
    g.a = a->gates; g.x = a->inputs;
    g.initial = a->initial;
    g.rows = a->offsets ? a->row_info : nullptr;
    g.a_batch = a->gates_batch_stride; g.a_time = a->gates_time_stride;
    g.x_batch = a->inputs_batch_stride; g.x_time = a->inputs_time_stride;
    g.time = a->time;
    g.channels = a->channels;
    g.blocks_c = p.blocks_c;
    g.chains = (int32_t)p.chains; g.tiles = (int32_t)p.tiles;
    if (p.tiles > 0) {
        g.ticket = static_cast<uint32_t*>(workspace);
        g.words = static_cast<uint64_t*>(workspace) + 2;
        g.state_words = g.words + map_words(p);
    }
    return g;
}

template <int S, typename T, int VC, int W>
klay_status run_scan(const klay::ScanArgs& g, const ScanPlan& p, bool back, void* stream) {
    const dim3 block(64, W), grid((uint32_t)(p.tiles > 0 ? p.chains * p.tiles : p.chains));
    if constexpr (W == 8 && (VC == 1 || sizeof(T) == 2)) {
        if (p.tiles > 0) {
            if constexpr (S != klay::SEMI_MAX)
                if (back) {
                    KLAY_LAUNCH((klay::scan_back_chain_kernel<S, T, VC, W>), grid, block, stream, g);
                    return KLAY_OK;
                }
            KLAY_LAUNCH((klay::scan_chain_kernel<S, T, VC, W>), grid, block, stream, g);
            return KLAY_OK;
        }
    }
    if constexpr (S != klay::SEMI_MAX)
        if (back) {
            KLAY_LAUNCH((klay::scan_back_kernel<S, T, VC, W>), grid, block, stream, g);
            return KLAY_OK;
        }
    KLAY_LAUNCH((klay::scan_kernel<S, T, VC, W>), grid, block, stream, g);
    return KLAY_OK;
}

template <int S, typename T, int VC>
klay_status run_scan(const klay::ScanArgs& g, const ScanPlan& p, bool back, void* stream) {
    // (a grid times its block has to stay below 2^32 threads; tiles do by their plan)
    if (p.tiles == 0 && p.chains * 64 * p.waves > (int64_t)UINT32_MAX)
        return fail(KLAY_EINVAL, "klay_scan: batch times channels exceeds one launch");
    if (p.waves == 1) return run_scan<S, T, VC, 1>(g, p, back, stream);
    if (p.waves == 4) return run_scan<S, T, VC, 4>(g, p, back, stream);
    return run_scan<S, T, VC, 8>(g, p, back, stream);
}

klay_status run_scan(const klay_scan_args* a, const klay::ScanArgs& g, const ScanPlan& p, bool back, void* stream) {
    using namespace klay;
    if (a->semiring == KLAY_LOG) return run_scan<SEMI_LOG, f32, 1>(g, p, back, stream);
    if (a->semiring == KLAY_MAXLOG) return run_scan<SEMI_MAX, f32, 1>(g, p, back, stream);
    if (a->dtype == KLAY_F32)
        return p.vec == 2 ? run_scan<SEMI_REAL, f32, 2>(g, p, back, stream) : run_scan<SEMI_REAL, f32, 1>(g, p, back, stream);
    if (a->dtype == KLAY_BF16)
        return p.vec == 2 ? run_scan<SEMI_REAL, bf16, 2>(g, p, back, stream) : run_scan<SEMI_REAL, bf16, 1>(g, p, back, stream);
    return p.vec == 2 ? run_scan<SEMI_REAL, f16, 2>(g, p, back, stream) : run_scan<SEMI_REAL, f16, 1>(g, p, back, stream);
}

klay_status prepare_scan(const klay::PrepareArgs& g, void* stream) {
    const int64_t most = std::max(std::max(g.count, g.states_count), g.words_count);
    if (most > 0) KLAY_LAUNCH(klay::scan_prepare_kernel, dim3((uint32_t)std::min<int64_t>((most + 255) / 256, 4096)), dim3(256), stream, g);
    return KLAY_OK;
}

klay_status scan_workspace(const klay_scan_args* a, const ScanPlan& p, const void* workspace, size_t bytes, const char* who) {
    const size_t need = (size_t)scan_words(p) * sizeof(uint64_t);
    if (need && (!workspace || bytes < need))
        return fail(KLAY_ENOMEM, std::string(who) + ": workspace too small: need " + std::to_string(need) + " bytes");
    if (need && reinterpret_cast<uintptr_t>(workspace) % 16)
        return fail(KLAY_EINVAL, std::string(who) + ": workspace must be 16-byte aligned");
    return KLAY_OK;
}

template <int S, typename T>
klay_status run_step(const klay::StepArgs& g, bool wide, void* stream) {
    constexpr int VC = 4;
    const int64_t lanes = wide ? g.channels / VC : g.channels;
    const int64_t across = (lanes + 255) / 256;                                       // (a workgroup takes every grid.y-th row)
    const dim3 grid((uint32_t)across, (uint32_t)std::min<int64_t>(g.batch, std::max<int64_t>(65535 / across, 1)));
    if (wide) KLAY_LAUNCH((klay::step_kernel<S, T, VC>), grid, dim3(256), stream, g);
    else KLAY_LAUNCH((klay::step_kernel<S, T, 1>), grid, dim3(256), stream, g);
    return KLAY_OK;
}

}  // namespace

extern "C" {

size_t klay_tokens_workspace_bytes(const klay_tokens_args* a) {
    if (!a || a->rows < 1 || a->vocab < 1 || !known_dtype(a->dtype) || a->top < 0) return 0;
    const int32_t parts = a->vocab <= kShortRow ? 1 : forward_plan(a).parts;
    return parts == 1 ? 0 : token_lists_at(a->rows, parts) + (size_t)a->rows * parts * a->top * sizeof(uint64_t);
}

klay_status klay_tokens_forward(const klay_tokens_args* a, float* logp, float* neg, float* entropy, float* stats, float* top_logp,
                                int64_t* top_tokens, void* workspace, size_t workspace_bytes, void* stream) try {
    const klay_status st = check_tokens(a, "klay_tokens_forward");
    if (st != KLAY_OK || a->rows == 0) return st;
    if ((a->num_tokens > 0 && !logp) || (a->top > 0 && (!top_logp || !top_tokens)))
        return fail(KLAY_EINVAL, "klay_tokens_forward: null argument");
    klay::TokenArgs g = token_args(a);
    const TokenPlan plan = a->vocab <= kShortRow ? TokenPlan() : forward_plan(a);
    g.parts = plan.parts; g.part = plan.part;
    const size_t need = klay_tokens_workspace_bytes(a);
    if (need && (!workspace || workspace_bytes < need))
        return fail(KLAY_ENOMEM, "klay_tokens_forward: workspace too small: need " + std::to_string(need) + " bytes");
    if (need && reinterpret_cast<uintptr_t>(workspace) % 16)
        return fail(KLAY_EINVAL, "klay_tokens_forward: workspace must be 16-byte aligned");
    g.logp = logp; g.neg = neg; g.entropy = entropy;
    g.stats = reinterpret_cast<klay::RowStats*>(stats);
    g.top_logp = top_logp; g.top_tokens = top_tokens;
    g.partial = static_cast<float*>(workspace);
    g.lists = need ? reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + token_lists_at(a->rows, g.parts)) : nullptr;
    OnDevice on(a->device);
    KLAY_HIP(on.status);
    if (a->dtype == KLAY_F32) return run_tokens<klay::f32>(g, plan.threads, stream);
    if (a->dtype == KLAY_BF16) return run_tokens<klay::bf16>(g, plan.threads, stream);
    return run_tokens<klay::f16>(g, plan.threads, stream);
} catch (const std::bad_alloc&) {
    return fail(KLAY_ENOMEM, "klay_tokens_forward: out of host memory");
}

klay_status klay_tokens_backward(const klay_tokens_args* a, const float* stats, const float* dlogp, const float* dneg,
                                 const float* dentropy, void* dlogits, void* stream) try {
    const klay_status st = check_tokens(a, "klay_tokens_backward");
    if (st != KLAY_OK || a->rows == 0) return st;
    if (!stats || !dlogits) return fail(KLAY_EINVAL, "klay_tokens_backward: null argument");
    if (dlogits == a->logits) return fail(KLAY_EINVAL, "klay_tokens_backward: dlogits must not be the logits, which are read again");
    klay::TokenArgs g = token_args(a);
    const TokenPlan plan = a->vocab <= kShortRow ? TokenPlan() : backward_plan(a);
    g.parts = plan.parts; g.part = plan.part;
    g.stats = const_cast<klay::RowStats*>(reinterpret_cast<const klay::RowStats*>(stats));
    g.dlogp = dlogp; g.dneg = dneg; g.dentropy = dentropy;
    g.dlogits = dlogits;
    OnDevice on(a->device);
    KLAY_HIP(on.status);
    if (a->dtype == KLAY_F32) return run_tokens_back<klay::f32>(g, plan.threads, stream);
    if (a->dtype == KLAY_BF16) return run_tokens_back<klay::bf16>(g, plan.threads, stream);
    return run_tokens_back<klay::f16>(g, plan.threads, stream);
} catch (const std::bad_alloc&) {
    return fail(KLAY_ENOMEM, "klay_tokens_backward: out of host memory");
}

size_t klay_scan_workspace_bytes(const klay_scan_args* a) {
    if (!a || a->batch < 1 || a->time < 1 || a->channels < 1 || !known_dtype(a->dtype)) return 0;
    return (size_t)scan_words(scan_plan(a)) * sizeof(uint64_t);
}

klay_status klay_scan_forward(const klay_scan_args* a, void* states, float* final, void* workspace, size_t workspace_bytes, void* stream) try {
    klay_status st = check_scan(a, true, "klay_scan_forward");
    if (st != KLAY_OK) return st;
    const int64_t sequences = a->offsets ? a->sequences : a->batch;
    const bool rows = a->batch > 0 && a->time > 0;
    if (rows && !states) return fail(KLAY_EINVAL, "klay_scan_forward: null argument");
    if (final && final == a->initial) return fail(KLAY_EINVAL, "klay_scan_forward: final must not be initial, which is read again");
    ScanPlan p = rows ? scan_plan(a) : ScanPlan();
    st = scan_workspace(a, p, workspace, workspace_bytes, "klay_scan_forward");
    if (st != KLAY_OK) return st;
    OnDevice on(a->device);
    KLAY_HIP(on.status);
    klay::PrepareArgs prepare{};
    prepare.none = a->semiring == KLAY_REAL ? 0.0f : -INFINITY;
    if (final && (a->offsets || !rows)) {
        prepare.states = final;
        prepare.from = a->initial;
        prepare.states_count = sequences * a->channels;
    }
    if (rows && a->offsets) {
        prepare.rows = a->row_info;
        prepare.offsets = a->offsets;
        prepare.count = a->time;
        prepare.sequences = (int32_t)a->sequences;
    }
    prepare.words = static_cast<uint64_t*>(workspace);
    prepare.words_count = scan_words(p);
    st = prepare_scan(prepare, stream);
    if (st != KLAY_OK || !rows) return st;
    if (!aligned_to(2 * dtype_bytes(a->dtype), {states})) narrow(&p, a);
    klay::ScanArgs g = scan_args(a, p, workspace);
    g.out = states;
    g.final = final;
    return run_scan(a, g, p, false, stream);
} catch (const std::bad_alloc&) {
    return fail(KLAY_ENOMEM, "klay_scan_forward: out of host memory");
}

klay_status klay_scan_backward(const klay_scan_args* a, const void* states, const void* dstates, const float* dfinal, void* dgates,
                               void* dinputs, float* dinitial, void* workspace, size_t workspace_bytes, void* stream) try {
    klay_status st = check_scan(a, a && a->semiring == KLAY_LOG, "klay_scan_backward");
    if (st != KLAY_OK) return st;
    if (a->semiring == KLAY_MAXLOG) return fail(KLAY_EINVAL, "klay_scan_backward: the (max, +) semiring is not differentiated");
    const int64_t sequences = a->offsets ? a->sequences : a->batch;
    const bool rows = a->batch > 0 && a->time > 0;
    if (rows && !states) return fail(KLAY_EINVAL, "klay_scan_backward: null argument");
    if ((dinitial && dinitial == dfinal) || (rows && (dgates == states || dinputs == states)))
        return fail(KLAY_EINVAL, "klay_scan_backward: dinitial must not be dfinal, nor dgates or dinputs the states, which are read again");
    ScanPlan p = rows ? scan_plan(a) : ScanPlan();
    st = scan_workspace(a, p, workspace, workspace_bytes, "klay_scan_backward");
    if (st != KLAY_OK) return st;
    OnDevice on(a->device);
    KLAY_HIP(on.status);
    klay::PrepareArgs prepare{};
    if (dinitial && (a->offsets || !rows)) {
        prepare.states = dinitial;
        prepare.from = dfinal;
        prepare.states_count = sequences * a->channels;
    }
    prepare.words = static_cast<uint64_t*>(workspace);
    prepare.words_count = scan_words(p);
    st = prepare_scan(prepare, stream);
    if (st != KLAY_OK || !rows) return st;
    if (!aligned_to(2 * dtype_bytes(a->dtype), {states, dstates, dgates, dinputs})) narrow(&p, a);
    klay::ScanArgs g = scan_args(a, p, workspace);
    g.h = states;
    g.dh = dstates;
    g.dfinal = dfinal;
    g.da = dgates; g.dx = dinputs;
    g.dinitial = dinitial;
    return run_scan(a, g, p, true, stream);
} catch (const std::bad_alloc&) {
    return fail(KLAY_ENOMEM, "klay_scan_backward: out of host memory");
}

klay_status klay_scan_step(int32_t dtype, int32_t semiring, int32_t device, int64_t rows, int32_t channels, const void* gates,
                           int64_t gates_stride, const void* inputs, int64_t inputs_stride, float* state, int64_t state_stride, void* out,
                           int64_t out_stride, void* stream) try {
    if (!known_dtype(dtype)) return fail(KLAY_EINVAL, "klay_scan_step: unknown dtype");
    if (semiring != KLAY_REAL && semiring != KLAY_LOG && semiring != KLAY_MAXLOG) return fail(KLAY_EINVAL, "klay_scan_step: unknown semiring");
    if (semiring != KLAY_REAL && dtype != KLAY_F32) return fail(KLAY_EINVAL, "klay_scan_step: the log-domain semirings take KLAY_F32 only");
    if (rows < 0 || rows > INT32_MAX || channels < 1 || channels > kMostChannels)
        return fail(KLAY_EINVAL, "klay_scan_step: rows must be 0 .. 2^31 - 1, channels 1 .. 2^25");
    if (rows == 0) return KLAY_OK;
    if (!gates || !inputs || !state) return fail(KLAY_EINVAL, "klay_scan_step: null argument");
    klay::StepArgs g{gates, inputs, out, state, gates_stride, inputs_stride, out_stride, state_stride, (int32_t)rows, channels};
    const bool wide = channels % 4 == 0;
    OnDevice on(device);
    KLAY_HIP(on.status);
    if (semiring == KLAY_LOG) return run_step<klay::SEMI_LOG, klay::f32>(g, wide, stream);
    if (semiring == KLAY_MAXLOG) return run_step<klay::SEMI_MAX, klay::f32>(g, wide, stream);
    if (dtype == KLAY_F32) return run_step<klay::SEMI_REAL, klay::f32>(g, wide, stream);
    if (dtype == KLAY_BF16) return run_step<klay::SEMI_REAL, klay::bf16>(g, wide, stream);
    return run_step<klay::SEMI_REAL, klay::f16>(g, wide, stream);
} catch (const std::bad_alloc&) {
    return fail(KLAY_ENOMEM, "klay_scan_step: out of host memory");
}

}  // extern "C"
