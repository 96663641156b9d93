// Entry points of the losses that take a network's head along (klay_head_*), and of the divergence from a teacher's list (klay_distill_*).
#include "klay_distill.hip.h"
#include "klay_entry.h"
#include "klay_head_rows.hip.h"

#include <algorithm>
#include <new>

namespace {

using klay::report;
using klay::RowMap;

constexpr int64_t kMostRows = 1 << 20, kMostWidth = 1 << 20;     // strides of copies and of the adjoints stay below klay::kMostStride
constexpr int32_t kMostVocab = INT32_MAX - 4096;                 // a tile's columns stay below 2^31
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t tiles(int64_t x, int64_t by) { return (x + by - 1) / by; }
RowMap map_of(const klay_rows& r) { return RowMap{r.outer_stride, r.inner_stride, (int32_t)std::max<int64_t>(r.inner, 1)}; }

// ---- what a forward call keeps of its rows ----------------------------------------------------------------------------
struct Kept {
    float* stats = nullptr;
    int32_t *sorted = nullptr, *slots = nullptr;
    float* values = nullptr;
};
size_t kept_bytes(int64_t rows, int32_t num_tokens) { return (size_t)rows * (klay::kRowFloats + 3 * (size_t)num_tokens) * 4; }
Kept kept_at(void* p, int64_t rows, int32_t num_tokens) {
    Kept k;
    const int64_t each = rows * num_tokens;
    k.stats = static_cast<float*>(p);
    k.sorted = reinterpret_cast<int32_t*>(k.stats + rows * klay::kRowFloats);
    k.slots = k.sorted + each;
    k.values = reinterpret_cast<float*>(k.slots + each);
    return k;
}

// ---- checks ------------------------------------------------------------------------------------------------------------
bool bad_rows(const klay_rows& r) { return r.inner < 1 || r.inner > INT32_MAX; }

klay_status check_head(const klay_head_args* a, const char* who) {
    auto refused = [who](const std::string& why) { return report(KLAY_EINVAL, who + (": " + why)); };
    if (!a) return refused("null argument");
    if (!klay::known_dtype(a->dtype)) return refused("unknown dtype");
    if (a->vocab < 1 || a->vocab > kMostVocab || a->num_tokens < 0 || a->num_tokens > klay::kMaxListed)
        return refused("vocab must be 1 .. " + std::to_string(kMostVocab) + " and num_tokens 0 .. " + std::to_string(klay::kMaxListed));
    if (a->width < 1 || a->width > kMostWidth || a->rows < 0 || a->rows > kMostRows) return refused("width must be 1 .. 2^20, rows 0 .. 2^20");
    if (a->rows == 0) return KLAY_OK;
    if (!a->hidden || !a->weight || (a->num_tokens > 0 && !a->tokens)) return refused("null argument");
    if (bad_rows(a->hidden_rows) || (a->num_tokens > 0 && bad_rows(a->token_rows))) return refused("the inner axis of rows must be 1 .. 2^31 - 1");
    if (a->weight_stride < 0) return refused("weight_stride must not be negative");
    return KLAY_OK;
}
klay_status check_teacher(const klay_teacher* t, int64_t rows, int32_t num_tokens, const char* who) {
    auto refused = [who](const std::string& why) { return report(KLAY_EINVAL, who + (": " + why)); };
    if (!t) return refused("null argument");
    if (!(t->temperature >= 1e-3 && t->temperature <= 1e3)) return refused("temperature must be 0.001 .. 1000");
    if (rows == 0) return KLAY_OK;
    if (num_tokens < 1) return refused("a teacher lists at least one token");
    if (!t->logits) return refused("null argument");
    if (bad_rows(t->rows)) return refused("the inner axis of rows must be 1 .. 2^31 - 1");
    return KLAY_OK;
}
klay_status check_distill(const klay_tokens_args* a, const klay_teacher* t, const char* who) {
    auto refused = [who](const std::string& why) { return report(KLAY_EINVAL, who + (": " + why)); };
    if (!a) return refused("null argument");
    if (!klay::known_dtype(a->dtype)) return refused("unknown dtype");
    if (a->top != 0) return refused("top must be 0");
    if (a->vocab < 1 || a->num_tokens < 0 || a->num_tokens > klay::kMaxListed)
        return refused("vocab must be >= 1 and num_tokens 0 .. " + std::to_string(klay::kMaxListed));
    if (a->rows < 0 || a->rows > INT32_MAX) return refused("rows must be 0 .. 2^31 - 1");
    const klay_status st = check_teacher(t, a->rows, a->num_tokens, who);
    if (st != KLAY_OK || a->rows == 0) return st;
    if (!a->logits || !a->tokens) return refused("null argument");
    if (bad_rows(a->logit_rows) || bad_rows(a->token_rows)) return refused("the inner axis of rows must be 1 .. 2^31 - 1");
    return KLAY_OK;
}
klay_status check_memory(const void* p, size_t bytes, size_t need, const char* what, const char* who) {
    if (need && (!p || bytes < need)) return report(KLAY_ENOMEM, std::string(who) + ": " + what + " too small: need " + std::to_string(need) + " bytes");
    if (need && reinterpret_cast<uintptr_t>(p) % 16) return report(KLAY_EINVAL, std::string(who) + ": " + what + " must be 16-byte aligned");
    return KLAY_OK;
}

// ---- plans -------------------------------------------------------------------------------------------------------------
struct Sizes {
    int64_t bytes, lot;                     // of an element; elements of 16 bytes
    explicit Sizes(int32_t dtype) : bytes(klay::dtype_bytes(dtype)), lot(16 / bytes) {}
};

// Rows that the products can read where they are: one stride, starts at multiples of 4 bytes.
bool direct(const void* p, const klay_rows& rows, int64_t count, int64_t width, const Sizes& s) {
    if (reinterpret_cast<uintptr_t>(p) % 4) return false;
    if (count == 1) return width * s.bytes % 4 == 0;
    return rows.inner >= count && rows.inner_stride >= width && rows.inner_stride * s.bytes % 4 == 0 && rows.inner_stride * s.bytes <= klay::kMostStride;
}

// The largest tile of which there are three for four CUs; the smaller ones only where there are rows for more than one.
klay::HeadTile logits_tile(int64_t rows, int64_t columns) {
    const auto count = [&](klay::HeadTile t) { return tiles(rows, klay::kTileSizes[t].rows) * tiles(columns, klay::kTileSizes[t].columns); };
    for (klay::HeadTile t : {klay::TILE_256, klay::TILE_128, klay::TILE_64})
        if (rows > klay::kTileSizes[t].rows / 2 && count(t) >= 192) return t;
    return rows > 32 && count(klay::TILE_32) > 4 * klay::kComputeUnits ? klay::TILE_64 : klay::TILE_32;
}

struct ProductPlan {
    klay::HeadTile tile;
    int32_t splits;
};
// The largest tile of which there are as many as CUs, its stages shared out where need be, at least eight each.
klay::HeadTile product_tile(int64_t rows, int64_t columns, int64_t stages) {
    if (rows <= 32) return klay::TILE_32;
    if (rows <= 64) return klay::TILE_64;
    const int64_t large = tiles(rows, klay::kTileSizes[klay::TILE_256].rows) * tiles(columns, klay::kTileSizes[klay::TILE_256].columns);
    return rows > 128 && columns > 128 && large * std::min<int64_t>(stages / 8, 8) >= 192 ? klay::TILE_256 : klay::TILE_128;
}
ProductPlan product_plan(klay::HeadTile tile, int64_t rows, int64_t columns, int64_t stages) {
    const int64_t count = tiles(rows, klay::kTileSizes[tile].rows) * tiles(columns, klay::kTileSizes[tile].columns);
    const int64_t want = tile == klay::TILE_256 ? klay::kComputeUnits : 2 * klay::kComputeUnits;
    return ProductPlan{tile, (int32_t)std::max<int64_t>(1, std::min<int64_t>({want / count, stages / 8, 32}))};
}

constexpr int64_t kRowBlock = 16384;        // rows whose tiles' sums are held at a time, at most
constexpr int64_t kMostSums = 1 << 22;      // such sums of 16 bytes, of more than one tile of rows: 16384 tiles of 256 x 256, 64 for every compute unit
constexpr int64_t kPieceElements = 1 << 25; // adjoints of logits that are held at a time, about: 128 MB
// Bytes of weights that are copied with the hidden states, which saves a launch: longer ones cost more than that (backward of 256 rows of 1024 features in
// bf16, in a graph, copied / only if need be: 1 MB 38.5 / 38.6 us, 2 MB 43.6 / 41.9, 4 MB 48.1 / 45.0, 8 MB 53.5 / 49.1).
constexpr int64_t kSmallCopy = 1 << 20;
// Up to here (rows x width x tokens) the two products are one launch, by the smaller of the tiles that they would take alone: a launch less, and as fast or
// faster (32 x 1024 x 8192 bf16 40.2 us, 43.0 in two; 2^26 to 2^30 terms of 64 to 512 rows within 1%); beyond, the smaller tiles cost more (16 x 4096 x 16384
// 159.8 us, 103.2 in two).
constexpr int64_t kSmallProduct = 1ll << 30;

struct HeadPlan {
    bool copy_hidden = false, copy_weight = false;
    int64_t padded = 0;                     // elements of a copied row
    int64_t row_block = 0, tiles_n = 0;
    klay::HeadTile tile = klay::TILE_32;
    // backward
    int64_t piece = 0;
    int64_t cut = 1;                        // numbers of the operands' type that an adjoint is held in
    ProductPlan dh{}, dw{};
    // bytes from the start of the workspace
    size_t hidden = 0, weight = 0, partial = 0, kept = 0, coefs = 0, entries = 0, largest = 0, g = 0, clean_hidden = 0, clean_weight = 0,
           dh_sums = 0, dw_sums = 0, db_sums = 0, bytes = 0;
};
int64_t stages_of(int64_t elements, const Sizes& s) { return tiles(elements * s.bytes, klay::kMostStageBytes); }

// Adjoints of 16-bit heads are held in two numbers of the type as the products' operands, the second, of what the first's rounding leaves, as rows of its own:
// rounded once they would make as large an error as the results' own rounding, and of few entries (one of a row's own tokens, mostly) or equal ones 1.5 times
// it.  It costs what products of twice the terms cost (bf16, a step of training of 4096 features and 131072 tokens, with / without: 16 rows 863 / 856 us, 64
// 1132 / 883, 512 3211 / 2302, 4096 22.2 / 14.7 ms).
int64_t cut_of(const Sizes& s) { return s.bytes == 2 ? 2 : 1; }

HeadPlan head_plan(const klay_head_args* a, bool back) {
    const Sizes s(a->dtype);
    HeadPlan p;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const klay_rows weight_rows{INT64_MAX, 0, a->weight_stride};
    p.copy_hidden = !direct(a->hidden, a->hidden_rows, a->rows, a->width, s);
    p.copy_weight = !direct(a->weight, weight_rows, a->vocab, a->width, s);
    p.padded = up(a->width, s.lot);
    if (p.copy_hidden) p.hidden = take(a->rows * p.padded * s.bytes);
    if (p.copy_weight) p.weight = take(a->vocab * p.padded * s.bytes);
    const int64_t asked = a->rows * a->num_tokens;
    if (!back) {
        const auto block = [&](int64_t rows) {
            p.row_block = rows;
            p.tile = logits_tile(rows, a->vocab);
            p.tiles_n = tiles(a->vocab, klay::kTileSizes[p.tile].columns);
        };
        block(std::min(a->rows, kRowBlock));
        if (p.row_block > 256 && p.row_block * p.tiles_n > kMostSums) block(std::max<int64_t>(256, kMostSums / p.tiles_n / 256 * 256));
        p.partial = take(p.row_block * p.tiles_n * sizeof(float4));
        p.kept = take(kept_bytes(a->rows, a->num_tokens));
    } else {
        const int64_t all = up(a->vocab, 256);
        p.piece = std::min(all, std::max<int64_t>(256, kPieceElements / up(a->rows, 256) / 256 * 256));
        const int64_t columns = up(std::min<int64_t>(p.piece, a->vocab), 8);
        p.cut = cut_of(s);
        const int64_t rows = p.cut * a->rows;       // of the adjoints
        p.tile = logits_tile(a->rows, columns);
        p.coefs = take(a->rows * sizeof(float4));
        p.entries = take(asked * 4);
        p.largest = take(8);
        p.g = take(rows * columns * s.bytes);
        p.clean_hidden = take(rows * p.padded * s.bytes);
        // (Room for the piece's weights, of few rows all weights.  In pieces of 256 MB of them steps cost more: 16 x 4096 x 131072 bf16 680 / 761 us, 256 rows 1482 /
        // 1670, 16 x 4096 x 65536 fp32 688 / 894.)
        if (a->bias) p.clean_weight = take(columns * p.padded * s.bytes);
        const int64_t dw_rows = std::min<int64_t>(p.piece, a->vocab), dh_stages = stages_of(columns, s), dw_stages = stages_of(rows, s);
        klay::HeadTile dh = product_tile(rows, a->width, dh_stages), dw = product_tile(dw_rows, a->width, dw_stages);
        if (a->rows * a->width * dw_rows < kSmallProduct) dh = dw = std::min(dh, dw);
        else if (dw_stages == 1 && dw_rows > 64) dw = klay::TILE_ONE;      // (always a single sum, stored as it is)
        p.dh = product_plan(dh, rows, a->width, dh_stages);
        p.dw = product_plan(dw, dw_rows, a->width, dw_stages);
        p.dh_sums = take(p.dh.splits * rows * a->width * 4);
        p.dw_sums = take(p.dw.splits == 1 ? 0 : p.dw.splits * columns * a->width * 4);
        p.db_sums = take(tiles(a->rows, klay::kTileSizes[p.tile].rows) * columns * 4);
    }
    p.bytes = at;
    return p;
}

klay::ListArgs list_args(const int64_t* tokens, const klay_rows& rows, int64_t stride, int64_t count, int32_t num_tokens, int32_t vocab) {
    klay::ListArgs l{};
    l.tokens = tokens;
    l.token_rows = map_of(rows);
    l.token_stride = stride;
    l.rows = count;
    l.num_tokens = num_tokens;
    l.vocab = vocab;
    return l;
}
klay::TeachArgs teach_args(const klay_teacher* t) {
    klay::TeachArgs g{};
    g.teacher = t->logits;
    g.teacher_rows = map_of(t->rows);
    g.teacher_stride = t->stride;
    g.inverse_temperature = 1.0 / t->temperature;
    g.rest = t->rest != 0;
    return g;
}
float scale_of(const klay_teacher* t) { return t ? (float)(1.4426950408889634 / t->temperature) : klay::kTokLog2e; }
void* in(void* workspace, size_t at) { return static_cast<char*>(workspace) + at; }
#define KLAY_DO(call)                          \
    do {                                       \
        const klay_status st__ = (call);       \
        if (st__ != KLAY_OK) return st__;      \
    } while (0)

template <typename T> struct Head {
    const klay_head_args* a;
    HeadPlan p;
    void* workspace;
    void* stream;
    Sizes s{0};
    klay::Operand hidden{}, weight{};
    Head(const klay_head_args* args, const HeadPlan& plan, void* w, void* on) : a(args), p(plan), workspace(w), stream(on), s(args->dtype) {}

    klay::PackArgs copy(const void* from, const klay_rows& rows, int64_t count) const {
        klay::PackArgs g{};
        g.from = from;
        g.outer = rows.outer_stride;
        g.inner_stride = rows.inner_stride;
        g.inner = std::max<int64_t>(rows.inner, 1);
        g.count = count;
        g.columns = a->width;
        return g;
    }
    klay_rows weight_rows() const { return klay_rows{INT64_MAX, 0, a->weight_stride}; }
    // the operands as the products take them
    klay::PacksArgs packs{};
    klay::PackArgs& pack(const void* from, const klay_rows& rows, int64_t count, size_t to) {
        klay::PackArgs& c = packs.copy[packs.copies++];
        c = copy(from, rows, count);
        c.padded = p.padded;
        c.to = in(workspace, to);
        return c;
    }
    klay_status run_packs() {
        const klay_status st = klay::HeadLaunch<T>::pack(packs, stream);
        packs = klay::PacksArgs{};
        return st;
    }
    // The operands as the products take them, their copies among `packs`.  (Where only one is copied, the other's rows have no zeros behind
    // their ends: both are read as if they had none.)
    int32_t tail = 0;
    void operands() {
        const bool padded = p.copy_hidden && p.copy_weight;
        const int32_t pieces = (int32_t)(padded ? p.padded / s.lot : a->width / s.lot);
        tail = padded ? 0 : (int32_t)(a->width % s.lot);
        hidden = klay::Operand{a->hidden, (a->rows == 1 ? a->width : a->hidden_rows.inner_stride) * s.bytes, a->rows, pieces};
        weight = klay::Operand{a->weight, (a->vocab == 1 ? a->width : a->weight_stride) * s.bytes, a->vocab, pieces};
        if (p.copy_hidden) {
            hidden.p = pack(a->hidden, a->hidden_rows, a->rows, p.hidden).to;
            hidden.stride = p.padded * s.bytes;
        }
        if (p.copy_weight) {
            weight.p = pack(a->weight, weight_rows(), a->vocab, p.weight).to;
            weight.stride = p.padded * s.bytes;
        }
    }
    klay::HeadArgs args(const Kept& kept) const {
        klay::HeadArgs g{};
        g.hidden = hidden;
        g.weight = weight;
        g.bias = a->bias;
        g.tail = tail;
        g.rows = a->rows;
        g.num_tokens = a->num_tokens;
        g.sorted = kept.sorted;
        return g;
    }

    klay_status forward(const klay_teacher* teacher, const Kept& kept, bool stats, float* logp, float* neg, float* entropy, float* loss) {
        klay::ListArgs lists = list_args(a->tokens, a->token_rows, a->token_stride, a->rows, a->num_tokens, a->vocab);
        lists.sorted = kept.sorted;
        lists.slots = kept.slots;
        if (a->num_tokens > 1) KLAY_LAUNCH(klay::head_lists_kernel, dim3((uint32_t)tiles(a->rows, 4)), dim3(256), stream, lists);
        operands();
        KLAY_DO(run_packs());
        const float scale = scale_of(teacher);
        for (int64_t r0 = 0; r0 < a->rows; r0 += p.row_block) {
            const int64_t rows = std::min(p.row_block, a->rows - r0), at = r0 * a->num_tokens;
            klay::HeadArgs g = args(kept);
            g.hidden.p = static_cast<const char*>(g.hidden.p) + r0 * g.hidden.stride;
            g.hidden.rows = g.rows = rows;
            g.scale = scale;
            g.sorted = a->num_tokens > 1 ? g.sorted + at : nullptr;
            g.list = lists;
            g.list_row = r0;
            g.values = kept.values + at;
            g.partial = static_cast<float4*>(in(workspace, p.partial));
            KLAY_DO(klay::HeadLaunch<T>::forward(p.tile, g, !teacher && (entropy || stats), stream));
            const klay::FinishArgs f{g.partial, p.tiles_n, rows, a->num_tokens, scale, kept.sorted + at, kept.slots + at, g.values, lists, r0};
            const dim3 grid((uint32_t)tiles(rows, 4));
            if (teacher) {
                klay::TeachArgs t = teach_args(teacher);
                t.first = r0;
                t.loss = loss + r0;
                t.stats = stats ? kept.stats + r0 * klay::kRowFloats : nullptr;
                t.moved = stats ? g.values : nullptr;
                KLAY_LAUNCH(klay::head_distill_finish_kernel, grid, dim3(256), stream, f, t);
            } else {
                const klay::RowOut out{logp ? logp + at : nullptr, neg ? neg + at : nullptr, entropy ? entropy + r0 : nullptr,
                                       stats ? kept.stats + r0 * klay::kRowFloats : nullptr};
                KLAY_LAUNCH(klay::head_logprobs_finish_kernel, grid, dim3(256), stream, f, out);
            }
        }
        return KLAY_OK;
    }

    klay_status backward(const klay_teacher* teacher, const Kept& kept, const float* dlogp, const float* dneg, const float* dentropy, const float* dloss,
                         void* dhidden, void* dweight, float* dbias);
};

template <typename T>
klay_status Head<T>::backward(const klay_teacher* teacher, const Kept& kept, const float* dlogp, const float* dneg, const float* dentropy,
                              const float* dloss, void* dhidden, void* dweight, float* dbias) {
    klay::AdjointArgs ad{};
    ad.stats = kept.stats;
    ad.sorted = kept.sorted;
    ad.slots = kept.slots;
    ad.values = kept.values;
    ad.dlogp = dlogp; ad.dneg = dneg; ad.dentropy = dentropy; ad.dloss = dloss;
    ad.inverse_temperature = teacher ? (float)(1.0 / teacher->temperature) : 1.0f;
    ad.rows = a->rows;
    ad.num_tokens = a->num_tokens;
    ad.coefs = static_cast<float4*>(in(workspace, p.coefs));
    ad.entries = static_cast<float*>(in(workspace, p.entries));
    operands();
    uint32_t* const words = static_cast<uint32_t*>(in(workspace, p.largest));
    if (a->dtype == KLAY_F16) ad.largest = words;
    // A row without a gradient gives none, whatever it holds: its adjoints are zeros, so that only what is not finite has to go.  (In a row that has one
    // the logits, and with them the adjoints, are NaN then.)
    for (int64_t i = 0; dweight && i < p.cut; ++i) pack(a->hidden, a->hidden_rows, a->rows, p.clean_hidden + i * a->rows * p.padded * s.bytes).finite = 1;
    // Nor does a token that the bias bars, whatever its weights hold.  Few weights are copied along; many only if the adjoints' launch has found something in
    // them that is not finite, since that would be as much to read and write as the products have.
    const bool whole = p.piece >= a->vocab;             // one piece
    const bool few = whole && a->vocab * a->width * s.bytes <= kSmallCopy;
    uint32_t* const odd = dhidden && a->bias && !few ? words + 1 : nullptr;
    const auto clean_weights = [&](int64_t first, int64_t count) {
        pack(static_cast<const char*>(a->weight) + first * a->weight_stride * s.bytes, weight_rows(), count, p.clean_weight).bias = a->bias + first;
    };
    if (dhidden && a->bias && few) clean_weights(0, a->vocab);
    if (ad.largest || odd) packs.clear = words;
    KLAY_DO(run_packs());
    const dim3 row_grid((uint32_t)tiles(a->rows, 4));
    if (teacher) KLAY_LAUNCH(klay::head_distill_adjoint_kernel, row_grid, dim3(256), stream, ad);
    else KLAY_LAUNCH(klay::head_logprobs_adjoint_kernel, row_grid, dim3(256), stream, ad);
    klay::SumsArgs sums{};
    for (int64_t first = 0; first < a->vocab; first += p.piece) {
        const int64_t count = std::min(p.piece, a->vocab - first), columns = up(count, 8);
        klay::HeadArgs g = args(kept);
        g.weight.p = static_cast<const char*>(g.weight.p) + first * g.weight.stride;
        g.weight.rows = count;
        g.bias = a->bias ? a->bias + first : nullptr;
        g.first = (int32_t)first;
        g.scale = scale_of(teacher);
        g.coefs = ad.coefs;
        g.entries = ad.entries;
        g.largest = ad.largest;
        g.odd = odd;
        g.g = dhidden || dweight ? in(workspace, p.g) : nullptr;
        g.g_low = g.g && p.cut == 2 ? static_cast<char*>(g.g) + a->rows * columns * s.bytes : nullptr;
        g.g_columns = columns;
        g.bias_partial = dbias ? static_cast<float*>(in(workspace, p.db_sums)) : nullptr;
        KLAY_DO(klay::HeadLaunch<T>::adjoint(p.tile, g, stream));
        klay::ProductJob jobs[2] = {};
        klay::HeadTile job_tile[2];
        int n = 0;
        if (dhidden) {
            if (odd) {
                clean_weights(first, count);
                packs.only = odd;
                KLAY_DO(run_packs());
            }
            klay::ProductJob& j = jobs[n];
            job_tile[n++] = p.dh.tile;
            j.a = klay::Operand{g.g, columns * s.bytes, p.cut * a->rows, (int32_t)(columns / s.lot)};
            j.odd = odd;
            j.clean = in(workspace, p.clean_weight);
            j.clean_stride = p.padded * s.bytes;
            j.b = a->bias && few ? klay::Operand{j.clean, j.clean_stride, a->width, (int32_t)count}
                                 : klay::Operand{g.weight.p, g.weight.stride, a->width, (int32_t)count};
            j.splits = (int32_t)std::min<int64_t>(p.dh.splits, stages_of(columns, s));
            j.rows = p.cut * a->rows;
            j.columns = a->width;
            j.out = whole && j.splits * p.cut == 1 ? dhidden : nullptr;
            j.sums = static_cast<float*>(in(workspace, p.dh_sums));
            j.add = first > 0;
            const int64_t all = a->rows * a->width;
            const int32_t parts = (int32_t)((whole ? j.splits : p.dh.splits) * p.cut);
            if (first + p.piece >= a->vocab && !j.out) sums.sum[sums.sums++] = klay::SumArgs{j.sums, all, all, parts, 1, dhidden};
        }
        if (dweight) {
            klay::ProductJob& j = jobs[n];
            job_tile[n++] = p.dw.tile;
            j.a_across = 1;
            j.a = klay::Operand{g.g, columns * s.bytes, columns, (int32_t)(p.cut * a->rows)};
            j.b = klay::Operand{in(workspace, p.clean_hidden), p.padded * s.bytes, a->width, (int32_t)(p.cut * a->rows)};
            j.splits = p.dw.splits;
            j.rows = count;
            j.columns = a->width;
            void* out = static_cast<char*>(dweight) + first * a->width * s.bytes;
            j.out = j.splits == 1 ? out : nullptr;
            j.stream = a->width * s.bytes % 128 == 0 && reinterpret_cast<uintptr_t>(out) % 128 == 0;
            j.sums = static_cast<float*>(in(workspace, p.dw_sums));
            j.add = 0;
            if (!j.out) sums.sum[sums.sums++] = klay::SumArgs{j.sums, count * a->width, count * a->width, j.splits, 1, out};
        }
        if (dbias)
            sums.sum[sums.sums++] = klay::SumArgs{g.bias_partial, count, columns, (int32_t)tiles(a->rows, klay::kTileSizes[p.tile].rows), 0, dbias + first};
        for (int i = 0; i < n;) {
            klay::ProductArgs pr{};
            pr.largest = ad.largest;
            pr.job[pr.jobs++] = jobs[i];
            const klay::HeadTile tile = job_tile[i++];
            if (i < n && job_tile[i] == tile) pr.job[pr.jobs++] = jobs[i++];
            KLAY_DO(klay::HeadLaunch<T>::products(tile, pr, stream));
        }
        KLAY_DO(klay::HeadLaunch<T>::sums(sums, stream));
        sums.sums = 0;
    }
    return KLAY_OK;
}

klay_status head_forward(const klay_head_args* a, const klay_teacher* teacher, void* kept, float* logp, float* neg, float* entropy, float* loss,
                         void* workspace, size_t workspace_bytes, void* stream, const char* who) {
    const HeadPlan p = head_plan(a, false);
    KLAY_DO(check_memory(workspace, workspace_bytes, p.bytes, "workspace", who));
    if (reinterpret_cast<uintptr_t>(kept) % 16) return report(KLAY_EINVAL, std::string(who) + ": kept must be 16-byte aligned");
    klay::OnDevice on(a->device);
    if (on.status != hipSuccess) return report(KLAY_EHIP, std::string(who) + ": " + hipGetErrorString(on.status));
    const Kept k = kept_at(kept ? kept : in(workspace, p.kept), a->rows, a->num_tokens);
    if (a->dtype == KLAY_F32) return Head<klay::f32>(a, p, workspace, stream).forward(teacher, k, kept, logp, neg, entropy, loss);
    if (a->dtype == KLAY_BF16) return Head<klay::bf16>(a, p, workspace, stream).forward(teacher, k, kept, logp, neg, entropy, loss);
    return Head<klay::f16>(a, p, workspace, stream).forward(teacher, k, kept, logp, neg, entropy, loss);
}

klay_status head_backward(const klay_head_args* a, const klay_teacher* teacher, const void* kept, const float* dlogp, const float* dneg,
                          const float* dentropy, const float* dloss, void* dhidden, void* dweight, float* dbias, void* workspace,
                          size_t workspace_bytes, void* stream, const char* who) {
    if (!kept) return report(KLAY_EINVAL, std::string(who) + ": null argument");
    if (reinterpret_cast<uintptr_t>(kept) % 16) return report(KLAY_EINVAL, std::string(who) + ": kept must be 16-byte aligned");
    if ((dhidden && (dhidden == a->hidden || dhidden == a->weight)) || (dweight && (dweight == a->weight || dweight == a->hidden)) ||
        (dbias && dbias == a->bias))
        return report(KLAY_EINVAL, std::string(who) + ": a gradient must not be an input, which is read again");
    const HeadPlan p = head_plan(a, true);
    KLAY_DO(check_memory(workspace, workspace_bytes, p.bytes, "workspace", who));
    if (!dhidden && !dweight && !dbias) return KLAY_OK;
    klay::OnDevice on(a->device);
    if (on.status != hipSuccess) return report(KLAY_EHIP, std::string(who) + ": " + hipGetErrorString(on.status));
    const Kept k = kept_at(const_cast<void*>(kept), a->rows, a->num_tokens);
    if (a->dtype == KLAY_F32) return Head<klay::f32>(a, p, workspace, stream).backward(teacher, k, dlogp, dneg, dentropy, dloss, dhidden, dweight, dbias);
    if (a->dtype == KLAY_BF16) return Head<klay::bf16>(a, p, workspace, stream).backward(teacher, k, dlogp, dneg, dentropy, dloss, dhidden, dweight, dbias);
    return Head<klay::f16>(a, p, workspace, stream).backward(teacher, k, dlogp, dneg, dentropy, dloss, dhidden, dweight, dbias);
}

// ---- divergence of given logits -----------------------------------------------------------------------------------------
constexpr int64_t kManyRows = 2 * klay::kComputeUnits;
// (a launch has less than 2^32 threads; the kernels run through what is left)
uint32_t capped_grid(int64_t units) { return (uint32_t)std::min<int64_t>(units, 1 << 20); }

klay::DistillArgs distill_args(const klay_tokens_args* a, const klay_teacher* t) {
    klay::DistillArgs g{};
    g.logits = a->logits;
    g.logit_rows = map_of(a->logit_rows);
    g.list = list_args(a->tokens, a->token_rows, a->token_stride, a->rows, a->num_tokens, a->vocab);
    g.scale = scale_of(t);
    g.teach = teach_args(t);
    return g;
}
template <typename T> klay_status run_distill(const klay::DistillArgs& g, void* stream) {
    const dim3 grid(capped_grid(g.list.rows)), waves(capped_grid(tiles(g.list.rows, 4)));
    if (g.list.vocab <= klay::kShortDistill) {
        if (g.list.num_tokens <= 64) KLAY_LAUNCH((klay::distill_short_kernel<T, 64>), waves, dim3(256), stream, g);
        else KLAY_LAUNCH((klay::distill_short_kernel<T, klay::kMaxListed>), waves, dim3(256), stream, g);
    } else if (g.list.rows >= kManyRows) {
        KLAY_LAUNCH((klay::distill_row_kernel<T, 256, false>), grid, dim3(256), stream, g);
        KLAY_LAUNCH(klay::distill_finish_kernel, waves, dim3(256), stream, g);
    } else {
        KLAY_LAUNCH((klay::distill_row_kernel<T, 1024, true>), grid, dim3(1024), stream, g);
    }
    return KLAY_OK;
}
template <typename T> klay_status run_distill_back(klay::DistillArgs g, void* stream) {
    const int64_t bytes = (int64_t)g.list.vocab * sizeof(T), round = 256 * 16 / (int64_t)sizeof(T);
    int64_t parts = std::max<int64_t>((bytes + 32767) / 32768, std::min<int64_t>((4 * klay::kComputeUnits + g.list.rows - 1) / g.list.rows, (bytes + 8191) / 8192));
    int64_t size = tiles(g.list.vocab, parts);
    if (parts > 1) size = up(size, round);
    g.part = (int32_t)std::min<int64_t>(size, INT32_MAX);
    g.parts = (int32_t)tiles(g.list.vocab, size);
    const dim3 grid(capped_grid(g.list.rows * g.parts));
    if (bytes <= 4096) KLAY_LAUNCH((klay::distill_back_kernel<T, 64>), grid, dim3(64), stream, g);
    else KLAY_LAUNCH((klay::distill_back_kernel<T, 256>), grid, dim3(256), stream, g);
    return KLAY_OK;
}

}  // namespace

extern "C" {

size_t klay_list_kept_bytes(int64_t rows, int32_t num_tokens) { return rows < 1 || num_tokens < 0 ? 0 : kept_bytes(rows, num_tokens); }

size_t klay_head_workspace_bytes(const klay_head_args* a, int32_t backward) {
    if (!a || a->rows < 1 || a->rows > kMostRows || a->vocab < 1 || a->vocab > kMostVocab || a->width < 1 || a->width > kMostWidth ||
        !klay::known_dtype(a->dtype) || a->num_tokens < 0 || a->num_tokens > klay::kMaxListed)
        return 0;
    return head_plan(a, backward != 0).bytes;
}

klay_status klay_head_forward(const klay_head_args* a, float* logp, float* neg, float* entropy, void* kept, void* workspace, size_t workspace_bytes,
                              void* stream) try {
    KLAY_DO(check_head(a, "klay_head_forward"));
    if (a->rows == 0) return KLAY_OK;
    if (a->num_tokens > 0 && !logp) return report(KLAY_EINVAL, "klay_head_forward: null argument");
    return head_forward(a, nullptr, kept, logp, neg, entropy, nullptr, workspace, workspace_bytes, stream, "klay_head_forward");
} catch (const std::bad_alloc&) {
    return report(KLAY_ENOMEM, "klay_head_forward: out of host memory");
}

klay_status klay_head_backward(const klay_head_args* a, const void* kept, const float* dlogp, const float* dneg, const float* dentropy,
                               void* dhidden, void* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream) try {
    KLAY_DO(check_head(a, "klay_head_backward"));
    if (a->rows == 0) return KLAY_OK;
    return head_backward(a, nullptr, kept, dlogp, dneg, dentropy, nullptr, dhidden, dweight, dbias, workspace, workspace_bytes, stream,
                         "klay_head_backward");
} catch (const std::bad_alloc&) {
    return report(KLAY_ENOMEM, "klay_head_backward: out of host memory");
}

klay_status klay_head_distill_forward(const klay_head_args* a, const klay_teacher* teacher, float* loss, void* kept, void* workspace,
                                      size_t workspace_bytes, void* stream) try {
    KLAY_DO(check_head(a, "klay_head_distill_forward"));
    KLAY_DO(check_teacher(teacher, a->rows, a->num_tokens, "klay_head_distill_forward"));
    if (a->rows == 0) return KLAY_OK;
    if (!loss) return report(KLAY_EINVAL, "klay_head_distill_forward: null argument");
    return head_forward(a, teacher, kept, nullptr, nullptr, nullptr, loss, workspace, workspace_bytes, stream, "klay_head_distill_forward");
} catch (const std::bad_alloc&) {
    return report(KLAY_ENOMEM, "klay_head_distill_forward: out of host memory");
}

klay_status klay_head_distill_backward(const klay_head_args* a, const klay_teacher* teacher, const void* kept, const float* dloss, void* dhidden,
                                       void* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream) try {
    KLAY_DO(check_head(a, "klay_head_distill_backward"));
    KLAY_DO(check_teacher(teacher, a->rows, a->num_tokens, "klay_head_distill_backward"));
    if (a->rows == 0) return KLAY_OK;
    if (!dloss) return report(KLAY_EINVAL, "klay_head_distill_backward: null argument");
    return head_backward(a, teacher, kept, nullptr, nullptr, nullptr, dloss, dhidden, dweight, dbias, workspace, workspace_bytes, stream,
                         "klay_head_distill_backward");
} catch (const std::bad_alloc&) {
    return report(KLAY_ENOMEM, "klay_head_distill_backward: out of host memory");
}

klay_status klay_distill_forward(const klay_tokens_args* a, const klay_teacher* teacher, float* loss, void* kept, void* stream) try {
    KLAY_DO(check_distill(a, teacher, "klay_distill_forward"));
    if (a->rows == 0) return KLAY_OK;
    if (!loss || !kept) return report(KLAY_EINVAL, "klay_distill_forward: null argument");
    if (reinterpret_cast<uintptr_t>(kept) % 16) return report(KLAY_EINVAL, "klay_distill_forward: kept must be 16-byte aligned");
    klay::DistillArgs g = distill_args(a, teacher);
    g.teach.loss = loss;
    const Kept k = kept_at(kept, a->rows, a->num_tokens);
    g.teach.stats = g.sums = k.stats;
    g.teach.moved = k.values;
    g.list.sorted = k.sorted;
    g.list.slots = k.slots;
    klay::OnDevice on(a->device);
    if (on.status != hipSuccess) return report(KLAY_EHIP, std::string("klay_distill_forward: ") + hipGetErrorString(on.status));
    if (a->dtype == KLAY_F32) return run_distill<klay::f32>(g, stream);
    if (a->dtype == KLAY_BF16) return run_distill<klay::bf16>(g, stream);
    return run_distill<klay::f16>(g, stream);
} catch (const std::bad_alloc&) {
    return report(KLAY_ENOMEM, "klay_distill_forward: out of host memory");
}

klay_status klay_distill_backward(const klay_tokens_args* a, const klay_teacher* teacher, const void* kept, const float* dloss, void* dlogits,
                                  void* stream) try {
    KLAY_DO(check_distill(a, teacher, "klay_distill_backward"));
    if (a->rows == 0) return KLAY_OK;
    if (!kept || !dloss || !dlogits) return report(KLAY_EINVAL, "klay_distill_backward: null argument");
    if (reinterpret_cast<uintptr_t>(kept) % 16) return report(KLAY_EINVAL, "klay_distill_backward: kept must be 16-byte aligned");
    if (dlogits == a->logits) return report(KLAY_EINVAL, "klay_distill_backward: dlogits must not be the logits, which are read again");
    klay::DistillArgs g = distill_args(a, teacher);
    const Kept k = kept_at(const_cast<void*>(kept), a->rows, a->num_tokens);
    g.teach.stats = k.stats;
    g.teach.moved = k.values;
    g.list.sorted = k.sorted;
    g.dloss = dloss;
    g.dlogits = dlogits;
    klay::OnDevice on(a->device);
    if (on.status != hipSuccess) return report(KLAY_EHIP, std::string("klay_distill_backward: ") + hipGetErrorString(on.status));
    if (a->dtype == KLAY_F32) return run_distill_back<klay::f32>(g, stream);
    if (a->dtype == KLAY_BF16) return run_distill_back<klay::bf16>(g, stream);
    return run_distill_back<klay::f16>(g, stream);
} catch (const std::bad_alloc&) {
    return report(KLAY_ENOMEM, "klay_distill_backward: out of host memory");
}

}  // extern "C"
