// The launches of one type of a head's elements.
#pragma once

#include "klay_entry.h"
#include "klay_head.hip.h"

#include <algorithm>

namespace klay {

template <typename T> using Tile32 = Tile<T, 128, 32, 4, 1, 3, 128>;
template <typename T> using Tile64 = Tile<T, 128, 64, 4, 1, 3, 128>;
// TileOne: the weights' gradient of at most 32 rows is all writing: little shared memory, for more workgroups at a time, and in 16 bits rows of 256
// bytes a wave, past the caches where they are whole lines (16 x 4096 x 131072 bf16: 280 us; 318 through the caches, 378 by Tile128.  Rows that share lines take
// twice the time past the caches).
template <typename T> struct Large {
    typedef Tile<T, 128, 128, 2, 2, 2, 128> Tile128;
    typedef Tile<T, 256, 256, 2, 4, 2, 128> Tile256;
    typedef Tile<T, 128, 128, 1, 4, 1, 128> TileOne;
};
// fp32: six products a pair of elements, so that a quarter of the k's is as long a stage for the largest tile; the next one adds its sums half as often with
// 32 k's a stage (1183 x 3272 x 7032: 477 us, 528 with sixteen), and writes better with sixteen (20 x 3214 x 96569: 395, 447 with 32, 448 in a single stage).
template <> struct Large<f32> {
    typedef Tile<f32, 128, 128, 2, 2, 2, 128> Tile128;
    typedef Tile<f32, 256, 256, 2, 4, 2, 64> Tile256;
    typedef Tile<f32, 128, 128, 2, 2, 2, 64> TileOne;
};
template <typename T> using Tile128 = typename Large<T>::Tile128;
template <typename T> using Tile256 = typename Large<T>::Tile256;
template <typename T> using TileOne = typename Large<T>::TileOne;

template <typename Tile> Tiles tiles_of(int64_t rows, int64_t columns) {
    return Tiles{(rows + Tile::kN - 1) / Tile::kN, (columns + Tile::kM - 1) / Tile::kM};
}
inline uint32_t grid_of(int64_t items, int64_t each, int64_t most) { return (uint32_t)std::max<int64_t>(1, std::min((items + each - 1) / each, most)); }

template <typename Tile> klay_status run_forward(const HeadArgs& g, bool entropy, void* stream) {
    const Tiles tiles = tiles_of<Tile>(g.rows, g.weight.rows);
    const dim3 grid((uint32_t)(tiles.m * tiles.n)), block(Tile::kThreads);
    if (entropy) KLAY_LAUNCH((head_forward_kernel<Tile, true>), grid, block, stream, g, tiles);
    else KLAY_LAUNCH((head_forward_kernel<Tile, false>), grid, block, stream, g, tiles);
    return KLAY_OK;
}
template <typename Tile> klay_status run_adjoint(const HeadArgs& g, void* stream) {
    const Tiles tiles = tiles_of<Tile>(g.rows, g.g_columns);
    KLAY_LAUNCH((head_adjoint_kernel<Tile>), dim3((uint32_t)(tiles.m * tiles.n)), dim3(Tile::kThreads), stream, g, tiles);
    return KLAY_OK;
}
template <typename Tile> klay_status run_products(const ProductArgs& g, void* stream) {
    int64_t blocks[2] = {0, 0};
    for (int i = 0; i < g.jobs; ++i) {
        const Tiles tiles = tiles_of<Tile>(g.job[i].rows, g.job[i].columns);
        blocks[i] = tiles.m * tiles.n * g.job[i].splits;
    }
    if (blocks[0] + blocks[1] > 0)
        KLAY_LAUNCH((head_product_kernel<Tile>), dim3((uint32_t)(blocks[0] + blocks[1])), dim3(Tile::kThreads), stream, g, blocks[0]);
    return KLAY_OK;
}

template <typename T> klay_status HeadLaunch<T>::forward(HeadTile tile, const HeadArgs& g, bool entropy, void* stream) {
    switch (tile) {
        case TILE_32: return run_forward<Tile32<T>>(g, entropy, stream);
        case TILE_64: return run_forward<Tile64<T>>(g, entropy, stream);
        case TILE_128: return run_forward<Tile128<T>>(g, entropy, stream);
        default: return run_forward<Tile256<T>>(g, entropy, stream);
    }
}
template <typename T> klay_status HeadLaunch<T>::adjoint(HeadTile tile, const HeadArgs& g, void* stream) {
    switch (tile) {
        case TILE_32: return run_adjoint<Tile32<T>>(g, stream);
        case TILE_64: return run_adjoint<Tile64<T>>(g, stream);
        case TILE_128: return run_adjoint<Tile128<T>>(g, stream);
        default: return run_adjoint<Tile256<T>>(g, stream);
    }
}
template <typename T> klay_status HeadLaunch<T>::products(HeadTile tile, const ProductArgs& g, void* stream) {
    switch (tile) {
        case TILE_32: return run_products<Tile32<T>>(g, stream);
        case TILE_64: return run_products<Tile64<T>>(g, stream);
        case TILE_128: return run_products<Tile128<T>>(g, stream);
        case TILE_ONE: return run_products<TileOne<T>>(g, stream);
        default: return run_products<Tile256<T>>(g, stream);
    }
}
template <typename T> klay_status HeadLaunch<T>::sums(const SumsArgs& g, void* stream) {
    int64_t most = 0;
    for (int i = 0; i < g.sums; ++i) most = std::max<int64_t>(most, g.sum[i].count);
    if (most > 0) KLAY_LAUNCH((head_sums_kernel<T>), dim3(grid_of(most, 256, 8192)), dim3(256), stream, g);
    return KLAY_OK;
}
template <typename T> klay_status HeadLaunch<T>::pack(PacksArgs& g, void* stream) {
    uint32_t blocks = 0;
    for (int i = 0; i < g.copies; ++i) {
        const PackArgs& c = g.copy[i];
        blocks += grid_of(c.count * (c.padded * (int64_t)sizeof(T) / 16), 256, 8192);
        g.until[i] = blocks;
    }
    if (blocks > 0 || g.clear) KLAY_LAUNCH((head_pack_kernel<T>), dim3(std::max<uint32_t>(blocks, 1)), dim3(256), stream, g);
    return KLAY_OK;
}

}  // namespace klay

// Kernels are instantiated by name: the compiler leaves out the host side of some that are only launched.
#define KLAY_HEAD_TILE(TILE)                                                                   \
    template __global__ void klay::head_forward_kernel<TILE, true>(klay::HeadArgs, klay::Tiles);  \
    template __global__ void klay::head_forward_kernel<TILE, false>(klay::HeadArgs, klay::Tiles); \
    template __global__ void klay::head_adjoint_kernel<TILE>(klay::HeadArgs, klay::Tiles);        \
    template __global__ void klay::head_product_kernel<TILE>(klay::ProductArgs, int64_t);
#define KLAY_HEAD(T)                          \
    KLAY_HEAD_TILE(klay::Tile32<klay::T>)     \
    KLAY_HEAD_TILE(klay::Tile64<klay::T>)     \
    KLAY_HEAD_TILE(klay::Tile128<klay::T>)    \
    KLAY_HEAD_TILE(klay::Tile256<klay::T>)    \
    template __global__ void klay::head_product_kernel<klay::TileOne<klay::T>>(klay::ProductArgs, int64_t); \
    template struct klay::HeadLaunch<klay::T>;
