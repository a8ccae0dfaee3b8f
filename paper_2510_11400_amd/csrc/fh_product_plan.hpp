// Which kernel takes a product of rows in chunks of 128 bytes, apart from the kernels so that it can be looked at on any machine: plain C++, no HIP.
#pragma once

#include <stdint.h>

namespace fh {

// A kernel, and how many workgroups share a tile's sum.
enum class ProductTile : int32_t { waves32, waves32_wide, waves64, square128, square256 };

// The rows that a workgroup's sums of columns stand for.
inline int64_t product_sum_rows(ProductTile t) { return t == ProductTile::waves32 || t == ProductTile::waves32_wide ? 32 : t == ProductTile::square256 ? 128 : 64; }

// m x n sums (a pair's both) over `chunks` chunks; `slow`: fp32, whose matrix instructions take eight times as long a chunk.
struct ProductPlan { ProductTile tile; uint32_t parts, chunks_each; };
inline ProductTile product_tile(int64_t m, int64_t n, int64_t chunks, bool slow)
{
    const auto tiles = [&](int64_t side) { return ((m + side - 1) / side) * ((n + side - 1) / side); };
    const auto rounds = [&](int64_t side) { return (tiles(side) + 255) / 256; };
    (void)slow;
    if (tiles(32) <= 256 && chunks >= 8) return ProductTile::waves32_wide;
    const int64_t times[4] = {230 + rounds(32) * (30 + 9 * chunks), 340 + rounds(64) * (90 + 22 * chunks),
                              tiles(128) <= 256 ? 310 + tiles(128) / 3 + 66 * chunks : 250 + (360 + 102 * chunks) * tiles(128) / 512,
                              500 + rounds(256) * (480 + (tiles(256) <= 128 ? 125 : 179) * chunks)};
    const ProductTile kernels[4] = {ProductTile::waves32, ProductTile::waves64, ProductTile::square128, ProductTile::square256};
    int best = 0;
    for (int i = 1; i < 4 && chunks > 0; ++i)
        if (times[i] < times[best]) best = i;
    return kernels[best];
}

// The same for a product whose sums may be shared: parts of `chunks` where the tiles leave compute units idle.
inline ProductPlan product_plan(int64_t m, int64_t n, int64_t chunks, bool slow, bool shared)
{
    const ProductTile tile = product_tile(m, n, chunks, slow);
    const ProductPlan whole = {tile, 1, (uint32_t)chunks};
    if (!shared) return whole;
    const int64_t side = tile == ProductTile::square256 ? 256 : tile == ProductTile::square128 ? 128 : tile == ProductTile::waves64 ? 64 : 32;
    const int64_t tiles = ((m + side - 1) / side) * ((n + side - 1) / side), held = tile == ProductTile::square256 ? 256 : 512;
    int64_t parts = held / tiles;
    if (parts > chunks / 16) parts = chunks / 16;
    if (parts < 2) return whole;
    const int64_t each = (chunks + parts - 1) / parts;
    return ProductPlan{tile, (uint32_t)((chunks + each - 1) / each), (uint32_t)each};
}

}  // namespace fh
