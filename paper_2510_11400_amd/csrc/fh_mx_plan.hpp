// Which kernel takes a product of stored matrices, apart from the kernels so that it can be looked at on any machine: plain C++, no HIP.
#pragma once

#include <stdint.h>

namespace fh {

enum class Tile : int32_t { waves32, waves32_wide, waves64, square128, square256 };
struct Plan { Tile tile; int32_t parts; int64_t chunks_each; };

// A sum is split over workgroups where its outputs leave compute units idle, in parts of sixteen chunks at least.  Otherwise the kernel
// with the shortest time, in hundredths of a microsecond with c chunks, by lines through what they measured (bf16 out; us,
// in the order 32 (four waves), 64, 128, 256):
//     1024 x 768 x 768    3.8  4.7  4.9  8.8     700 x 700 x 8192    9.3 11.7 23.9 51.3     4096 x 4096 x 4096  99   66 39.2 36.7
//     4096 x 768 x 768    9.6  9.6  5.7  9.4     512 x 4096 x 4096  16.1 11.7 14.0 27.2     2304 x 768 x 8192  25.6 20.2 24.0 49.1
//     8192 x 2304 x 768  44.3 36.3 15.5 20.5     2048^3             17.6 13.9  9.6 16.9     3000^3             47.1 44.7 25.2 26.7
//     4096 x 4096 x 1024 40.9 35.3 15.9 15.7     8192 x 8192 x 1024  176  143   68   54     8192 x 8192 x 4096  422  278  172  139
// Workgroups of a kernel run in rounds of 256 (32: up to four a compute unit share it; 128: two, which one round of 512 makes).
// Up to one tile of 32 a compute unit, eight waves share its sum where each has a chunk (300 x 300 x 8192 7.1 -> 5.8).
inline Plan plan_of(int64_t m, int64_t n, int64_t chunks)
{
    const auto tiles = [&](int64_t side) { return ((m + side - 1) / side) * ((n + side - 1) / side); };
    const auto rounds = [&](int64_t side) { return (tiles(side) + 255) / 256; };
    const int64_t small = tiles(32);
    if (small <= 128 && chunks >= 32) {
        int64_t parts = 256 / small;
        if (parts > chunks / 16) parts = chunks / 16;
        const int64_t each = (chunks + parts - 1) / parts;
        return Plan{Tile::waves32_wide, (int32_t)((chunks + each - 1) / each), each};
    }
    if (small <= 256 && chunks >= 8) return Plan{Tile::waves32_wide, 1, chunks};
    const int64_t times[4] = {230 + rounds(32) * (30 + 9 * chunks), 340 + rounds(64) * (90 + 22 * chunks),
                              tiles(128) <= 256 ? 310 + tiles(128) / 3 + 66 * chunks : 250 + (360 + 102 * chunks) * tiles(128) / 512,
                              500 + rounds(256) * (480 + (tiles(256) <= 128 ? 125 : 179) * chunks)};
    const Tile kernels[4] = {Tile::waves32, Tile::waves64, Tile::square128, Tile::square256};
    int best = 0;
    for (int i = 1; i < 4 && chunks > 0; ++i)
        if (times[i] < times[best]) best = i;
    return Plan{kernels[best], 1, chunks};
}

// Whether the tiles of 64 go to the XCDs in runs.  In their order an XCD works on every eighth tile: all rows of a, and of b an eighth or all.
// Where that is more than its L2 holds it is given a run instead (2304 x 768 x 8192 19.8 -> 17.5 us; 512 x 4096 x 4096, which fits, 11.1 -> 11.4).
inline bool tiles_in_runs(int64_t m, int64_t n, int64_t chunks)
{
    const int64_t rows = m + ((n + 63) / 64 % 8 == 0 ? n / 8 : n);
    return rows * chunks * 128 > (int64_t)4 << 20;
}

}  // namespace fh
