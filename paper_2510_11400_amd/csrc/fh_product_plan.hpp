// Which kernel takes a product of rows in chunks of 128 bytes, apart from the kernels so that it can be looked at on any machine: plain C++, no HIP.
#pragma once

#include <stdint.h>

namespace fh {

// Sums of 32 x 32 by four or eight waves that share them, of 64 x 64 by four, tiles of 128 x 128 and 256 x 256.
enum class ProductTile : int32_t { waves32, waves32_wide, waves64, square128, square256 };
// A kernel, and how many workgroups share a tile's sum.
struct ProductPlan { ProductTile tile; uint32_t parts, chunks_each; };

constexpr int64_t product_side(ProductTile t)
{
    return t == ProductTile::square256 ? 256 : t == ProductTile::square128 ? 128 : t == ProductTile::waves64 ? 64 : 32;
}
// The rows that a partial sum of columns stands for: a workgroup's, of the tiles through LDS a wave's.
constexpr int64_t product_sum_rows(ProductTile t) { return product_side(t) / (t == ProductTile::square128 || t == ProductTile::square256 ? 2 : 1); }

// The expected time in hundredths of a microsecond, from `tiles` of c chunks each: lines through what the kernels measured.  The choice by them is within
// 1 % of the best on average over 55 products of 8-bit integers and bf16, plain and gated, and 4 % of 10 in fp32; the worst one met took a fifth longer than
// the best (fp32, pairs of 1748 x 1557 x 690, 103 us and 85: 350 tiles of 128 on 256 units take two rounds where the line counts 1.4).  A time itself may be
// off by more, most for pairs of few chunks, whose activations no line knows (8 bits, 509 x 2731 x 1023: 9.8 us expected, 14 taken).  Some (us, in the order above):
//     8-bit  64 x 8192 x 4096    9.3  10.0  10.4  25.2  46.6     1024 x 2048 x 2048   15.0  18.8  11.5  13.8  27.5     4096 x 4096 x 1024  65.0  94.4  51.9  27.1  23.7
//           512 x 768 x 768      4.1   4.2   5.2   8.3  16.3     2048 x 2048 x 768    15.6  21.6  12.1   9.7  17.1     8192 x 1024 x 8192 283.0 283.9 150.2  71.4  84.1
//     bf16, pairs of 1024 x 2048 x 768  21.4 28.9 15.0 13.2 25.9    4096 x 2048 x 768   111.1 129.4  66.2  34.8  32.3     256 x 4096 x 4096   49.5  47.5  27.8  47.6  83.6
//     fp32, pairs of  512 x 2048 x 768  36.1 38.7 32.3 53.8 184.8   2048 x 2048 x 1024  177.7 179.5 143.6 128.1 243.2     333 x 1001 x 515    20.7  22.3  23.3  48.1 143.3
// `slow`: fp32, whose matrix instructions take eight times as long a chunk.
inline int64_t product_time(ProductTile t, int64_t tiles, int64_t c, bool slow)
{
    const auto rounds = [&](int64_t each) { return tiles <= 256 ? each : each * tiles / 256; };
    switch (t) {
        case ProductTile::waves32: return slow ? 315 + rounds(41 + 16 * c) : 205 + rounds(23 + 10 * c);
        case ProductTile::waves32_wide: return slow ? 300 + rounds(119 + 14 * c) : 187 + rounds(72 + 9 * c);
        case ProductTile::waves64: return slow ? 606 + rounds(170 + 47 * c) : 233 + rounds(155 + 19 * c);
        case ProductTile::square128: return slow ? 912 + rounds(183 * c) + 6 * c : 322 + rounds(237 + 46 * c) + 7 * c;
        case ProductTile::square256: break;
    }
    return (tiles + 255) / 256 * (slow ? 1326 + 718 * c : 1095 + 116 * c);
}

// m x n sums (a pair's both) over `chunks` chunks, by a kernel up to `last`.
inline ProductPlan product_plan(int64_t m, int64_t n, int64_t chunks, bool slow, bool shared, ProductTile last = ProductTile::square256)
{
    ProductPlan best = {ProductTile::waves32, 1, (uint32_t)chunks};
    int64_t least = 0;
    if (chunks == 0) return best;
    for (int32_t i = 0; i <= (int32_t)last; ++i) {
        const ProductTile t = (ProductTile)i;
        const int64_t side = product_side(t), tiles = ((m + side - 1) / side) * ((n + side - 1) / side);
        // A shared sum's parts, eight chunks of it at least, are written and read once more by a kernel of their own.
        for (int64_t parts = 1; parts == 1 || (shared && parts <= 16 && chunks / parts >= 8 && tiles * (parts - 1) < 512); ++parts) {
            const int64_t each = (chunks + parts - 1) / parts, time = product_time(t, tiles * parts, each, slow) + (parts > 1 ? 300 + parts * m * n / 6250 : 0);
            if (least && time >= least) continue;
            least = time;
            best = ProductPlan{t, (uint32_t)((chunks + each - 1) / each), (uint32_t)each};
        }
    }
    return best;
}
inline ProductTile product_tile(int64_t m, int64_t n, int64_t chunks, bool slow, ProductTile last = ProductTile::square256)
{
    return product_plan(m, n, chunks, slow, false, last).tile;
}

// Whether the kernel that is made for few rows takes a product.  In 8 bits 1, 4 and 8 rows of 4096 x 8192 took it 6.2, 6.9 and 7.6 us, the kernels above 6.8, 7.1
// and 7.0; of 4096 x 4096 4.1, 4.5, 4.8 and 5.1, 5.0, 5.2; pairs of 8192 x 4096 14.8, 15.2, 11.5 and 16.1, 16.1, 12.5; fp32 4 and 16 rows, pairs of 2048 x 1024 and
// 2048 x 768 6.4 and 6.2, the others 7.8 and 6.6.  Dense bf16 is no better off (8192 x 4096, 4 rows 26.4 and 23.2), but where its
// operands would have to be laid out first.
constexpr int64_t kMostFewRows = 16;
inline bool few_rows_of_bytes(int64_t m, bool pair) { return m <= (pair ? 8 : 4); }
inline bool few_rows_dense(int64_t m, bool slow, bool laid_out) { return m <= kMostFewRows && (slow || laid_out); }


// Whether a backward pass keeps what the rounding of [dg | du] to bf16 leaves, as two bf16 values for one (by the kernels up to waves64 alone).  The sums of dx and dW
// average a rounding's errors where many gradients are summed; where few are, or a few outweigh the others, the results' errors are up to three times those of their own
// rounding (over 1.5 times in 13 of 100 random layers of 2^14 to 2^18 gradients, 7 and 2 in the next doublings, against 1.4 for large ones).  Within these limits it costs
// (us; tokens x features x hidden, without and with): 26 x 63 x 49 16.5 and 16.3, 200 x 400 x 300 15.3 and 17.1, 333 x 515 x 700 27 and 30, 4096 x 512 x 64 26.5 and 29,
// 1024 x 256 x 512 23 and 28.5, 512 x 256 x 1024 24.5 and 32, 16 x 4000 x 2048 38.5 and 55.7; beyond them 4096 x 1024 x 64 would take 30.6 and 33.8, 1024 x 512 x 512
// 24 and 33.5, 8 x 4000 x 8192 104 and 174.
constexpr int64_t kMostWithRests = (int64_t)1 << 19, kMostTermsWithRests = (int64_t)1 << 27;
inline bool product_with_rests(int64_t tokens, int64_t features, int64_t hidden, bool slow)
{
    return !slow && tokens * hidden <= kMostWithRests && tokens * hidden * features <= kMostTermsWithRests;
}
inline ProductTile product_last(bool rests) { return rests ? ProductTile::waves64 : ProductTile::square256; }

}  // namespace fh
