// Which kernel takes an 8-bit linear layer: host arithmetic only, no HIP.
#pragma once

#include <stdint.h>

namespace rs {

enum class GemmI8Tile { Split32x32, Split32x64, Private64x64, Direct64x256, Direct128x256, Direct256x256 };

// By the number of tiles and the length of K.  us per launch, bf16 output with bias, operands out of the caches in turn:
//  - Up to one 32 x 32 tile per CU: the split kernel, which has the shortest way through (32 x 32 / 32 x 64 / private / direct 128 x 256: 768 -> 2304 at one row
//    3.4 / 3.8 / 4.8 / 8.0, at 64 rows 4.0 / 4.5 / 4.9 / 7.9; 4096 -> 1024 at one row 4.6 / 6.0 / 7.5 / 20.5, at 197 8.0 / 9.2 / 8.2 / 21.8).
//  - Up to one 32 x 64 tile per CU and K <= 1024: the same with twice the features (768 -> 2304 at 197 rows 5.4 / 4.8 / 5.0 / 8.3, 768 x 768 at 394 5.2 / 4.6 / 5.0 /
//    8.2); at K = 4096 its operands, which come in pieces of lines, cost more than that (394 x 4096 -> 1024 13.0 / 10.4 / 9.7 / 21.9).
//  - Up to one 64 x 64 tile per CU, two where K >= 1024: the private kernel (private / direct 64 x 256 / direct 128 x 256: 768 x 768 at 788 rows 5.0 / 6.1 / 8.4, at
//    2200 (420 tiles) 7.0 / 6.2 / 8.4; 4096 -> 1024 at 1576 (400) 15.0 / 18.2 / 22.4, at 2200 (560) 20.9 / 18.6 / 22.6; 1024 -> 4096 at 394 (448) 6.7 / 6.8 / 9.3).
//  - At most 64 features and K >= 512, or 128 and K >= 2048: the private kernel for any number of rows, the direct one's tiles being mostly empty (private / direct
//    64 x 256 / direct 128 x 256: 768 -> 64 at 50432 rows 13.7 / 16.4 / 15.2, 4096 -> 64 at 25000 26 / 34 / 34, 2048 -> 128 at 34508 22.0 / 24.1 / 25.7; but 192 -> 64 at
//    50432 8.1 / 8.3 / 7.6, 768 -> 128 there 19.3 / 17.4 / 15.7).
//  - Beyond: the direct kernel.  Two of its 128 x 256 tiles run on a CU at a time and feed the matrix cores best (50432 x 768 -> 768, 64 / 128 rows a tile, 48 / 41; 12552 x
//    4096 -> 1024 64 / 52; 32768 x 4096 -> 4096 580 / 462), but a grid that is not many rounds of them leaves CUs idle at its end.  64 rows a tile:
//     . up to one such tile per CU (1576 x 768 -> 2304 7.6 / 9.8, 3152 x 4096 -> 1024 19.4 / 22.8);
//     . where a quarter of the CUs or fewer would get a second 128-row tile (2200 x 1024 -> 4096 17.9 / 20.2, 4400 x 2048 -> 2048 27.3 / 28.1), or less than a third of a second
//       round (4400 x 1024 -> 4096 25.9 / 28.0, 16388 x 1024 -> 1024 25.7 / 26.9; at 1.1 of K = 2048 a tie);
//     . up to two rounds at K <= 768, where a tile is mostly its ends (9000 x 768 -> 2304 22.8 / 24.9, 12608 x 384 -> 1536 15.3 / 18.5, 25216 x 768 -> 768 22.6 / 24.1), but
//       for one round nearly full (9000 x 384 -> 1536 13.6 / 11.3).
//     . 256 rows a tile, one per CU, at K >= 2048 where the last round of them is full or at least 0.7 so (128 / 256 rows a tile: 16384 x 2048 -> 2048 69.8 / 67.7,
//       16384 x 8192 -> 2048 232 / 216, 14000 x 4096 -> 1024 (0.86) 61 / 57, 12000 x 8192 -> 1024 (0.73) 98 / 93, 32768 x 4096 -> 4096 465 / 449; 1.5 rounds: 6000 x
//       4096 -> 4096 88 / 101; 16388 x 1024 -> 4096 80 / 97: a shorter K leaves the tile's ends uncovered).
inline GemmI8Tile gemm_i8_choose(int64_t M, int64_t N, int K, int64_t cus) {
    auto tiles = [&](int bm, int bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
    if (tiles(32, 32) <= cus) return GemmI8Tile::Split32x32;
    if (K <= 1024 && tiles(32, 64) <= cus) return GemmI8Tile::Split32x64;
    const int64_t t64 = tiles(64, 64);
    if (t64 <= cus || (K >= 1024 && t64 <= 2 * cus)) return GemmI8Tile::Private64x64;
    if ((N <= 64 && K >= 512) || (N <= 128 && K >= 2048)) return GemmI8Tile::Private64x64;
    const int64_t last = tiles(256, 256) % cus;
    if (K >= 2048 && (last == 0 || 10 * last >= 7 * cus)) return GemmI8Tile::Direct256x256;
    const int64_t t = tiles(128, 256);
    if (tiles(64, 256) <= cus || (t > cus && 4 * t <= 5 * cus) || (t > 2 * cus && 10 * t <= 23 * cus)) return GemmI8Tile::Direct64x256;
    if (K <= 768 && t <= 4 * cus && !(2 * t > 3 * cus && t <= 2 * cus)) return GemmI8Tile::Direct64x256;
    return GemmI8Tile::Direct128x256;
}

}  // namespace rs
