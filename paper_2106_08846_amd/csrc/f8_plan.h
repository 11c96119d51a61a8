// Which tile an 8-bit floating-point product takes (host only).
#pragma once

#include <cstddef>
#include <cstdint>

#include "dense_plan.h"

namespace bsr {

// Tiles by number, and the threads of their workgroups.
struct F8Tile {
    int bm, bn, threads;
};
constexpr F8Tile kF8Tiles[] = {{256, 256, 512}, {192, 256, 512}, {128, 256, 512}, {128, 128, 512}, {64, 64, 256}};
constexpr int kF8TileCount = int(sizeof kF8Tiles / sizeof kF8Tiles[0]);

// What a round of workgroups over the chip takes in each tile, in tenths of a microsecond (MI355X, grids of
// 1 to 64 rounds): at K = 4096 (`round`), of that independent of K (`fixed`: the first loads and the epilogue,
// which a tile that fills its CU does not hide), and at K = 4096 where a workgroup has its CU to itself
// (`alone`: the smaller tiles leave room for two to four on a CU).  0: not used, because its registers do not
// hold it or two rounds of half its size take less.  In this order: rows on 16-byte boundaries or not; bf16
// or fp32 output; a scale for 128 rows of B or for each.  So bf16 4096 x 4096 x 4096 with a weight's scales
// takes 61 us in 256 x 256 tiles, 75 in 128 x 128 and 112 in 64 x 64; 2048 x 2048 x 4096 49, 27 and 31; and
// 8192 x 8192 x 256 56, 47 and 65.
struct F8Cost {
    int round[kF8TileCount], fixed[kF8TileCount], alone[kF8TileCount];
};
constexpr F8Cost kF8Costs[2][2][2] = {
    {{{{990, 783, 0, 340, 141}, {218, 157, 0, 45, 19}, {990, 783, 0, 510, 265}},
      {{0, 835, 0, 343, 141}, {0, 156, 0, 46, 19}, {0, 835, 0, 518, 267}}},
     {{{0, 1155, 885, 545, 168}, {0, 166, 140, 85, 27}, {0, 1155, 885, 592, 309}},
      {{0, 0, 923, 588, 172}, {0, 0, 142, 84, 26}, {0, 0, 923, 633, 318}}}},
    {{{{605, 430, 355, 183, 66}, {110, 68, 51, 19, 7}, {605, 430, 355, 268, 118}},
      {{692, 500, 400, 200, 69}, {111, 67, 51, 18, 6}, {692, 500, 400, 270, 118}}},
     {{{1070, 770, 612, 320, 100}, {166, 84, 69, 21, 7}, {1070, 770, 612, 433, 171}},
      {{1210, 843, 658, 404, 106}, {170, 85, 69, 39, 6}, {1210, 843, 658, 459, 177}}}}};

inline const F8Cost &f8_cost(bool aligned, bool wide, bool w_rows) {
    return kF8Costs[aligned ? 1 : 0][wide ? 1 : 0][w_rows ? 1 : 0];
}
inline int64_t f8_tiles(int tile, int64_t M, int64_t N) {
    return tiles_across(M, kF8Tiles[tile].bm) * tiles_across(N, kF8Tiles[tile].bn);
}
// In units of 1 / 4096 of the table's.
inline int64_t f8_tile_cost(const F8Cost &c, int tile, int64_t M, int64_t N, int64_t K, int64_t cus) {
    const int64_t fixed = int64_t(c.fixed[tile]) * 4096;
    const int64_t rounds =
        tiles_across(f8_tiles(tile, M, N), cus) * (fixed + (c.round[tile] - c.fixed[tile]) * K);
    const int64_t alone = fixed + (c.alone[tile] - c.fixed[tile]) * K;
    return rounds > alone ? rounds : alone;
}
// The tile of least cost whose grid has under 2^32 threads, the larger of equals.
inline int f8_tile(const F8Cost &c, int64_t M, int64_t N, int64_t K, int64_t cus) {
    int best = -1;
    int64_t least = 0;
    for (int i = 0; i < kF8TileCount; ++i) {
        if (c.round[i] == 0 || f8_tiles(i, M, N) * kF8Tiles[i].threads >= int64_t(1) << 32) continue;
        const int64_t cost = f8_tile_cost(c, i, M, N, K, cus);
        if (best < 0 || cost < least) best = i, least = cost;
    }
    return best;
}
// A product whose last round of its largest tile is not full goes in two launches where that saves a
// twentieth, the second launch's 2 us counted: as many channels as fill whole rounds, then the rest in the
// tile that suits it.  The channels of the first launch, whole tiles; 0: one launch.
inline int64_t f8_whole_rounds(const F8Cost &c, int large, int64_t M, int64_t N, int64_t K, int64_t cus) {
    const int64_t tiles_m = tiles_across(M, kF8Tiles[large].bm), tiles_n = tiles_across(N, kF8Tiles[large].bn);
    const int64_t columns = tiles_m * tiles_n / cus * cus / tiles_m;
    if (columns == 0 || columns == tiles_n) return 0;
    const int64_t first = columns * kF8Tiles[large].bn, rest = N - first;
    const int64_t whole = f8_tile_cost(c, f8_tile(c, M, N, K, cus), M, N, K, cus);
    const int64_t parts = f8_tile_cost(c, large, M, first, K, cus) +
                          f8_tile_cost(c, f8_tile(c, M, rest, K, cus), M, rest, K, cus) + 20 * 4096;
    return parts * 20 <= whole * 19 ? first : 0;
}
inline int f8_largest(const F8Cost &c) {
    int i = 0;
    while (c.round[i] == 0) ++i;
    return i;
}

// Parts of the waves of a 64 x 64 workgroup that share out the blocks of a long contraction where every
// workgroup has a CU to itself.  Rows on 16-byte boundaries: 128 x 4096 x 4096 takes 13.3 us with one part,
// 10.6 with two and 10.9 with four (fp32 output 20.9, 16.1 and 15.9), 1024 x 1024 x 16384 60, 42 and 35.
// Others go through registers, too many for four parts where B has a scale for each row (1000 x 1000 x 8191
// with fp32 output 57, 48 and 70 us); 333 x 1024 x 1531 takes 15.8 and 14.8 us, 333 x 2304 x 770 8.9 and 9.0.
inline int f8_parts(bool aligned, int64_t M, int64_t N, int64_t K, int64_t cus) {
    if (tiles_across(M, 64) * tiles_across(N, 64) > cus) return 1;
    if (!aligned) return K >= 1024 ? 2 : 1;
    return K >= 8192 ? 4 : K >= 2048 ? 2 : 1;
}

// Whether a product goes to the kernel for few tokens: up to 32, or as many groups of 32 tokens x 16
// channels, each with a whole contraction to itself, as fit the chip in one round.
inline bool f8_few_tokens(int64_t M, int64_t N, int64_t cus) {
    return M <= 32 || tiles_across(M, 32) * tiles_across(N, 16) <= cus;
}

}  // namespace bsr
