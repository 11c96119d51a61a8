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

// What a round of workgroups over the chip takes in each tile, in tenths of a microsecond at K = 4096
// (MI355X, grids of 1 to 32 rounds), and what one workgroup takes that has its CU to itself: the smaller
// tiles leave room for two to four on a CU.  0: not used, its registers do not hold it.  In this order:
// rows on 16-byte boundaries or not; bf16 or fp32 output; a scale for 128 rows of B or for each.
// So bf16 4096 x 4096 x 4096 with a weight's scales takes 64 us in 256 x 256 tiles, 76 in 128 x 128 and 107
// in 64 x 64; 2048 x 2048 x 4096 58, 28 and 31.
struct F8Cost {
    int round[kF8TileCount], alone[kF8TileCount];
};
constexpr F8Cost kF8Costs[2][2][2] = {
    {{{{979, 790, 700, 320, 140}, {979, 790, 700, 521, 270}}, {{0, 825, 700, 330, 143}, {0, 825, 700, 528, 270}}},
     {{{0, 1140, 880, 525, 163}, {0, 1140, 880, 582, 330}}, {{0, 0, 910, 545, 168}, {0, 0, 910, 603, 330}}}},
    {{{{640, 460, 372, 190, 67}, {640, 460, 372, 278, 140}}, {{726, 530, 415, 212, 71}, {726, 530, 415, 287, 145}}},
     {{{1100, 797, 620, 330, 103}, {1100, 797, 620, 431, 210}}, {{0, 874, 665, 403, 110}, {0, 874, 665, 453, 215}}}}};

inline const F8Cost &f8_cost(bool aligned, bool wide, bool w_rows) {
    return kF8Costs[aligned ? 1 : 0][wide ? 1 : 0][w_rows ? 1 : 0];
}
inline int64_t f8_tiles(int tile, int64_t M, int64_t N) {
    return tiles_across(M, kF8Tiles[tile].bm) * tiles_across(N, kF8Tiles[tile].bn);
}
inline int64_t f8_tile_cost(const F8Cost &c, int tile, int64_t M, int64_t N, int64_t cus) {
    const int64_t rounds = tiles_across(f8_tiles(tile, M, N), cus) * c.round[tile];
    return rounds > c.alone[tile] ? rounds : c.alone[tile];
}
// The tile of least cost, the larger of equals.
inline int f8_tile(const F8Cost &c, int64_t M, int64_t N, int64_t cus) {
    int best = -1;
    int64_t least = 0;
    for (int i = 0; i < kF8TileCount; ++i) {
        if (c.round[i] == 0) continue;
        const int64_t cost = f8_tile_cost(c, i, M, N, cus);
        if (best < 0 || cost < least) best = i, least = cost;
    }
    return best;
}
// A product whose last round of its largest tile is not full goes in two launches where that saves a
// twentieth: as many channels as fill whole rounds, then the rest in the tile that suits it.  The channels
// of the first launch, whole tiles; 0: one launch.
inline int64_t f8_whole_rounds(const F8Cost &c, int large, int64_t M, int64_t N, int64_t cus) {
    const int64_t tiles_m = tiles_across(M, kF8Tiles[large].bm), tiles_n = tiles_across(N, kF8Tiles[large].bn);
    const int64_t columns = tiles_m * tiles_n / cus * cus / tiles_m;
    if (columns == 0 || columns == tiles_n) return 0;
    const int64_t first = columns * kF8Tiles[large].bn, rest = N - first;
    const int64_t whole = f8_tile_cost(c, f8_tile(c, M, N, cus), M, N, cus);
    const int64_t parts = f8_tile_cost(c, large, M, first, cus) +
                          f8_tile_cost(c, f8_tile(c, M, rest, cus), M, rest, cus);
    return parts * 20 <= whole * 19 ? first : 0;
}
inline int f8_largest(const F8Cost &c) {
    int i = 0;
    while (c.round[i] == 0) ++i;
    return i;
}

// Whether a product goes to the kernel for few tokens: up to 32, or as many groups of 32 tokens x 16
// channels, each with a whole contraction to itself, as fit the chip in one round.
inline bool f8_few_tokens(int64_t M, int64_t N, int64_t cus) {
    return M <= 32 || tiles_across(M, 32) * tiles_across(N, 16) <= cus;
}

}  // namespace bsr
