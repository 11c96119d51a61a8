// Which tile a dense product takes, and the grids that follow from it (host only).
#pragma once

#include <cstddef>
#include <cstdint>

namespace bsr {

// A tile of bm tokens x bn rows of the weights (the gated block's two matrices together), the threads of
// its workgroup, and what a round of workgroups over the chip costs in it.
struct DenseTile {
    int bm, bn, threads, cost;
};

// The costs are those of a round of each tile, measured (MI355X, K = 4096) over grids of 1 to 32 rounds, in
// hundredths of a round of 256 x 256.
//
// bf16 and int8 rows on 16-byte boundaries, where a round of 256 x 256 takes 110 us in bf16 and 61 in
// int8.  So bf16 4096 x 4096 x 4096 takes 110 us in 256 x 256 tiles, 160 in 128 x 128 and 259 in 64 x 64;
// 2048^3 51, 24 and 33; 128 x 8192 x 4096 84, 35 and 20; and 6144 x 2048 x 16384, whose 192 tiles of
// 256 x 256 leave a quarter of the CUs idle, 438 against 368 in 192 x 256; int8 2048 x 20480 x 4096 184
// in 256 x 256 (2.5 rounds) and 196 in 192 x 256 (3.4).
constexpr DenseTile kRingTiles[] = {
    {256, 256, 512, 100}, {192, 256, 512, 78}, {128, 256, 512, 62}, {128, 128, 512, 38}, {64, 64, 256, 16}};
// On other boundaries: bf16 4096 x 4096 x 4095 takes 146 us in 256 x 256 tiles, 183 in 128 x 256, 194 in
// 128 x 128 and 368 in 64 x 64; 2048 x 2048 x 4095 136, 89, 68 and 100; int8 333 x 2304 x 770 28, 18, 12
// and 9.
constexpr DenseTile kRegisterTiles[] = {
    {256, 256, 512, 100}, {128, 256, 512, 63}, {128, 128, 512, 38}, {64, 64, 256, 17}};
// fp32: 1000 x 768 x 3064 takes 102 us in 128 x 128 tiles and 49 in 64 x 64, 896 x 4096 x 768 36 and 45.
constexpr DenseTile kSplitTiles[] = {{128, 128, 512, 168}, {64, 64, 512, 55}};

inline int64_t tiles_across(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }

// Workgroups that M tokens and `rows` rows of weights take in this tile, and the cost of their rounds.
inline int64_t dense_tiles(const DenseTile &t, int64_t M, int64_t rows) {
    return tiles_across(M, t.bm) * tiles_across(rows, t.bn);
}
inline int64_t dense_cost(const DenseTile &t, int64_t M, int64_t rows, int64_t cus) {
    return tiles_across(dense_tiles(t, M, rows), cus) * t.cost;
}

// The tile of least cost, the larger of equals.
template <size_t N>
int cheapest_tile(const DenseTile (&tiles)[N], int64_t M, int64_t rows, int64_t cus) {
    int best = 0;
    int64_t least = dense_cost(tiles[0], M, rows, cus);
    for (int i = 1; i < int(N); ++i) {
        const int64_t cost = dense_cost(tiles[i], M, rows, cus);
        if (cost < least) best = i, least = cost;
    }
    return best;
}

// A product whose last round of 256 x 256 tiles is not full goes in two launches where that saves a
// twentieth: as many rows of the weights as fill whole rounds, then the rest in the tile that suits it
// (int8 2048 tokens through 2 x 10240 x 4096: 640 tiles in 2.5 rounds).  The rows of the first launch; 0:
// one launch.
inline int64_t rows_in_whole_rounds(int64_t M, int64_t rows, int64_t cus) {
    const DenseTile &large = kRingTiles[0];
    const int64_t tiles_m = tiles_across(M, large.bm), tiles_n = tiles_across(rows, large.bn);
    const int64_t columns = tiles_m * tiles_n / cus * cus / tiles_m;    // of tiles, in full rounds
    if (columns == 0 || columns == tiles_n) return 0;
    const int64_t first = columns * large.bn, rest = rows - first;
    const int64_t whole = dense_cost(kRingTiles[cheapest_tile(kRingTiles, M, rows, cus)], M, rows, cus);
    const int64_t parts = dense_cost(large, M, first, cus) +
                          dense_cost(kRingTiles[cheapest_tile(kRingTiles, M, rest, cus)], M, rest, cus);
    return parts * 20 <= whole * 19 ? first : 0;
}

// Workgroups of the gradients' transposes: beyond this many, each takes several tiles.
constexpr int64_t kTransposeGroups = int64_t(1) << 16;

}  // namespace bsr
