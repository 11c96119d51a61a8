// The grids of the 8-bit floating-point product's launches over the sizes that its entry point accepts
// (csrc/f8_plan.h and the limits of csrc/bsr_internal.h): fewer than 2^32 threads along x and 2^16
// workgroups along y, and tiles that every variant has.  The corners of the accepted sizes, and random
// ones.  Prints "ok" and the most threads of a grid.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "bsr_internal.h"
#include "f8_plan.h"

namespace {

using namespace bsr;

int64_t g_most = 0;

void grid(int64_t x, int64_t threads, int64_t y, int64_t M, int64_t N) {
    if (x >= 1 && x < (int64_t(1) << 31) && x * threads < (int64_t(1) << 32) && y >= 1 && y < 65536) {
        if (x * threads > g_most) g_most = x * threads;
        return;
    }
    std::printf("%lld x %lld workgroups of %lld threads for %lld, %lld\n", (long long)x, (long long)y,
                (long long)threads, (long long)M, (long long)N);
    std::exit(1);
}

void tiled(const F8Cost &c, int tile, int64_t M, int64_t N) {
    if (tile < 0 || tile >= kF8TileCount || c.round[tile] == 0) {
        std::printf("tile %d for %lld, %lld\n", tile, (long long)M, (long long)N);
        std::exit(1);
    }
    const int parts = tile == 4 ? f8_parts(true, M, N, 1 << 20, 256) : 1;
    grid(f8_tiles(tile, M, N), kF8Tiles[tile].threads * parts, 1, M, N);
}

void product(int64_t M, int64_t N, int64_t K, int64_t cus) {
    if (M < 1 || N < 1 || M > kDenseMaxTokens || N > kDenseMaxWidth || M * N > kDenseMaxOut) return;
    if (f8_few_tokens(M, N, cus))
        return grid(tiles_across(N, 16), 1024, tiles_across(M, M <= 16 ? 16 : 32), M, N);
    for (int v = 0; v < 8; ++v) {
        const F8Cost &c = f8_cost(v & 1, v & 2, v & 4);
        const int large = f8_largest(c);
        const int64_t whole = f8_whole_rounds(c, large, M, N, K, cus);
        if (whole == 0) {
            tiled(c, f8_tile(c, M, N, K, cus), M, N);
        } else {
            if (whole % kF8Block || whole >= N) std::exit(1);
            tiled(c, large, M, whole);
            tiled(c, f8_tile(c, M, N - whole, K, cus), M, N - whole);
        }
    }
}

uint64_t g_state = 88172645463325252ull;
double unit() {
    g_state ^= g_state << 13;
    g_state ^= g_state >> 7;
    g_state ^= g_state << 17;
    return double(g_state >> 11) / 9007199254740992.0;
}

}  // namespace

int main() {
    const int64_t sizes[] = {1, 15, 16, 17, 32, 33, 63, 64, 65, 128, 255, 256, 257, 4096, 65535, 65536,
                             (1 << 20) - 1, 1 << 20, (1 << 20) + 1, (1 << 24) - 1, 1 << 24};
    for (const int64_t cus : {1, 64, 256, 304}) {
        for (const int64_t M : sizes)
            for (const int64_t N : sizes)
                for (const int64_t K : {int64_t(1), int64_t(300), kDenseMaxWidth}) product(M, N, K, cus);
        for (const int64_t M : sizes) product(M, kDenseMaxOut / M, 4096, cus);
        for (const int64_t N : sizes) product(kDenseMaxOut / N, N, 4096, cus);
    }
    for (int i = 0; i < 300000; ++i) {
        const int64_t M = int64_t(std::exp2(24 * unit())), most = kDenseMaxOut / M;
        const double bits = std::log2(double(most < kDenseMaxWidth ? most : kDenseMaxWidth));
        product(M, int64_t(std::exp2(bits * (1 - unit() * unit()))), int64_t(std::exp2(20 * unit())), 256);
    }
    std::printf("ok %lld\n", (long long)g_most);
    return 0;
}
