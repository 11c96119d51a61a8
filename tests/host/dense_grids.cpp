// The grids of the dense products' launches over the sizes that their entry points accept
// (csrc/dense_plan.h and the limits of csrc/bsr_internal.h): fewer than 2^32 threads along x and 2^16
// workgroups along y, and tile counts that fit the kernels' 32-bit arithmetic.  The corners of the
// accepted sizes, and random ones.  Prints "ok" and the most threads of a grid.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "bsr_internal.h"
#include "dense_plan.h"

namespace {

using namespace bsr;

int64_t g_most = 0;

void grid(const char *what, int64_t x, int64_t threads, int64_t y, int64_t a, int64_t b) {
    if (x >= 1 && x < (int64_t(1) << 31) && x * threads < (int64_t(1) << 32) && y >= 1 && y < 65536) {
        if (x * threads > g_most) g_most = x * threads;
        return;
    }
    std::printf("%s: %lld x %lld workgroups of %lld threads for %lld, %lld\n", what, (long long)x,
                (long long)y, (long long)threads, (long long)a, (long long)b);
    std::exit(1);
}

// A product of M tokens with `rows` rows of weights, in every way that it can be launched.
void product(int64_t M, int64_t rows, int64_t cus) {
    const auto one = [&](const char *what, const DenseTile &t, int64_t m, int64_t n) {
        grid(what, dense_tiles(t, m, n), t.threads, 1, m, n);
    };
    int64_t rest = rows;
    if (const int64_t first = rows_in_whole_rounds(M, rows, cus)) {
        if (first <= 0 || first >= rows || first % kRingTiles[0].bn != 0) {
            std::printf("%lld of %lld rows in whole rounds\n", (long long)first, (long long)rows);
            std::exit(1);
        }
        one("ring, whole rounds", kRingTiles[0], M, first);
        rest = rows - first;
    }
    one("ring", kRingTiles[cheapest_tile(kRingTiles, M, rest, cus)], M, rest);
    one("register", kRegisterTiles[cheapest_tile(kRegisterTiles, M, rows, cus)], M, rows);
    one("split", kSplitTiles[cheapest_tile(kSplitTiles, M, rows, cus)], M, rows);
}

// The few-token kernel: 16 channels and up to 32 tokens to a workgroup of 512.
void rows_kernel(int64_t M, int64_t N, int64_t cus) {
    const int64_t gm = tiles_across(M, 32), gn = tiles_across(N, 16);
    if (M <= 16) grid("few tokens", gn, 512, 1, M, N);
    if (M <= 32 || gm * gn <= cus) grid("few tokens", gn, 512, gm, M, N);
}

void backward(int64_t T, int64_t K, int64_t F, int64_t cus) {
    for (int32_t dt : {int32_t(BSR_F32), int32_t(BSR_BF16)}) {
        const GatedWorkspace l = gated_workspace_layout(T, K, F, dt);
        const bool bf16 = dt == BSR_BF16;
        grid("slopes", tiles_across(bf16 ? T : l.Tp, 64), 256, tiles_across(l.Fp, 64), T, F);
        grid("bias", tiles_across(2 * F, 16), 256, 1, T, F);
        const int64_t tiles = 2 * tiles_across(l.Fp, 64) * tiles_across(K, 64) +
                              tiles_across(bf16 ? 1 : l.Tp, 64) * tiles_across(K, 64);
        if (tiles >= int64_t(1) << 31) grid("transposes' tiles", tiles, 1, 1, T, F);
        grid("transposes", tiles < kTransposeGroups ? tiles : kTransposeGroups, 256, 1, T, F);
        const int64_t dw = bf16 ? 2 * l.Fp : 2 * F;
        const DenseTile &small = kRingTiles[4];
        if (l.x_slices > 1) grid("dX in slices", dense_tiles(small, T, K), 512, l.x_slices, T, K);
        if (l.w_slices > 1) grid("dW in slices", dense_tiles(small, dw, K), 512, l.w_slices, dw, K);
        product(T, K, cus);
        product(dw, K, cus);
    }
}

uint64_t g_state = 0x9E3779B97F4A7C15ull;
double uniform() {   // xorshift64*
    g_state ^= g_state >> 12;
    g_state ^= g_state << 25;
    g_state ^= g_state >> 27;
    return double((g_state * 0x2545F4914F6CDD1Dull) >> 11) / 9007199254740992.0;
}
int64_t some(int64_t most) {   // a size, uniform in its logarithm, often at a corner
    if (uniform() < 0.2) return most;
    int64_t n = int64_t(std::exp(uniform() * std::log(double(most) + 0.99)));
    if (uniform() < 0.5) n = (n + 63) / 64 * 64 + int64_t(uniform() * 3) - 1;
    return n < 1 ? 1 : n > most ? most : n;
}

}  // namespace

int main() {
    const int64_t wide = kDenseMaxWidth, tall = kDenseMaxTokens;
    for (int n = 0; n < 400000; ++n) {
        const int64_t cus = n % 4 ? 256 : some(304);
        int64_t T = some(tall);
        int64_t N = some(wide);
        if (T > kDenseMaxOut / N) T = kDenseMaxOut / N;         // an 8-bit product
        product(T, N, cus);
        rows_kernel(T, N, cus);
        T = some(tall);
        N = some(wide);
        if (T > kDenseMaxOut / 2 / N) T = kDenseMaxOut / 2 / N; // the gated block
        product(T, 2 * N, cus);
        rows_kernel(T, N, cus);
        T = some(kGatedMaxBackwardTokens);
        int64_t F = some(kGatedMaxBackwardWidth), K = some(wide);
        if (K > kDenseMaxOut / 2 / F) K = kDenseMaxOut / 2 / F;
        if (T > kDenseMaxOut / 2 / F) T = kDenseMaxOut / 2 / F;
        if (T > kDenseMaxOut / K) T = kDenseMaxOut / K;
        backward(T, K, F, cus);
    }
    std::printf("ok %lld\n", (long long)g_most);
    return 0;
}
