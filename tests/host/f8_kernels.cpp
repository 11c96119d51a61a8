// Which kernels of the 8-bit floating-point product a list of calls launches, by the rules of
// csrc/f8_plan.h on a chip of 256 CUs, and which kernels there are.  The list, CALLS, comes from the
// command line (-include): {T, N, K, rows aligned, fp32 output, a scale for each row of B}.  Prints "ok",
// then a line for each kernel: how many of the calls launch it, and its name.
#include <cstdio>
#include <map>
#include <string>

#include "bsr_internal.h"
#include "f8_plan.h"

namespace {

using namespace bsr;

struct Call {
    int64_t M, N, K;
    bool aligned, wide, w_rows;
};
constexpr Call kCalls[] = {CALLS};
constexpr int64_t kCus = 256;

std::map<std::string, int> g_launches;

std::string form(bool aligned, bool w_rows) {
    return std::string(aligned ? " aligned" : " unaligned") + (w_rows ? " rows" : " blocks");
}
std::string few(int waves, int tokens, bool aligned, bool w_rows) {
    return "few " + std::to_string(waves) + " " + std::to_string(tokens) + form(aligned, w_rows);
}
std::string tiled(int tile, int parts, bool aligned, bool wide, bool w_rows) {
    return "tile " + std::to_string(kF8Tiles[tile].bm) + "x" + std::to_string(kF8Tiles[tile].bn) + " " +
           std::to_string(parts) + form(aligned, w_rows) + (wide ? " f32" : " bf16");
}

void launch(const Call &c, int tile, int64_t N) {
    const int parts = tile == kF8TileCount - 1 ? f8_parts(c.aligned, c.M, N, c.K, kCus) : 1;
    ++g_launches.at(tiled(tile, parts, c.aligned, c.wide, c.w_rows));
}

void product(const Call &c) {
    if (f8_few_tokens(c.M, c.N, kCus)) {
        const int tokens = c.M <= 16 ? 16 : 32;
        const int waves = tiles_across(c.M, tokens) * tiles_across(c.N, 16) <= kCus ? 16 : 8;
        ++g_launches.at(few(waves, tokens, c.aligned, c.w_rows));
        return;
    }
    const F8Cost &cost = f8_cost(c.aligned, c.wide, c.w_rows);
    const int large = f8_largest(cost);
    const int64_t whole = f8_whole_rounds(cost, large, c.M, c.N, c.K, kCus);
    if (whole > 0) launch(c, large, whole);
    launch(c, f8_tile(cost, c.M, c.N - whole, c.K, kCus), c.N - whole);
}

}  // namespace

int main() {
    for (int v = 0; v < 4; ++v)
        for (const int waves : {8, 16})
            for (const int tokens : {16, 32}) g_launches[few(waves, tokens, v & 1, v & 2)] = 0;
    for (int v = 0; v < 8; ++v)
        for (int i = 0; i < kF8TileCount; ++i) {
            if (f8_cost(v & 1, v & 2, v & 4).round[i] == 0) continue;
            for (const int parts : {1, 2, 4})
                if (parts == 1 || (i == kF8TileCount - 1 && (parts == 2 || (v & 1))))
                    g_launches[tiled(i, parts, v & 1, v & 2, v & 4)] = 0;
        }
    for (const Call &c : kCalls) product(c);
    std::printf("ok\n");
    for (const auto &k : g_launches) std::printf("%d %s\n", k.second, k.first.c_str());
    return 0;
}
