// Host-side fuzz of the layer norm's and the 8-bit floating-point entry points' argument checks
// (csrc/validate.cpp), built with AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_norm_f8_abi.py: hostile sizes, pitches, enum values and pointers, which the checks never
// dereference.  A call that is accepted must keep to the limits that the kernels' 32-bit offsets and grids
// rest on.  Prints "ok" and the number of calls and of accepted ones.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>

#include "bsr_internal.h"

namespace {

uint64_t g_state = 0x9E3779B97F4A7C15ull;
uint64_t next() {   // xorshift64*
    g_state ^= g_state >> 12;
    g_state ^= g_state << 25;
    g_state ^= g_state >> 27;
    return g_state * 0x2545F4914F6CDD1Dull;
}
int64_t i64() {
    static const int64_t some[] = {0, 1, 2, 15, 16, 17, 64, 768, 4096, 131071, 131072, (1 << 20) - 64,
                                   (1 << 20) - 1, 1 << 20, (1 << 20) + 1, 1 << 24, (1 << 24) + 1,
                                   int64_t(1) << 31, int64_t(1) << 40, int64_t(1) << 62, -1, -4096,
                                   std::numeric_limits<int64_t>::max(),
                                   std::numeric_limits<int64_t>::min()};
    return next() % 3 ? int64_t(next() % 3000) + 1 : some[next() % (sizeof some / sizeof some[0])];
}
int64_t pitch(int64_t width) {   // mostly a valid one
    if (next() % 8 == 0) return i64();
    return width > (int64_t(1) << 61) || width < 0 ? width : width + int64_t(next() % 40);
}
int32_t e32(int32_t n) { return next() % 10 ? int32_t(next() % n) : int32_t(next()); }
template <class T> const T *p() {
    if (next() % 40 == 0) return nullptr;
    return reinterpret_cast<const T *>(uintptr_t(next() % 4096) << 44 | (next() % 64) * 4);
}
void require(bool ok, const char *what) {
    if (!ok) {
        std::printf("accepted beyond its limits: %s\n", what);
        std::exit(1);
    }
}

}  // namespace

int main() {
    const int64_t wide = bsr::kDenseMaxWidth, tall = bsr::kDenseMaxTokens;
    long calls = 0, accepted = 0;
    auto blocks = [](int64_t n, int64_t rows) { return (n + rows - 1) / rows; };
    for (int n = 0; n < 400000; ++n) {
        const int64_t T = i64(), K = i64(), N = i64();
        const int64_t a = pitch(K), b = pitch(K), c = pitch(K), d = pitch(K);
        const float eps = next() % 8 ? 1e-5f : next() % 2 ? -1.0f : std::nanf("");
        calls += 4;
        const bool residual = next() % 2, keep = next() % 2;
        if (bsr::check_layer_norm(p<void>(), a, residual ? p<void>() : nullptr, b, T, K, e32(3), p<float>(),
                                  p<float>(), eps, p<void>(), c, residual ? p<void>() : nullptr, d,
                                  keep ? p<float>() : nullptr, keep ? p<float>() : nullptr) == BSR_OK) {
            ++accepted;
            require(T >= 0 && T <= tall && K >= 1 && K <= a && a <= wide && K <= c && c <= wide &&
                        eps >= 0.0f, "norm");
        }
        const size_t room = next() % 2 ? size_t(1) << 60 : size_t(next() % (1 << 24));
        if (bsr::check_layer_norm_backward(p<void>(), a, p<void>(), b, T, K, e32(3), p<float>(), p<float>(),
                                           p<float>(), p<void>(), c, p<void>(), d, p<void>(), p<void>(),
                                           e32(3), reinterpret_cast<void *>(uintptr_t(1) << 62), room) ==
            BSR_OK) {
            ++accepted;
            require(T >= 0 && T <= tall && K >= 1 && K <= a && a <= wide && K <= b && b <= wide, "gradients");
            const size_t need = bsr_layer_norm_workspace_bytes(T, K);
            require(need > 0 && need < size_t(1) << 33, "workspace");
            const bsr::NormWorkspace w = bsr::layer_norm_workspace(T, K);
            require(w.groups >= (T > 0) && w.groups <= 512 && w.groups <= (T > 0 ? T : 0), "groups");
        }
        const int32_t rows = next() % 2 ? 1 : next() % 8 ? 128 : int32_t(next());
        const int64_t ls = pitch(T), lt = pitch(T), lst = pitch(K);
        const bool by_rows = next() % 2, by_columns = !by_rows || next() % 2;
        const void *QT = by_columns ? p<void>() : nullptr;
        if (bsr::check_quantize_f8(p<void>(), e32(3), T, K, a, rows, e32(2), by_rows ? p<void>() : nullptr, b,
                                   by_rows ? p<float>() : nullptr, ls, QT, lt,
                                   by_columns ? p<float>() : nullptr, lst) == BSR_OK) {
            ++accepted;
            require(T >= 0 && T <= tall && K >= 1 && K <= a && a <= wide && (rows == 1 || rows == 128),
                    "codes");
            if (T > 0 && QT) require(lt >= T && lt <= wide && lst >= blocks(K, rows), "transpose");
        }
        const int64_t ly = pitch(N), lsw = pitch(N);
        if (bsr::check_matmul_f8(p<void>(), e32(2), T, K, a, p<float>(), ls, p<void>(), N, b, p<float>(), lsw,
                                 rows, p<float>(), p<void>(), e32(3), ly) == BSR_OK) {
            ++accepted;
            require(T >= 0 && T <= tall && K >= 1 && K <= a && a <= wide && K <= b && b <= wide && N >= 1 &&
                        N <= ly && ly <= wide && T <= ls && blocks(N, rows) <= lsw && lsw <= tall &&
                        T * N <= bsr::kDenseMaxOut, "product");
        }
    }
    if (accepted < calls / 20) {
        std::printf("only %ld of %ld accepted\n", accepted, calls);
        return 1;
    }
    std::printf("ok %ld %ld\n", calls, accepted);
    return 0;
}
