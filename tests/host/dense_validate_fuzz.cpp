// Host-side fuzz of the 8-bit and gated entry points' argument checks (csrc/validate.cpp), built with
// AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_dense_host.py: hostile sizes, pitches,
// enum values and pointers, which the checks never dereference.  A call that is accepted must keep to
// the limits that the kernels' 32-bit offsets and grids rest on.  Prints "ok" and the number of calls
// and of accepted ones.
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

bsr_gated_t block(int32_t dtype) {
    bsr_gated_t w{};
    w.K = i64();
    w.F = i64();
    w.ldg = pitch(w.K);
    w.ldu = pitch(w.K);
    w.Wg = p<void>();
    w.Wu = p<void>();
    w.sg = p<float>();
    w.su = p<float>();
    w.bg = next() % 2 ? p<float>() : nullptr;
    w.bu = next() % 2 ? p<float>() : nullptr;
    std::memcpy(&w.dtype, &dtype, 4);
    w.act = e32(4);
    return w;
}

}  // namespace

int main() {
    const int64_t wide = bsr::kDenseMaxWidth, tall = bsr::kDenseMaxTokens;
    long calls = 0, accepted = 0;
    for (int n = 0; n < 400000; ++n) {
        const int64_t T = i64(), K = i64(), N = i64();
        const int64_t ldx = pitch(K), ldw = pitch(K), ldy = pitch(N), ldq = pitch(K);
        ++calls;
        if (bsr::check_quantize_rows(p<void>(), e32(3), T, K, ldx, p<int8_t>(), ldq, p<float>()) ==
            BSR_OK) {
            ++accepted;
            require(T >= 0 && T <= tall && K >= 1 && K <= ldx && ldx <= wide && K <= ldq && ldq <= wide,
                    "quantize");
        }
        if (bsr::check_matmul_i8(p<int8_t>(), T, K, ldx, p<float>(), p<int8_t>(), N, ldw, p<float>(),
                                 p<float>(), p<void>(), e32(3), ldy) == BSR_OK) {
            ++accepted;
            require(T >= 0 && T <= tall && K >= 1 && K <= bsr::kI8MaxK && K <= ldx && ldx <= wide &&
                        K <= ldw && ldw <= wide && N >= 1 && N <= ldy && ldy <= wide &&
                        T * N <= bsr::kDenseMaxOut, "matmul");
        }
        const int32_t dt = e32(3);
        const bsr_gated_t w = block(dt);
        const int64_t lx = pitch(w.K), lh = pitch(w.F), lp = pitch(w.F), ldd = pitch(w.K);
        auto sound = [&](const char *what) {
            ++accepted;
            require(T >= 0 && T <= tall && w.K >= 1 && w.F >= 1 && w.K <= w.ldg && w.ldg <= wide &&
                        w.K <= w.ldu && w.ldu <= wide && w.K <= lx && lx <= wide &&
                        T * w.F <= bsr::kDenseMaxOut / 2 && w.act >= 0 && w.act <= 3, what);
        };
        const bool keep = next() % 2;
        if (bsr::check_gated(p<void>(), T, lx, &w, p<void>(), lh, keep ? p<float>() : nullptr,
                             keep ? p<float>() : nullptr, lp) == BSR_OK)
            sound("gated"), require(dt != BSR_I8 && lh >= w.F && lh <= wide, "gated");
        if (bsr::check_gated_i8(p<int8_t>(), T, lx, p<float>(), &w, p<void>(), e32(3), lh) == BSR_OK)
            sound("gated_i8"), require(dt == BSR_I8 && w.K <= bsr::kI8MaxK, "gated_i8");
        const size_t room = next() % 2 ? size_t(1) << 60 : size_t(next() % (1 << 24));
        if (bsr::check_gated_backward(p<void>(), lh, p<void>(), T, lx, &w, p<float>(), p<float>(), lp,
                                      p<void>(), ldd, p<void>(), p<void>(), ldd, p<void>(), p<void>(),
                                      e32(3), reinterpret_cast<void *>(uintptr_t(1) << 62), room) ==
            BSR_OK) {
            sound("backward");
            require(T <= bsr::kGatedMaxBackwardTokens && 2 * w.F <= wide, "backward");
            require(bsr_gated_workspace_bytes(T, w.K, w.F, w.dtype) <= room, "workspace");
        }
        (void)bsr_gated_workspace_bytes(T, K, N, next() % 2 ? BSR_BF16 : BSR_F32);
    }
    if (accepted < calls / 20) {
        std::printf("only %ld of %ld accepted\n", accepted, calls);
        return 1;
    }
    std::printf("ok %ld %ld\n", calls, accepted);
    return 0;
}
