// Launches of the 8-bit floating-point product.
#include "f8_plan.h"
#include "f8_ring.h"
#include "f8_rows.h"

namespace bsr {

namespace {

template <class K, int BM> void launch_tiles(void (*kernel)(F8Args), F8Args a, void *stream) {
    a.p.tiles_m = int((a.p.M + BM - 1) / BM);
    a.p.tiles_n = int((a.p.N + K::kTileN - 1) / K::kTileN);
    hipLaunchKernelGGL(kernel, dim3(unsigned(a.p.tiles_m) * unsigned(a.p.tiles_n)), dim3(K::kThreads), 0,
                       as_stream(stream), a);
}

template <int BM, int BN, int WM, int WN, int XF, bool WROWS, bool WIDE, bool DIRECT, int PARTS = 1>
void launch_ring(const F8Args &a, void *stream) {
    launch_tiles<F8RingKernel<BM, BN, WM, WN, XF, WROWS, WIDE, DIRECT, PARTS>, BM>(
        f8_ring_kernel<BM, BN, WM, WN, XF, WROWS, WIDE, DIRECT, PARTS>, a, stream);
}
template <int XF, bool WROWS, bool WIDE, bool DIRECT> void launch_tile(const F8Args &a, int tile, void *stream) {
    constexpr F8Cost cost = kF8Costs[DIRECT ? 1 : 0][WIDE ? 1 : 0][WROWS ? 1 : 0];
    switch (tile) {
        case 0:
            if constexpr (cost.round[0] > 0)
                return launch_ring<256, 256, 2, 4, XF, WROWS, WIDE, DIRECT>(a, stream);
            break;
        case 1:
            if constexpr (cost.round[1] > 0)
                return launch_ring<192, 256, 2, 4, XF, WROWS, WIDE, DIRECT>(a, stream);
            break;
        case 2:
            if constexpr (cost.round[2] > 0)
                return launch_ring<128, 256, 2, 4, XF, WROWS, WIDE, DIRECT>(a, stream);
            break;
        case 3: return launch_ring<128, 128, 2, 4, XF, WROWS, WIDE, DIRECT>(a, stream);
        default:
            const int parts = f8_parts(DIRECT, a.p.M, a.p.N, a.p.Kb, device_cu_count());
            if constexpr (DIRECT)
                if (parts == 4) return launch_ring<64, 64, 2, 2, XF, WROWS, WIDE, DIRECT, 4>(a, stream);
            if (parts == 2) return launch_ring<64, 64, 2, 2, XF, WROWS, WIDE, DIRECT, 2>(a, stream);
            return launch_ring<64, 64, 2, 2, XF, WROWS, WIDE, DIRECT>(a, stream);
    }
}

// The product's channels from n on (a multiple of 128), as a product of its own.
F8Args channels_from(F8Args a, int64_t n, bool w_rows) {
    a.p.B0 += n * a.p.ldb0;
    a.p.b0 = a.p.b0 ? a.p.b0 + n : nullptr;
    a.p.out = static_cast<char *>(a.p.out) + n * (a.p.out_bf16 ? 2 : 4);
    a.p.N -= n;
    a.sw += w_rows ? n : n / kF8Block;
    return a;
}

bool rows_aligned(const void *p, int64_t ld) {
    return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(ld)) & 15) == 0;
}

template <int WAVES, int NT, int XF, bool WROWS> void launch_rows(const F8Args &a, bool aligned, void *stream) {
    using K = F8RowsKernel<WAVES, NT, XF, WROWS, true>;
    const auto kernel = aligned ? f8_rows_kernel<WAVES, NT, XF, WROWS, true>
                                : f8_rows_kernel<WAVES, NT, XF, WROWS, false>;
    const unsigned groups_n = unsigned((a.p.N + K::kChannels - 1) / K::kChannels);
    const unsigned groups_m = unsigned((a.p.M + 16 * NT - 1) / (16 * NT));
    hipLaunchKernelGGL(kernel, dim3(groups_n, groups_m), dim3(64 * K::kWaves), 0, as_stream(stream), a);
}
template <int NT, int XF, bool WROWS>
void launch_few(const F8Args &a, bool aligned, int64_t cus, void *stream) {
    const int64_t groups = tiles_across(a.p.M, 16 * NT) * tiles_across(a.p.N, 16);
    groups <= cus ? launch_rows<16, NT, XF, WROWS>(a, aligned, stream)
                  : launch_rows<8, NT, XF, WROWS>(a, aligned, stream);
}

template <int XF, bool WROWS, bool WIDE> void product(const F8Args &a, void *stream) {
    const bool aligned = rows_aligned(a.p.A, a.p.lda) && rows_aligned(a.p.B0, a.p.ldb0);
    const int64_t cus = device_cu_count(), M = a.p.M, N = a.p.N, K = a.p.Kb;
    // 64 x 1024 x 4096 takes 9 us there and 14 in tiles (fp32 output 21), 128 x 1024 x 8192 14 and 25; two
    // rounds of it, 32 x 12288 x 4096, 20 and 19 (fp32 22).
    if (f8_few_tokens(M, N, cus))
        return M <= 16 ? launch_few<1, XF, WROWS>(a, aligned, cus, stream)
                       : launch_few<2, XF, WROWS>(a, aligned, cus, stream);
    const F8Cost &cost = f8_cost(aligned, WIDE, WROWS);
    const auto launch = aligned ? launch_tile<XF, WROWS, WIDE, true> : launch_tile<XF, WROWS, WIDE, false>;
    const int large = f8_largest(cost);
    const int64_t whole = f8_whole_rounds(cost, large, M, N, K, cus);
    if (whole == 0) return launch(a, f8_tile(cost, M, N, K, cus), stream);
    const F8Args rest = channels_from(a, whole, WROWS);
    F8Args first = a;
    first.p.N = whole;
    launch(first, large, stream);
    launch(rest, f8_tile(cost, M, rest.p.N, K, cus), stream);
}
template <int XF> void product(const F8Args &a, bool w_rows, void *stream) {
    const auto f = w_rows ? (a.p.out_bf16 ? product<XF, true, false> : product<XF, true, true>)
                          : (a.p.out_bf16 ? product<XF, false, false> : product<XF, false, true>);
    f(a, stream);
}

}  // namespace

bsr_status launch_matmul_f8(const void *Xq, int x_format, int64_t T, int64_t K, int64_t ldx,
                            const float *sx, int64_t ldsx, const void *Wq, int64_t N, int64_t ldw,
                            const float *sw, int64_t ldsw, int w_block_rows, const float *bias, void *Y,
                            int y_dtype, int64_t ldy, void *stream) {
    F8Args a{};
    a.p.A = static_cast<const char *>(Xq);
    a.p.B0 = static_cast<const char *>(Wq);
    a.p.lda = ldx;
    a.p.ldb0 = ldw;
    a.p.M = T;
    a.p.N = N;
    a.p.Kb = int(K);
    a.p.b0 = bias;
    a.p.out = Y;
    a.p.ldo = ldy;
    a.p.out_bf16 = y_dtype == BSR_BF16;
    a.sx = sx;
    a.sw = sw;
    a.ldsx = ldsx;
    a.ldsw = ldsw;
    (x_format == BSR_E4M3 ? product<BSR_E4M3> : product<BSR_E5M2>)(a, w_block_rows == 1, stream);
    return launch_status();
}

}  // namespace bsr
