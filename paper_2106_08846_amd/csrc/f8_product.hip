// Launches of the 8-bit floating-point product.
#include "dense_plan.h"
#include "f8_product.h"

namespace bsr {

namespace {

template <class K, int BM> void launch_tiles(void (*kernel)(F8Args), F8Args a, void *stream) {
    a.p.tiles_m = int((a.p.M + BM - 1) / BM);
    a.p.tiles_n = int((a.p.N + K::kTileN - 1) / K::kTileN);
    hipLaunchKernelGGL(kernel, dim3(unsigned(a.p.tiles_m) * unsigned(a.p.tiles_n)), dim3(K::kThreads), 0,
                       as_stream(stream), a);
}

template <int XF, bool WROWS, bool WIDE> void product(const F8Args &a, void *stream) {
    launch_tiles<F8TileKernel<64, 64, 2, 2, XF, WROWS, WIDE>, 64>(
        f8_tile_kernel<64, 64, 2, 2, XF, WROWS, WIDE>, a, stream);
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
