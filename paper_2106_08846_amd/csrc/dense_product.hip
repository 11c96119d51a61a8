// The dense products: 8-bit rows with scales, the gated block's projections and its gradients.  A
// 64 x 64 tile of the output per workgroup, 16 columns of the contraction in LDS at a time, four by
// four outputs to a thread, fp32 (8-bit operands: int32) accumulation.
#include <type_traits>

#include "dense_math.h"

namespace bsr {

namespace {

constexpr int kTile = 64;
constexpr int kDepth = 16;
constexpr int kThreads = 256;

template <class T> struct Acc { using type = float; };
template <> struct Acc<int8_t> { using type = int; };
__device__ __forceinline__ int widen(int8_t x) { return x; }
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16 x) { return to_float(x); }

// One operand: element (row, k) at p[row * rs + k * cs], zero outside rows x K.
template <class T> struct Operand {
    const T *p;
    int64_t rs, cs, rows;
};

template <class T>
__device__ void accumulate(typename Acc<T>::type (&acc)[4][4], const Operand<T> &A,
                           const Operand<T> &B, int64_t m0, int64_t n0, int64_t K,
                           typename Acc<T>::type (*sa)[kTile + 1],
                           typename Acc<T>::type (*sb)[kTile + 1]) {
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int64_t k0 = 0; k0 < K; k0 += kDepth) {
        for (int e = threadIdx.x; e < kTile * kDepth; e += kThreads) {
            const int r = e / kDepth, k = e % kDepth;
            const bool in = k0 + k < K;
            sa[k][r] = in && m0 + r < A.rows ? widen(A.p[(m0 + r) * A.rs + (k0 + k) * A.cs]) : 0;
            sb[k][r] = in && n0 + r < B.rows ? widen(B.p[(n0 + r) * B.rs + (k0 + k) * B.cs]) : 0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDepth; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += sa[k][ty + 16 * i] * sb[k][tx + 16 * j];
        __syncthreads();
    }
}

// DUAL: two products of the same A, passed to the epilogue together; otherwise the sum of one or two
// products (A2.p set) over K each.
template <class T, bool DUAL, class Epi>
__global__ __launch_bounds__(kThreads) void product_kernel(Operand<T> A, Operand<T> B,
                                                           Operand<T> A2, Operand<T> B2,
                                                           int64_t K, int64_t ntiles, Epi epi) {
    using A_t = typename Acc<T>::type;
    __shared__ A_t sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
    const int64_t m0 = int64_t(blockIdx.x) / ntiles * kTile, n0 = int64_t(blockIdx.x) % ntiles * kTile;
    A_t acc[DUAL ? 2 : 1][4][4] = {};
    accumulate(acc[0], A, B, m0, n0, K, sa, sb);
    if (A2.p) accumulate(acc[DUAL ? 1 : 0], A2, B2, m0, n0, K, sa, sb);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < A.rows && n < B.rows)
                epi(m, n, float(acc[0][i][j]), float(acc[DUAL ? 1 : 0][i][j]));
        }
}

template <class T> struct StoreEpi {   // out[m][n], or out2[m - split][n] for m >= split
    T *out, *out2;
    int64_t ld, split;
    __device__ void operator()(int64_t m, int64_t n, float v, float) const {
        if (m < split)
            out[m * ld + n] = from_float<T>(v);
        else
            out2[(m - split) * ld + n] = from_float<T>(v);
    }
};

template <class T> struct ScaleEpi {
    const float *sx, *sw, *bias;
    T *Y;
    int64_t ldy;
    __device__ void operator()(int64_t m, int64_t n, float v, float) const {
        const float y = v * sx[m] * sw[n];
        Y[m * ldy + n] = from_float<T>(bias ? y + bias[n] : y);
    }
};

template <class T, int ACT> struct GatedEpi {
    const float *sx, *sg, *su, *bg, *bu;
    T *H;
    float *G, *U;
    int64_t ldh, ldp;
    __device__ void operator()(int64_t m, int64_t n, float g, float u) const {
        if (sx) {
            g = g * sx[m] * sg[n];
            u = u * sx[m] * su[n];
        }
        if (bg) g += bg[n];
        if (bu) u += bu[n];
        H[m * ldh + n] = from_float<T>(activate<ACT>(g) * u);
        if (G) {
            G[m * ldp + n] = g;
            U[m * ldp + n] = u;
        }
    }
};

template <class T, bool DUAL, class Epi>
void launch(const Operand<T> &A, const Operand<T> &B, const Operand<T> &A2, const Operand<T> &B2,
            int64_t K, const Epi &epi, void *stream) {
    const int64_t mt = (A.rows + kTile - 1) / kTile, nt = (B.rows + kTile - 1) / kTile;
    hipLaunchKernelGGL((product_kernel<T, DUAL, Epi>), dim3(unsigned(mt * nt)), dim3(kThreads), 0,
                       as_stream(stream), A, B, A2, B2, K, nt, epi);
}

// f(constant activation) for the block's activation.
template <class F> void with_act(int act, F &&f) {
    switch (act) {
        case BSR_ACT_SILU: f(std::integral_constant<int, BSR_ACT_SILU>{}); break;
        case BSR_ACT_GELU: f(std::integral_constant<int, BSR_ACT_GELU>{}); break;
        case BSR_ACT_GELU_TANH: f(std::integral_constant<int, BSR_ACT_GELU_TANH>{}); break;
        default: f(std::integral_constant<int, BSR_ACT_RELU>{}); break;
    }
}

template <class T, class TO>
void gated(const void *X, int64_t T_, int64_t ldx, const float *sx, const bsr_gated_t &W, void *H,
           int64_t ldh, float *G, float *U, int64_t ldp, void *stream) {
    const Operand<T> A{static_cast<const T *>(X), ldx, 1, T_};
    const Operand<T> Bg{static_cast<const T *>(W.Wg), W.ldg, 1, W.F};
    const Operand<T> Bu{static_cast<const T *>(W.Wu), W.ldu, 1, W.F};
    with_act(W.act, [&](auto act) {
        const GatedEpi<TO, decltype(act)::value> epi{sx, W.sg, W.su, W.bg, W.bu,
                                                     static_cast<TO *>(H), G, U, ldh, ldp};
        launch<T, true>(A, Bg, A, Bu, W.K, epi, stream);
    });
}

// D[t][f] = dH U act'(G), D[t][F + f] = dH act(G), and the sums of their columns over 64 rows.
template <class T, int ACT>
__global__ __launch_bounds__(kThreads) void gated_slope_kernel(
    const T *__restrict__ dH, int64_t lddh, const float *__restrict__ G,
    const float *__restrict__ U, int64_t ldp, int64_t T_, int64_t F, T *__restrict__ D,
    float *__restrict__ partial) {
    const int64_t f = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (f >= F) return;
    const int64_t t0 = int64_t(blockIdx.y) * kGatedRowsPerPartial;
    const int64_t t1 = min(t0 + kGatedRowsPerPartial, T_);
    float sg = 0.0f, su = 0.0f;
    for (int64_t t = t0; t < t1; ++t) {
        float a, da;
        activate_slope<ACT>(G[t * ldp + f], a, da);
        const float dh = to_float(dH[t * lddh + f]);
        const float dg = dh * U[t * ldp + f] * da, du = dh * a;
        D[t * 2 * F + f] = from_float<T>(dg);
        D[t * 2 * F + F + f] = from_float<T>(du);
        sg += dg;
        su += du;
    }
    partial[int64_t(blockIdx.y) * 2 * F + f] = sg;
    partial[int64_t(blockIdx.y) * 2 * F + F + f] = su;
}

template <class T>
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(const float *__restrict__ partial,
                                                             int64_t blocks, int64_t F,
                                                             T *__restrict__ dbg,
                                                             T *__restrict__ dbu) {
    const int64_t f = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (f >= 2 * F) return;
    float s = 0.0f;
    for (int64_t b = 0; b < blocks; ++b) s += partial[b * 2 * F + f];
    if (f < F) {
        if (dbg) dbg[f] = from_float<T>(s);
    } else if (dbu) {
        dbu[f - F] = from_float<T>(s);
    }
}

template <class T, class TG>
void backward(const void *dH, int64_t lddh, const void *X, int64_t T_, int64_t ldx,
              const bsr_gated_t &W, const float *G, const float *U, int64_t ldp, void *dX,
              int64_t lddx, void *dWg, void *dWu, int64_t lddw, void *dbg, void *dbu, void *ws,
              void *stream) {
    const int64_t K = W.K, F = W.F;
    const GatedWorkspace lay = gated_workspace_layout(T_, K, F, raw_enum(W.dtype));
    T *D = reinterpret_cast<T *>(static_cast<char *>(ws) + lay.grad_offset);
    float *partial = reinterpret_cast<float *>(static_cast<char *>(ws) + lay.partial_offset);
    const int64_t blocks = (T_ + kGatedRowsPerPartial - 1) / kGatedRowsPerPartial;
    if (T_ > 0)
        with_act(W.act, [&](auto act) {
            hipLaunchKernelGGL((gated_slope_kernel<T, decltype(act)::value>),
                               dim3(unsigned((F + kThreads - 1) / kThreads), unsigned(blocks)),
                               dim3(kThreads), 0, as_stream(stream), static_cast<const T *>(dH),
                               lddh, G, U, ldp, T_, F, D, partial);
        });
    if (dbg || dbu)
        hipLaunchKernelGGL(bias_grad_kernel<TG>, dim3(unsigned((2 * F + kThreads - 1) / kThreads)),
                           dim3(kThreads), 0, as_stream(stream), partial, blocks, F,
                           static_cast<TG *>(dbg), static_cast<TG *>(dbu));
    const Operand<T> none{nullptr, 0, 0, 0};
    if (dX && T_ > 0)
        launch<T, false>(Operand<T>{D, 2 * F, 1, T_},
                         Operand<T>{static_cast<const T *>(W.Wg), 1, W.ldg, K},
                         Operand<T>{D + F, 2 * F, 1, T_},
                         Operand<T>{static_cast<const T *>(W.Wu), 1, W.ldu, K}, F,
                         StoreEpi<T>{static_cast<T *>(dX), nullptr, lddx, T_}, stream);
    if (dWg)
        launch<T, false>(Operand<T>{D, 1, 2 * F, 2 * F},
                         Operand<T>{static_cast<const T *>(X), 1, ldx, K}, none, none, T_,
                         StoreEpi<TG>{static_cast<TG *>(dWg), static_cast<TG *>(dWu), lddw, F},
                         stream);
}

}  // namespace

bsr_status launch_matmul_i8(const int8_t *Xq, int64_t T, int64_t K, int64_t ldx, const float *sx,
                            const int8_t *Wq, int64_t N, int64_t ldw, const float *sw,
                            const float *bias, void *Y, int y_dtype, int64_t ldy, void *stream) {
    const Operand<int8_t> A{Xq, ldx, 1, T}, B{Wq, ldw, 1, N}, none{nullptr, 0, 0, 0};
    if (y_dtype == BSR_BF16)
        launch<int8_t, false>(A, B, none, none, K,
                              ScaleEpi<bf16>{sx, sw, bias, static_cast<bf16 *>(Y), ldy}, stream);
    else
        launch<int8_t, false>(A, B, none, none, K,
                              ScaleEpi<float>{sx, sw, bias, static_cast<float *>(Y), ldy}, stream);
    return launch_status();
}

bsr_status launch_gated(const void *X, int64_t T, int64_t ldx, const bsr_gated_t &W, void *H,
                        int64_t ldh, float *G, float *U, int64_t ldp, void *stream) {
    if (raw_enum(W.dtype) == BSR_BF16)
        gated<bf16, bf16>(X, T, ldx, nullptr, W, H, ldh, G, U, ldp, stream);
    else
        gated<float, float>(X, T, ldx, nullptr, W, H, ldh, G, U, ldp, stream);
    return launch_status();
}

bsr_status launch_gated_i8(const int8_t *Xq, int64_t T, int64_t ldx, const float *sx,
                           const bsr_gated_t &W, void *H, int h_dtype, int64_t ldh, void *stream) {
    if (h_dtype == BSR_BF16)
        gated<int8_t, bf16>(Xq, T, ldx, sx, W, H, ldh, nullptr, nullptr, 0, stream);
    else
        gated<int8_t, float>(Xq, T, ldx, sx, W, H, ldh, nullptr, nullptr, 0, stream);
    return launch_status();
}

bsr_status launch_gated_backward(const void *dH, int64_t lddh, const void *X, int64_t T,
                                 int64_t ldx, const bsr_gated_t &W, const float *G,
                                 const float *U, int64_t ldp, void *dX, int64_t lddx, void *dWg,
                                 void *dWu, int64_t lddw, void *dbg, void *dbu, int grad_dtype,
                                 void *workspace, void *stream) {
    const bool b = raw_enum(W.dtype) == BSR_BF16, g = grad_dtype == BSR_BF16;
    const auto f = b ? (g ? backward<bf16, bf16> : backward<bf16, float>)
                     : (g ? backward<float, bf16> : backward<float, float>);
    f(dH, lddh, X, T, ldx, W, G, U, ldp, dX, lddx, dWg, dWu, lddw, dbg, dbu, workspace, stream);
    return launch_status();
}

}  // namespace bsr
