// The product of 8-bit floating-point matrices with scales for blocks of 128:
//   Y[m][n] = sum over blocks b of sx[b][m] sw[b][n'] (sum over k in b of A[m][k] B[n][k])  +  bias[n].
//
// A lane's operand of a block is 32 bytes of one row: chunks c and c + 4 of the block's eight for lane group
// c, the same of both operands (the order within a block does not matter).  The block's four sums per lane
// are added to the outputs with the scales by four vector instructions.
//
// Two ways to sum a block, by what the output can hold:
//   bf16 output: one 8-bit matrix instruction (16x16x128).  It aligns the products of every eight
//     consecutive k to the largest of them and drops what lies below 2^-13 of that one's power of two, then
//     adds the groups of eight in fp32 (measured on MI355X, all the 8-bit instructions alike, scaled or
//     not): 1.5e-5 of a sum of 128 normally distributed products, which bf16's 2^-8 hides.
//   fp32 output: the codes widened to bf16, which holds them exactly, and four bf16 instructions, which
//     keep every product: fp32 accuracy at half the matrix rate.
#pragma once

#include "dense_tile.h"

namespace bsr {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct F8Args {
    ProductArgs p;                // A: tokens, B0: channels, b0: bias; its scales are not used
    const float *sx, *sw;         // [blocks][pitch]
    int64_t ldsx, ldsw;
};

// Two codes of format F in half HI of a register, as bf16.
template <int F, bool HI> __device__ __forceinline__ int widen2(int codes) {
    if constexpr (F == BSR_E4M3)
        return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, HI));
    else
        return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes, 1.0f, HI));
}

// A lane's part of a block of one operand: 32 codes, as they are or widened.
template <int F, bool WIDE> struct F8Fragment;
template <int F> struct F8Fragment<F, false> {
    i32x8 v;
    __device__ __forceinline__ void set(i32x8 codes) { v = codes; }
};
template <int F> struct F8Fragment<F, true> {
    i32x4 v[4];
    __device__ __forceinline__ void set(i32x8 codes) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i / 2][i % 2 * 2] = widen2<F, false>(codes[i]);
            v[i / 2][i % 2 * 2 + 1] = widen2<F, true>(codes[i]);
        }
    }
};

// A block's sums for 16 channels x 16 tokens: lane: token lane % 16, channels 4 (lane / 16) .. + 3.
template <int XF>
__device__ __forceinline__ f32x4 block_sums(const F8Fragment<BSR_E4M3, false> &w,
                                            const F8Fragment<XF, false> &x) {
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, zero, 0, XF, 0, 0, 0, 0);
}
template <int XF>
__device__ __forceinline__ f32x4 block_sums(const F8Fragment<BSR_E4M3, true> &w,
                                            const F8Fragment<XF, true> &x) {
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = Mma<bf16>::step(w.v[i], x.v[i], sum);
    return sum;
}
__device__ __forceinline__ i32x8 join_chunks(i32x4 lo, i32x4 hi) {
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// BM x BN tile, WM x WN waves: operands go through registers into one of two LDS stages of one block
// each, together with the scales of its rows.  WROWS: a scale for each row of B, else for 128.
template <int BM, int BN, int WM, int WN, int XF, bool WROWS, bool WIDE> struct F8TileKernel {
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int TM = BM / WM, TN = BN / WN;
    static constexpr int NM = TM / kMF, NN = TN / kMF;
    static constexpr int kRowBytes = kF8Block, kRowChunks = kRowBytes / kChunk;
    static constexpr int kRowsPerPass = kThreads / kRowChunks;
    static constexpr int LA = BM / kRowsPerPass, LB = BN / kRowsPerPass;
    static constexpr int kScales = BM + (WROWS ? BN : 0);
    static constexpr int kStageBytes = (BM + BN) * kRowBytes + kScales * 4;
    static constexpr int kEpiBytes = WM * WN * epilogue_bytes(NN);
    static constexpr int kLds = 2 * kStageBytes > kEpiBytes ? 2 * kStageBytes : kEpiBytes;
    static constexpr int kTileN = BN;
    static_assert(BM % kRowsPerPass == 0 && BN % kRowsPerPass == 0 && BM <= kThreads && BN <= kThreads,
                  "whole passes");
    static_assert(kF8Block % TN == 0 && kStageBytes % 16 == 0, "one scale of B for a wave's channels");

    static __device__ __forceinline__ int swizzled(int row, int c) { return c ^ ((row >> 1) & 7); }

    static __device__ __forceinline__ void run(const F8Args &args, char *lds) {
        const ProductArgs &a = args.p;
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
        const int wm = wave % WM, wn = wave / WM;
        const TileRows<BM, kTileN, false> rows(a);
        const int c = tid & (kRowChunks - 1), r0 = tid / kRowChunks;
        i32x4 ha[LA], hb[LB];
        float hx = 0.0f, hw = 0.0f;
        RowChunks<int8_t, Load::kBytes> ca[LA], cb[LB];
#pragma unroll
        for (int i = 0; i < LA; ++i) ca[i].set(rows.a, i * kRowsPerPass + r0, c * kChunk, a.Kb);
#pragma unroll
        for (int i = 0; i < LB; ++i) cb[i].set(rows.b0, i * kRowsPerPass + r0, c * kChunk, a.Kb);
        const int steps = (a.Kb + kRowBytes - 1) / kRowBytes;
        const bool has_x = tid < BM && rows.m0 + tid < a.M;
        const bool has_w = WROWS && tid < BN && rows.n0 + tid < a.N;
        // The wave's channels share a scale where B has one for 128 rows; beyond the last, any.
        const int64_t n_wave = rows.n0 + wn * TN;
        const float *sw = args.sw + (WROWS ? rows.n0 : (n_wave < a.N ? n_wave : a.N - 1) / kF8Block);
        auto load = [&](int step) {                // zeros from Kb on
            const int kb = step * kRowBytes, left = a.Kb - c * kChunk - kb;
#pragma unroll
            for (int i = 0; i < LA; ++i) ha[i] = ca[i].load(kb, left);
#pragma unroll
            for (int i = 0; i < LB; ++i) hb[i] = cb[i].load(kb, left);
            if (has_x && step < steps) hx = args.sx[step * args.ldsx + rows.m0 + tid];
            if (has_w && step < steps) hw = sw[step * args.ldsw + tid];
        };
        auto put = [&](int buf) {
            char *p = lds + buf * kStageBytes;
#pragma unroll
            for (int i = 0; i < LA + LB; ++i) {
                const int row = (i < LA ? i : i - LA) * kRowsPerPass + r0;
                *reinterpret_cast<i32x4 *>(p + (i < LA ? 0 : BM * kRowBytes) + row * kRowBytes +
                                           swizzled(row, c) * kChunk) = i < LA ? ha[i] : hb[i - LA];
            }
            float *s = reinterpret_cast<float *>(p + (BM + BN) * kRowBytes);
            if (tid < BM) s[tid] = hx;
            if (WROWS && tid < BN) s[BM + tid] = hw;
        };
        f32x4 acc[NN][NM] = {};
        const int fr = lane % kMF, fc = lane / kMF;
        load(0);
        put(0);
        load(1);
        for (int s = 0; s < steps; ++s) {
            const float one = WROWS ? 0.0f : sw[s * args.ldsw];
            __syncthreads();
            const char *p = lds + (s & 1) * kStageBytes;
            const float *scale = reinterpret_cast<const float *>(p + (BM + BN) * kRowBytes);
            auto fetch = [&](int row) {
                const char *q = p + row * kRowBytes;
                return join_chunks(*reinterpret_cast<const i32x4 *>(q + swizzled(fr, fc) * kChunk),
                                   *reinterpret_cast<const i32x4 *>(q + swizzled(fr, fc + 4) * kChunk));
            };
            F8Fragment<BSR_E4M3, WIDE> fb[NN];
#pragma unroll
            for (int j = 0; j < NN; ++j) fb[j].set(fetch(BM + wn * TN + j * kMF + fr));
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                F8Fragment<XF, WIDE> fa;
                fa.set(fetch(wm * TM + i * kMF + fr));
                const float sx = scale[wm * TM + i * kMF + fr];
#pragma unroll
                for (int j = 0; j < NN; ++j) {
                    f32x4 of = {one, one, one, one};
                    if constexpr (WROWS)
                        of = *reinterpret_cast<const f32x4 *>(scale + BM + wn * TN + j * kMF + 4 * fc);
                    const f32x4 sum = block_sums<XF>(fb[j], fa);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[j][i][e] = fmaf(sum[e], sx * of[e], acc[j][i][e]);
                }
            }
            put((s + 1) & 1);
            load(s + 2);
        }
        __syncthreads();
        epilogue<bf16, Out::kScale, NN, NM>(a, acc, reinterpret_cast<float *>(lds + wave * epilogue_bytes(NN)),
                                            rows.m0 + wm * TM, rows.n0 + wn * TN);
    }
};

template <int BM, int BN, int WM, int WN, int XF, bool WROWS, bool WIDE>
__global__ __launch_bounds__(64 * WM * WN) void f8_tile_kernel(F8Args a) {
    using K = F8TileKernel<BM, BN, WM, WN, XF, WROWS, WIDE>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
