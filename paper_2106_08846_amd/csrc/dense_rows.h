// The dense products of few tokens (up to 32, or as many as one round of the chip takes): the weights go
// straight into the operand registers of the matrix instructions, and that read is the whole cost.
//
// A workgroup makes 16 channels (gated: of each matrix) for 16 NT tokens, at most 32 (blockIdx.y counts
// groups of them, each of which reads the weights).  Its eight waves split the contraction: wave w takes
// every eighth block of kBlock bytes of the rows, loads a block's chunks all at once, and keeps its own
// sums; they are added over the waves, in order, through LDS.  What bounds a single token is latency: 16
// rows of 4096 bytes are one block per wave, so that everything a workgroup needs is in flight together.
// The tokens come from the L2 (every workgroup reads all of its group), which is why the tile kernels
// take over beyond that.
//
// On MI355X an int8 token through 4096 x 4096 takes 5.2 us (its 16.8 MB would take 3.5 at a large
// copy's rate), a bf16 gated block of 4 tokens, 1024 to 4096 features, 6.3 us, and an int8 one of 16
// tokens, 4096 to 10240 features, 21 us: 84 MB at 4.0 TB/s, where a large copy moves 4.9.  One token of
// that block takes 35 us in bf16 and 65 in fp32 (5 TB/s).  Rows that are not aligned cost more: each
// chunk takes two loads and the shifts that put it together, and the choice between whole and partial
// chunks takes more scalar registers than there are (int8, 4 tokens of 4095 to 10240 features 46 us).
#pragma once

#include "dense_tile.h"

namespace bsr {

// NT: groups of 16 tokens.
template <class E, int NT, bool ALIGNED, Out OUT> struct RowsKernel {
    static constexpr bool kDual = OUT == Out::kGated;
    static constexpr int kWaves = 8;
    static constexpr int kChannels = 16;
    static constexpr int NW = kDual ? 2 : 1;
    // Chunks of 64 bytes per row that a wave loads at once: 16 bytes a lane and operand each.
    static constexpr int kHeld = NT == 2 || kDual ? 4 : 8;
    static constexpr int kBlock = 64 * kHeld;
    using M_ = Mma<E>;
    using Acc = typename M_::Acc;
    static constexpr int kLds = kWaves * NW * NT * 64 * 16;

    static __device__ __forceinline__ void run(const ProductArgs &a, char *lds) {
        const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
        const int64_t n0 = int64_t(blockIdx.x) * kChannels;
        const int rows = int(a.N - n0 < kChannels ? a.N - n0 : kChannels);
        const int64_t m0 = int64_t(blockIdx.y) * (16 * NT), left_m = a.M - m0;
        const Source sx{a.A + m0 * a.lda, a.lda, int(left_m < 16 * NT ? left_m : 16 * NT)};
        const Source sw[2] = {{a.B0 + n0 * a.ldb0, a.ldb0, rows},
                              {kDual ? a.B1 + n0 * a.ldb1 : nullptr, a.ldb1, rows}};
        const int fr = lane & 15, fc = lane >> 4;
        Acc acc[NW][NT] = {};
        constexpr Load kLoad = ALIGNED ? Load::kAligned : sizeof(E) == 4 ? Load::kBytes : Load::kShifted;
        RowChunks<E, kLoad> cw[NW], cx[NT];
#pragma unroll
        for (int j = 0; j < NW; ++j) cw[j].set(sw[j], fr, fc * kChunk, a.Kb);
#pragma unroll
        for (int i = 0; i < NT; ++i) cx[i].set(sx, 16 * i + fr, fc * kChunk, a.Kb);
        for (int kb = wave * kBlock; kb < a.Kb; kb += kWaves * kBlock) {
            const int left = a.Kb - fc * kChunk - kb;
            i32x4 w[kHeld][NW], x[kHeld][NT];
#pragma unroll
            for (int s = 0; s < kHeld; ++s)
#pragma unroll
                for (int j = 0; j < NW; ++j) w[s][j] = cw[j].load(kb + s * 64, left - s * 64);
#pragma unroll
            for (int s = 0; s < kHeld; ++s)
#pragma unroll
                for (int i = 0; i < NT; ++i) x[s][i] = cx[i].load(kb + s * 64, left - s * 64);
#pragma unroll
            for (int s = 0; s < kHeld; ++s)
#pragma unroll
                for (int j = 0; j < NW; ++j)
#pragma unroll
                    for (int i = 0; i < NT; ++i) acc[j][i] = M_::step(w[s][j], x[s][i], acc[j][i]);
        }
        Acc *part = reinterpret_cast<Acc *>(lds);
#pragma unroll
        for (int j = 0; j < NW; ++j)
#pragma unroll
            for (int i = 0; i < NT; ++i) part[((wave * NW + j) * NT + i) * 64 + lane] = acc[j][i];
        __syncthreads();
        // Wave i joins token group i: token 16 i + fr, channels n0 + 4 fc .. + 3.
        if (wave >= NT) return;
        Acc sum[2] = {};
#pragma unroll
        for (int v = 0; v < kWaves; ++v)
#pragma unroll
            for (int j = 0; j < NW; ++j) sum[j] += part[((v * NW + j) * NT + wave) * 64 + lane];
        const int64_t m = m0 + 16 * wave + fr, n = n0 + 4 * fc;
        const int cnt = a.N - n < 4 ? int(a.N - n) : 4;
        if (m < a.M && cnt > 0)
            finish4<E, OUT, false>(a, ChannelQuad<E, OUT>(a, n, cnt), m, n, cnt,
                                   __builtin_bit_cast(i32x4, sum[0]), __builtin_bit_cast(i32x4, sum[1]));
    }
};

template <class E, int NT, bool ALIGNED, Out OUT>
__global__ __launch_bounds__(512) void dense_rows_kernel(ProductArgs a) {
    using K = RowsKernel<E, NT, ALIGNED, OUT>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
