// The product of 8-bit floating-point matrices (f8_product.h) for few tokens: the weights go straight from
// memory into the operand registers, and that read is the whole cost.
//
// A workgroup makes 16 channels for 16 NT tokens (blockIdx.y counts groups of them).  Its waves split the
// contraction: wave w takes every WAVES-th run of kHeld blocks, loads their codes and scales all at once,
// and keeps its own scaled sums; they are added over the waves, in order, through LDS.  A single token is
// bound by latency: 4096 columns are one run per wave, so that everything a workgroup needs is in flight
// together.  Where every workgroup has a CU to itself sixteen waves share the work, else eight (one token,
// 4096 to 4096: 6.0 and 6.7 us; 4096 to 12288: 15.4 and 13.7).  Codes are widened to bf16 for either output
// type, which costs nothing beside the loads.
#pragma once

#include "f8_product.h"

namespace bsr {

// One lane's view of a row: 16-byte chunks at byte `col` of it and whole blocks further.  Rows past the end
// stand for the last one: what they give reaches only outputs that do not exist.  ALIGNED: rows start on
// 16-byte boundaries, chunks are loaded whole through a range-checked load whose range ends with the dword
// that holds the last byte, and what lies beyond a row's end is replaced by zeros.
template <bool ALIGNED> struct F8Chunks;
template <> struct F8Chunks<true> {
    const char *base;
    unsigned bytes, off;
    __device__ __forceinline__ void set(const Source &s, int row, int col, int Kb) {
        base = s.base;
        bytes = (unsigned((s.rows - 1) * s.pitch) + unsigned(Kb) + 3u) & ~3u;
        off = unsigned(row < s.rows ? row : s.rows - 1) * unsigned(s.pitch) + unsigned(col);
    }
    // `left` bytes of the row are left from the chunk's start on.
    __device__ __forceinline__ i32x4 load(int kb, int left) const {
        const unsigned at = left > 0 ? off + unsigned(kb) : 0x80000000u;        // out of range: zeros
        return __builtin_bit_cast(i32x4,
                                  __builtin_amdgcn_raw_buffer_load_b128(buffer_rsrc(base, bytes), at, 0, 0));
    }
    static __device__ __forceinline__ i32x4 cut(i32x4 v, int left) { return first_bytes(v, left); }
};
template <> struct F8Chunks<false> : RowChunks<int8_t, Load::kShifted> {
    static __device__ __forceinline__ i32x4 cut(i32x4 v, int) { return v; }     // load() has zeros there
};

template <int WAVES, int NT, int XF, bool WROWS, bool ALIGNED> struct F8RowsKernel {
    static constexpr int kWaves = WAVES, kChannels = 16;
    static constexpr int kHeld = NT == 1 && WAVES <= 8 ? 4 : 2;        // blocks of a run
    static constexpr int kLds = kWaves * NT * 64 * 16;

    static __device__ __forceinline__ void run(const F8Args &args, char *lds) {
        const ProductArgs &a = args.p;
        const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
        const int64_t n0 = int64_t(blockIdx.x) * kChannels;
        const int64_t m0 = int64_t(blockIdx.y) * (16 * NT), left_m = a.M - m0;
        const int channels = int(a.N - n0 < kChannels ? a.N - n0 : kChannels);
        const int tokens = int(left_m < 16 * NT ? left_m : 16 * NT);
        const Source from_x{a.A + m0 * a.lda, a.lda, tokens}, from_w{a.B0 + n0 * a.ldb0, a.ldb0, channels};
        const int fr = lane & 15, fc = lane >> 4;
        F8Chunks<ALIGNED> cw, cx[NT];
        cw.set(from_w, fr, fc * kChunk, a.Kb);
        const float *sx[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            cx[i].set(from_x, 16 * i + fr, fc * kChunk, a.Kb);
            sx[i] = args.sx + m0 + (16 * i + fr < tokens ? 16 * i + fr : tokens - 1);
        }
        const float *sw = args.sw + (WROWS ? n0 + 4 * fc : n0 / kF8Block);
        const int cnt = channels - 4 * fc;               // of the lane's four channels; 4 or more: all
        const int blocks = (a.Kb + kF8Block - 1) / kF8Block;
        f32x4 acc[NT] = {};
        for (int b0 = wave * kHeld; b0 < blocks; b0 += kWaves * kHeld) {
            i32x4 w[kHeld][2], x[kHeld][NT][2];
            f32x4 scale_w[kHeld];
            float scale_x[kHeld][NT];
            const int kb0 = b0 * kF8Block, left0 = a.Kb - fc * kChunk - kb0;
#pragma unroll
            for (int s = 0; s < kHeld; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int at = s * kF8Block + h * 64;
                    w[s][h] = cw.load(kb0 + at, left0 - at);
#pragma unroll
                    for (int i = 0; i < NT; ++i) x[s][i][h] = cx[i].load(kb0 + at, left0 - at);
                }
#pragma unroll
            for (int s = 0; s < kHeld; ++s) {
                const int b = b0 + s < blocks ? b0 + s : blocks - 1;     // one that exists
#pragma unroll
                for (int i = 0; i < NT; ++i) scale_x[s][i] = sx[i][b * args.ldsx];
                if constexpr (WROWS) {
                    scale_w[s] = load4(sw, b * args.ldsw, cnt, 0.0f);
                } else {
                    const float one = sw[b * args.ldsw];
                    scale_w[s] = f32x4{one, one, one, one};
                }
            }
#pragma unroll
            for (int s = 0; s < kHeld; ++s) {
                if (b0 + s >= blocks) break;
                const int left = left0 - s * kF8Block;
                const auto whole = [&](i32x4 lo, i32x4 hi) {
                    if (ALIGNED && a.Kb - kb0 - s * kF8Block < kF8Block)         // the row ends in this block
                        return join_chunks(cw.cut(lo, left), cw.cut(hi, left - 64));
                    return join_chunks(lo, hi);
                };
                F8Fragment<BSR_E4M3, true> fw;
                fw.set(whole(w[s][0], w[s][1]));
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    F8Fragment<XF, true> fx;
                    fx.set(whole(x[s][i][0], x[s][i][1]));
                    const f32x4 sum = block_sums<XF>(fw, fx);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[i][e] = fmaf(sum[e], scale_w[s][e] * scale_x[s][i], acc[i][e]);
                }
            }
        }
        f32x4 *part = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
        for (int i = 0; i < NT; ++i) part[(wave * NT + i) * 64 + lane] = acc[i];
        __syncthreads();
        // Wave i joins token group i: token 16 i + fr, channels n0 + 4 fc .. + 3.
        if (wave >= NT) return;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < kWaves; ++v) sum += part[(v * NT + wave) * 64 + lane];
        const int64_t m = m0 + 16 * wave + fr, n = n0 + 4 * fc;
        if (m < a.M && cnt > 0)
            finish4<bf16, Out::kScale, false>(a, ChannelQuad<bf16, Out::kScale>(a, n, cnt), m, n, cnt,
                                              __builtin_bit_cast(i32x4, sum), i32x4{0, 0, 0, 0});
    }
};

template <int WAVES, int NT, int XF, bool WROWS, bool ALIGNED>
__global__ __launch_bounds__(64 * WAVES) void f8_rows_kernel(F8Args a) {
    using K = F8RowsKernel<WAVES, NT, XF, WROWS, ALIGNED>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
