// Matrices in 8-bit floating point: an fp32 scale for each block of 1 x 128 or 128 x 128, by rows, by
// columns (the transpose) or both.
//
// Memory bound: every element is read once and a byte is written for it in each order that is wanted.
// By rows alone a wave takes rows of 512 elements, four blocks side by side, each held by 16 lanes.
// Everything else goes by tiles of 128 x 128 that stay in registers between the maxima and the codes; the
// transpose is made of 8 x 8 pieces in the lanes and put together in LDS.
//
// MI355X: by rows 8192 x 4096 bf16 17.5 us (5.8 TB/s), in both orders 6144 x 2048 bf16 9.8 us (5.2 TB/s), fp32
// 8192 x 4096 in blocks of 128 x 128 in both orders 39.5 us (5.1 TB/s).  Half of the first kernel's time was
// the divisions of every lane for its block's scale, before the lanes shared them.
#include <type_traits>
#include <utility>

#include "row_vec.h"

namespace bsr {

namespace {

constexpr int kThreads = 256;

struct QuantizeArgs {
    const void *X;
    int64_t T, ldx;
    int K;
    uint8_t *Q, *QT;
    float *scale, *scale_t;
    int64_t ldq, ldscale, ldqt, ldscale_t;
    int64_t t0;              // first row of this launch (a multiple of 128)
};

// What a block's largest magnitude (its bits) makes of it.  Two divisions, so the lanes that hold a block
// share the work: each makes the scale of one of their rows.
template <int FMT> struct BlockScale {
    static constexpr float kLargest = FMT == BSR_E4M3 ? 448.0f : 57344.0f;
    float scale, lift, r;    // r: 0 for a block of zeros or with an infinity or a NaN, whose codes are 0
    __device__ __forceinline__ explicit BlockScale(unsigned top) {
        const float a = __uint_as_float(top);
        const bool plain = top > 0 && top < 0x7f800000u;
        lift = a < 0x1p-64f ? 0x1p64f : 1.0f;
        r = plain ? kLargest / (a * lift) : 0.0f;
        scale = a / kLargest;
    }
    // Codes are x r.
    __device__ __forceinline__ bool ordinary() const { return r > 0.0f && lift == 1.0f; }
};

// Codes of four values, the first in the lowest byte (nearest, ties to even; none is beyond the largest
// value by more than its rounding).
template <int FMT> __device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
    int v = 0;
    if constexpr (FMT == BSR_E4M3) {
        v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    } else {
        v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
    }
    return unsigned(v);
}
// Codes of a block's values.  ORDINARY: lift is 1 and r is not 0.
template <int FMT, bool ORDINARY>
__device__ __forceinline__ uint2 codes8(float lift, float r, const float (&v)[kVec]) {
    float x[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) x[i] = ORDINARY ? v[i] * r : r == 0.0f ? 0.0f : (v[i] * lift) * r;
    return uint2{codes4<FMT>(x[0], x[1], x[2], x[3]), codes4<FMT>(x[4], x[5], x[6], x[7])};
}

// The first n of N bytes of v at p.
template <int N, class V> __device__ __forceinline__ void store_bytes(uint8_t *p, int64_t n, const V &v) {
    static_assert(sizeof(V) == N, "whole values");
    if (n >= N) {
        stream_out(p, v);
    } else {
        uint8_t b[N];
        __builtin_memcpy(b, &v, N);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = b[i];
    }
}

__device__ __forceinline__ unsigned top_of(const float (&v)[kVec]) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) top = max(top, abs_bits(v[i]));
    return top;
}

// f(constant 0), ..., f(constant N - 1).
template <int... I, class F> __device__ __forceinline__ void each(std::integer_sequence<int, I...>, F &&f) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F> __device__ __forceinline__ void each(F &&f) {
    each(std::make_integer_sequence<int, N>{}, f);
}

// By rows, blocks of 1 x 128: 16 rows of 512 columns to a workgroup, four rows to a wave.  A wave's rows arrive
// partly in turn, bf16 ones wholly, since each is converted where its end is checked: many waves hide that, few
// do not.  The scales of one block lie side by side for the rows, so they are stored 16 at a time.
constexpr int kStripRows = 16, kStripColumns = 64 * kVec;
template <class T, int FMT> __global__ __launch_bounds__(kThreads) void quantize_strip_kernel(QuantizeArgs a) {
    constexpr int kRows = 4, kBlocks = kStripColumns / kF8Block;
    __shared__ float scales[kBlocks][kStripRows];
    const int strips = (a.K + kStripColumns - 1) / kStripColumns;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = a.K;
    const int64_t t0 = a.t0 + int64_t(blockIdx.x / strips) * kStripRows;
    const int c0 = int(blockIdx.x % strips) * kStripColumns, k = c0 + lane * kVec;
    float v[kRows][kVec] = {};
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t t = t0 + wave * kRows + i;
        if (t < a.T) load_vec<T, kAnyEnd>(static_cast<const T *>(a.X) + t * a.ldx, k, K, v[i]);
    }
    unsigned top[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) top[i] = row_max(top_of(v[i]));
    const int own = lane % kRows;              // the row whose scale this lane makes
    const BlockScale<FMT> s(own < 2 ? (own == 0 ? top[0] : top[1]) : (own == 2 ? top[2] : top[3]));
    if (lane % 16 < kRows) scales[lane / 16][wave * kRows + own] = s.scale;
    const auto store = [&](auto ordinary) {
        each<kRows>([&](auto i) {
            const int64_t t = t0 + wave * kRows + i;
            const uint2 codes =
                codes8<FMT, decltype(ordinary)::value>(quad_lane<i>(s.lift), quad_lane<i>(s.r), v[i]);
            if (t < a.T && k < K) store_bytes<8>(a.Q + t * a.ldq + k, K - k, codes);
        });
    };
    if (__all(s.ordinary()))
        store(std::true_type{});
    else
        store(std::false_type{});
    __syncthreads();
    const int b = threadIdx.x / kStripRows, i = threadIdx.x % kStripRows;
    if (b < kBlocks && c0 + b * kF8Block < K && t0 + i < a.T)
        a.scale[(c0 / kF8Block + b) * a.ldscale + t0 + i] = scales[b][i];
}

// Tiles of 128 x 128: a thread holds 8 rows of 8 columns, loaded as the rows above (2304 x 768 in blocks of 128
// x 128, 108 tiles, takes 7.3 us as fp32 and 9.5 as bf16).  ROWS: rows of a block by rows (1 or 128), which is
// the width of one by columns.
template <class T, int FMT, int ROWS>
__global__ __launch_bounds__(kThreads) void quantize_tile_kernel(QuantizeArgs a) {
    constexpr int kB = kF8Block, kWaves = kThreads / 64;
    __shared__ unsigned tops[kWaves][kB];
    __shared__ __align__(16) float column_r[kB], column_lift[kB];
    __shared__ __align__(16) uint8_t turned[kB * kB];
    const int tiles = (a.K + kB - 1) / kB;
    const int64_t t0 = a.t0 + int64_t(blockIdx.x / tiles) * kB;
    const int k0 = int(blockIdx.x % tiles) * kB, K = a.K;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = threadIdx.x % 16, r = threadIdx.x / 16;
    const int k = k0 + c * kVec;
    const int64_t t = t0 + r * kVec;
    float v[kVec][kVec] = {};
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (t + i < a.T) load_vec<T, kAnyEnd>(static_cast<const T *>(a.X) + (t + i) * a.ldx, k, K, v[i]);

    unsigned top[kVec];                        // of the thread's rows, in this tile
#pragma unroll
    for (int i = 0; i < kVec; ++i) top[i] = top_of(v[i]);
    unsigned own = 0;                          // ROWS = 1: of row c % 8; 128: the tile's
    if constexpr (ROWS > 1) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) own = max(own, top[i]);
        own = column_max(row_max(own));
        if (lane == 0) tops[wave][0] = own;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) own = max(own, tops[w][0]);
    } else if (a.Q) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const unsigned whole = row_max(top[i]);
            if (c % kVec == i) own = whole;
        }
    }
    const BlockScale<FMT> s(own);
    if (ROWS > 1 && threadIdx.x == 0) {
        if (a.Q) a.scale[(k0 / kB) * a.ldscale + t0 / kB] = s.scale;
        if (a.QT) a.scale_t[(t0 / kB) * a.ldscale_t + k0 / kB] = s.scale;
    }
    if (a.Q) {
        if (ROWS == 1 && c < kVec && t + c < a.T) a.scale[(k0 / kB) * a.ldscale + t + c] = s.scale;
        const auto store = [&](auto ordinary) {
            each<kVec>([&](auto i) {
                const float lift = ROWS > 1 ? s.lift : row_lane<i>(s.lift);
                const float scale = ROWS > 1 ? s.r : row_lane<i>(s.r);
                const uint2 codes = codes8<FMT, decltype(ordinary)::value>(lift, scale, v[i]);
                if (t + i < a.T && k < K) store_bytes<8>(a.Q + (t + i) * a.ldq + k, K - k, codes);
            });
        };
        if (__all(s.ordinary()))
            store(std::true_type{});
        else
            store(std::false_type{});
    }
    if (!a.QT) return;
    bool ordinary = s.ordinary();
    if constexpr (ROWS == 1) {                 // the scales of the columns, one to a thread
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            unsigned most = 0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) most = max(most, abs_bits(v[i][j]));
            most = column_max(most);
            if (lane < 16) tops[wave][c * kVec + j] = most;
        }
        __syncthreads();
        const int f = threadIdx.x;
        ordinary = true;
        if (f < kB) {
            unsigned most = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) most = max(most, tops[w][f]);
            const BlockScale<FMT> column(most);
            column_r[f] = column.r;
            column_lift[f] = column.lift;
            if (k0 + f < K) a.scale_t[(t0 / kB) * a.ldscale_t + k0 + f] = column.scale;
            ordinary = column.ordinary();
        }
        ordinary = __syncthreads_and(ordinary);
    }
    // Column f of the tile becomes row f of `turned`: rows are swapped in pairs and their 16-byte chunks
    // permuted by f / 8, so that the 8 bytes of a wave's lanes meet every bank twice.
    const auto turn = [&](auto plain) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const int f = c * kVec + j;
            float column[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) column[i] = v[i][j];
            const float lift = ROWS > 1 ? s.lift : column_lift[f], scale = ROWS > 1 ? s.r : column_r[f];
            *reinterpret_cast<uint2 *>(turned + (f ^ (c & 1)) * kB + (((r >> 1) ^ (c >> 1)) << 4) +
                                       (r & 1) * 8) = codes8<FMT, decltype(plain)::value>(lift, scale, column);
        }
    };
    if (ordinary)
        turn(std::true_type{});
    else
        turn(std::false_type{});
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kB * kB / 16 / kThreads; ++e) {
        const int at = e * kThreads + threadIdx.x, f = at / 8, part = at % 8, of = f / kVec;
        const int64_t left = a.T - t0 - part * 16;
        if (k0 + f < K && left > 0)
            store_bytes<16>(a.QT + (k0 + f) * a.ldqt + t0 + part * 16, left,
                            *reinterpret_cast<const uint4 *>(turned + (f ^ (of & 1)) * kB +
                                                             ((part ^ (of >> 1)) << 4)));
    }
}

// Workgroups of a launch: a grid has under 2^32 threads.
constexpr int64_t kGroupsPerLaunch = int64_t(1) << 23;

void launch(void (*kernel)(QuantizeArgs), QuantizeArgs a, int64_t tile_rows, int64_t tile_columns,
            void *stream) {
    const int64_t across = (a.K + tile_columns - 1) / tile_columns;
    const int64_t down = (a.T + tile_rows - 1) / tile_rows, most = kGroupsPerLaunch / across;
    for (int64_t first = 0; first < down; first += most) {
        const int64_t n = down - first < most ? down - first : most;
        a.t0 = first * tile_rows;
        hipLaunchKernelGGL(kernel, dim3(unsigned(n * across)), dim3(kThreads), 0, as_stream(stream), a);
    }
}

template <class T, int FMT> void quantize(const QuantizeArgs &a, int block_rows, void *stream) {
    if (block_rows > 1)
        launch(quantize_tile_kernel<T, FMT, kF8Block>, a, kF8Block, kF8Block, stream);
    else if (a.QT)
        launch(quantize_tile_kernel<T, FMT, 1>, a, kF8Block, kF8Block, stream);
    else
        launch(quantize_strip_kernel<T, FMT>, a, kStripRows, kStripColumns, stream);
}

}  // namespace

bsr_status launch_quantize_f8(const void *X, int x_dtype, int64_t T, int64_t K, int64_t ldx,
                              int block_rows, int format, void *Q, int64_t ldq, float *scale,
                              int64_t ldscale, void *QT, int64_t ldqt, float *scale_t,
                              int64_t ldscale_t, void *stream) {
    const QuantizeArgs a{X, T, ldx, int(K), static_cast<uint8_t *>(Q), static_cast<uint8_t *>(QT),
                         scale, scale_t, ldq, ldscale, ldqt, ldscale_t, 0};
    const auto f = x_dtype == BSR_BF16
                       ? (format == BSR_E4M3 ? quantize<bf16, BSR_E4M3> : quantize<bf16, BSR_E5M2>)
                       : (format == BSR_E4M3 ? quantize<float, BSR_E4M3> : quantize<float, BSR_E5M2>);
    f(a, block_rows, stream);
    return launch_status();
}

}  // namespace bsr
