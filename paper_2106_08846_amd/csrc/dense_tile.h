// The tiled matrix-core product behind the dense entry points:
//   P[m][n] = sum over k of A[m][k] B[n][k],
// rows of A ("tokens") and of B ("channels") contiguous along k.  With DUAL, B is two matrices of
// the same shape and every token meets both (the gate and up projections).
//
// A workgroup makes a BM x BN tile of P; DUAL interleaves MF rows of either matrix in the tile's BN
// rows, so that one lane holds the gate and the up value of the same outputs.  Every step of the
// contraction takes 128 bytes of each row (64 bf16, 128 int8 or 32 fp32) through LDS.  All three
// types use the same layout: a lane's operand of one matrix instruction is 16 consecutive bytes of
// one row (8 bf16 for 32x32x16 / 16x16x32, 16 int8 for 32x32x32 / 16x16x64); for fp32 the four
// values of such a chunk go to four 32x32x2 / 16x16x4 instructions, which is the same sum with its
// terms in another order.
#pragma once

#include "dense_math.h"

namespace bsr {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// One matrix-instruction step over a 16-byte chunk of MF rows each.
template <class E, int MF> struct Mma;
template <> struct Mma<bf16, 32> {
    using Acc = f32x16;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mma<bf16, 16> {
    using Acc = f32x4;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mma<int8_t, 32> {
    using Acc = i32x16;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
    }
};
template <> struct Mma<int8_t, 16> {
    using Acc = i32x4;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    }
};
template <> struct Mma<float, 32> {
    using Acc = f32x16;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};
template <> struct Mma<float, 16> {
    using Acc = f32x4;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};

// What becomes of the product.
enum class Out { kStore, kScale, kGated };

struct ProductArgs {
    const char *A, *B0, *B1;      // B1: DUAL only
    int64_t lda, ldb0, ldb1;      // row pitches in bytes
    int64_t M, N;                 // tokens; channels (of each matrix)
    int Kb;                       // bytes of a row that are summed over
    int tiles_m, tiles_n;
    // epilogue
    const float *sx, *s0, *s1;    // scales of tokens and channels (int8)
    const float *b0, *b1;         // biases or NULL
    void *out, *out2;             // kStore: rows from `split` on go to out2
    float *G, *U;                 // kGated: pre-activations or NULL
    int64_t ldo, ldp, split;
    int out_bf16, act;
};

// 4 consecutive outputs, of which the first `n` exist.
__device__ __forceinline__ void store4(void *base, int64_t at, bool as_bf16, f32x4 v, int n) {
    if (as_bf16) {
        bf16x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = static_cast<__bf16>(v[i]);
        __bf16 *p = static_cast<__bf16 *>(base) + at;
        if (n >= 4) {
            __builtin_memcpy(p, &h, 8);
        } else {
            for (int i = 0; i < n; ++i) p[i] = h[i];
        }
    } else {
        float *p = static_cast<float *>(base) + at;
        if (n >= 4) {
            __builtin_memcpy(p, &v, 16);
        } else {
            for (int i = 0; i < n; ++i) p[i] = v[i];
        }
    }
}

// 4 consecutive values of a per-channel vector, the missing ones `other`.
__device__ __forceinline__ f32x4 load4(const float *p, int64_t at, int n, float other) {
    f32x4 v = {other, other, other, other};
    if (n >= 4) {
        __builtin_memcpy(&v, p + at, 16);
    } else {
        for (int i = 0; i < n; ++i) v[i] = p[at + i];
    }
    return v;
}

__device__ __forceinline__ float activate_by(int act, float g) {
    switch (act) {
        case BSR_ACT_SILU: return activate<BSR_ACT_SILU>(g);
        case BSR_ACT_GELU: return activate<BSR_ACT_GELU>(g);
        case BSR_ACT_GELU_TANH: return activate<BSR_ACT_GELU_TANH>(g);
        default: return activate<BSR_ACT_RELU>(g);
    }
}

// Four outputs of token m from channel n on (`cnt` of them exist): `p`, and for kGated `q`, hold
// the products (int8: as integers).
template <class E, Out OUT>
__device__ __forceinline__ void finish4(const ProductArgs &a, int64_t m, int64_t n, int cnt,
                                        i32x4 p, i32x4 q) {
    f32x4 x, y;
    if constexpr (sizeof(E) == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = float(p[i]);
            y[i] = float(q[i]);
        }
    } else {
        x = __builtin_bit_cast(f32x4, p);
        y = __builtin_bit_cast(f32x4, q);
    }
    if constexpr (OUT == Out::kStore) {
        if (m < a.split)
            store4(a.out, m * a.ldo + n, a.out_bf16, x, cnt);
        else
            store4(a.out2, (m - a.split) * a.ldo + n, a.out_bf16, x, cnt);
        return;
    }
    if constexpr (sizeof(E) == 1) {
        const float s = a.sx[m];
        x = x * s * load4(a.s0, n, cnt, 0.0f);
        if constexpr (OUT == Out::kGated) y = y * s * load4(a.s1, n, cnt, 0.0f);
    }
    if (a.b0) x += load4(a.b0, n, cnt, 0.0f);
    if constexpr (OUT == Out::kScale) {
        store4(a.out, m * a.ldo + n, a.out_bf16, x, cnt);
    } else {
        if (a.b1) y += load4(a.b1, n, cnt, 0.0f);
        f32x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = activate_by(a.act, x[i]) * y[i];
        store4(a.out, m * a.ldo + n, a.out_bf16, h, cnt);
        if (a.G) {
            store4(a.G, m * a.ldp + n, false, x, cnt);
            store4(a.U, m * a.ldp + n, false, y, cnt);
        }
    }
}

constexpr int kStepBytes = 128;   // of every row, per step of the contraction
constexpr int kChunk = 16;
constexpr int kRowChunks = kStepBytes / kChunk;

// LDS position of chunk c of a row: the chunks of a row are permuted by its number, so that a
// wave's 16-byte reads of one chunk column spread over the banks.
__device__ __forceinline__ int swizzled(int row, int c) { return c ^ ((row >> 1) & 7); }

// BM x BN tile, WM x WN waves, MF x MF matrix instructions.  ALIGNED: rows start on 16-byte
// boundaries and Kb is a multiple of 16, so 16-byte chunks are loaded whole through range-checked
// buffer loads; otherwise byte-aligned loads, with the last chunk of a row put together from what
// it has.
template <class E, int BM, int BN, int WM, int WN, int MF, bool DUAL, bool ALIGNED, Out OUT>
struct TileKernel {
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int TM = BM / WM, TN = BN / WN;     // a wave's tokens and channels
    static constexpr int NM = TM / MF, NN = TN / MF;
    static constexpr int kRowsPerPass = kThreads / kRowChunks;
    static constexpr int LA = BM / kRowsPerPass, LB = BN / kRowsPerPass;   // chunks per thread
    static constexpr int kStageBytes = (BM + BN) * kStepBytes;
    static constexpr int kPitch = TN + 4;                // epilogue: floats per token in LDS
    static constexpr int kEpiBytes = MF * kPitch * 4;    // per wave
    static constexpr int kLds = 2 * kStageBytes > WM * WN * kEpiBytes ? 2 * kStageBytes
                                                                     : WM * WN * kEpiBytes;
    static constexpr int kSteps = MF == 32 ? 4 : 2;      // matrix-instruction steps per stage
    static constexpr int kLaneChunks = 64 / MF;          // chunks of a row in one step
    static constexpr int kTileN = DUAL ? BN / 2 : BN;    // channels per tile
    using M_ = Mma<E, MF>;
    using Acc = typename M_::Acc;
    static_assert(BM % kRowsPerPass == 0 && BN % kRowsPerPass == 0, "whole passes");
    static_assert(!DUAL || NN % 2 == 0, "gate and up blocks in pairs");
    static_assert(kLds <= 160 * 1024, "LDS of a CU");

    struct Source {   // one operand's rows as this workgroup reads them
        const char *base;     // first row of the tile
        int64_t pitch;
        int rows;             // rows that exist (0: none; never read)
    };

    // The chunk at byte kb of row `row`; rows that do not exist may hold anything, bytes from Kb on
    // are zero.
    static __device__ __forceinline__ i32x4 load_chunk(const Source &s, int row, int kb, int Kb) {
        if constexpr (ALIGNED) {
            // Every existing row ends at or before byte (rows - 1) * pitch + Kb; a chunk past Kb or
            // a row past the end is sent out of range, which loads zeros.
            const unsigned bytes = s.rows > 0 ? unsigned((s.rows - 1) * s.pitch) + unsigned(Kb) : 0u;
            const unsigned off = kb < Kb ? unsigned(row) * unsigned(s.pitch) + unsigned(kb)
                                         : 0x80000000u;
            return __builtin_bit_cast(
                i32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer_rsrc(s.base, bytes), off, 0, 0));
        } else {
            i32x4 v = {0, 0, 0, 0};
            if (row >= s.rows || kb >= Kb) return v;
            const char *p = s.base + row * s.pitch + kb;
            if (Kb - kb >= kChunk) {
                __builtin_memcpy(&v, p, kChunk);
            } else {
                const E *e = reinterpret_cast<const E *>(p);
                const int n = (Kb - kb) / int(sizeof(E));
                E tail[kChunk / sizeof(E)] = {};
#pragma unroll
                for (int i = 0; i < int(kChunk / sizeof(E)); ++i)
                    if (i < n) tail[i] = e[i];
                __builtin_memcpy(&v, tail, kChunk);
            }
            return v;
        }
    }

    static __device__ __forceinline__ void run(const ProductArgs &a, char *lds) {
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
        const int wm = wave % WM, wn = wave / WM;
        int tm, tn;
        tile_of(a, tm, tn);
        const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * kTileN;
        const int64_t left_m = a.M - m0, left_n = a.N - n0;
        const Source sa{a.A + m0 * a.lda, a.lda, int(left_m < BM ? left_m : BM)};
        const int rows_n = int(left_n < kTileN ? left_n : kTileN);
        const Source sb0{a.B0 + n0 * a.ldb0, a.ldb0, rows_n};
        const Source sb1{DUAL ? a.B1 + n0 * a.ldb1 : nullptr, a.ldb1, rows_n};

        const int c = tid & (kRowChunks - 1), r0 = tid / kRowChunks;
        const int wave_row = wave * (64 / kRowChunks);      // first row of this wave in a pass
        i32x4 ra[LA], rb[LB];
        auto load = [&](int step) {
            const int kb = step * kStepBytes + c * kChunk;
#pragma unroll
            for (int i = 0; i < LA; ++i) ra[i] = load_chunk(sa, i * kRowsPerPass + r0, kb, a.Kb);
#pragma unroll
            for (int i = 0; i < LB; ++i) {
                const int row = i * kRowsPerPass + r0;
                if constexpr (DUAL) {
                    // row = (pair * 2 + which) * MF + r stands for channel pair * MF + r
                    const int first = i * kRowsPerPass + wave_row;      // uniform; MF % 8 == 0
                    const int channel = row / (2 * MF) * MF + row % MF;
                    const Source &s = (first / MF) & 1 ? sb1 : sb0;
                    rb[i] = load_chunk(s, channel, kb, a.Kb);
                } else {
                    rb[i] = load_chunk(sb0, row, kb, a.Kb);
                }
            }
        };
        auto put = [&](int buf) {
            char *p = lds + buf * kStageBytes;
#pragma unroll
            for (int i = 0; i < LA; ++i) {
                const int row = i * kRowsPerPass + r0;
                *reinterpret_cast<i32x4 *>(p + row * kStepBytes + swizzled(row, c) * kChunk) = ra[i];
            }
            p += BM * kStepBytes;
#pragma unroll
            for (int i = 0; i < LB; ++i) {
                const int row = i * kRowsPerPass + r0;
                *reinterpret_cast<i32x4 *>(p + row * kStepBytes + swizzled(row, c) * kChunk) = rb[i];
            }
        };

        Acc acc[NN][NM] = {};
        const int fr = lane % MF, fc = lane / MF;
        const int steps = (a.Kb + kStepBytes - 1) / kStepBytes;
        load(0);
        put(0);
        for (int s = 0; s < steps; ++s) {
            __syncthreads();
            if (s + 1 < steps) load(s + 1);
            const char *pa = lds + (s & 1) * kStageBytes + (wm * TM + fr) * kStepBytes;
            const char *pb = lds + (s & 1) * kStageBytes + (BM + wn * TN + fr) * kStepBytes;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int at = swizzled(fr, k * kLaneChunks + fc) * kChunk;
                i32x4 fa[NM], fb[NN];
#pragma unroll
                for (int i = 0; i < NM; ++i)
                    fa[i] = *reinterpret_cast<const i32x4 *>(pa + i * MF * kStepBytes + at);
#pragma unroll
                for (int j = 0; j < NN; ++j)
                    fb[j] = *reinterpret_cast<const i32x4 *>(pb + j * MF * kStepBytes + at);
#pragma unroll
                for (int j = 0; j < NN; ++j)
#pragma unroll
                    for (int i = 0; i < NM; ++i) acc[j][i] = M_::step(fb[j], fa[i], acc[j][i]);
            }
            if (s + 1 < steps) put((s + 1) & 1);
        }
        __syncthreads();

        // Epilogue: MF tokens of the wave's tile at a time go through LDS, so that consecutive
        // lanes finish consecutive channels of a token.
        float *mine = reinterpret_cast<float *>(lds + wave * kEpiBytes);
        constexpr int kQuads = (DUAL ? TN / 2 : TN) / 4;
#pragma unroll
        for (int i = 0; i < NM; ++i) {
#pragma unroll
            for (int j = 0; j < NN; ++j) {
                // lane: token fr; register group g: channels 4 fc + g (* 8 for 32x32) .. + 3
#pragma unroll
                for (int g = 0; g < MF * MF / 256; ++g) {
                    i32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const auto x = acc[j][i][4 * g + e];
                        v[e] = __builtin_bit_cast(int, x);
                    }
                    *reinterpret_cast<i32x4 *>(mine + fr * kPitch + j * MF + 8 * g + 4 * fc) = v;
                }
            }
            wave_sync();
            const int64_t mt = m0 + wm * TM + i * MF;
#pragma unroll 1
            for (int e = lane; e < MF * kQuads; e += 64) {
                const int t = e / kQuads, quad = e % kQuads;
                const int64_t m = mt + t;
                int64_t n;
                const float *p = mine + t * kPitch;
                i32x4 x, y = {0, 0, 0, 0};
                if constexpr (DUAL) {
                    const int pair = quad / (MF / 4), r = quad % (MF / 4) * 4;
                    n = n0 + wn * (TN / 2) + pair * MF + r;
                    x = *reinterpret_cast<const i32x4 *>(p + pair * 2 * MF + r);
                    y = *reinterpret_cast<const i32x4 *>(p + pair * 2 * MF + MF + r);
                } else {
                    n = n0 + wn * TN + quad * 4;
                    x = *reinterpret_cast<const i32x4 *>(p + quad * 4);
                }
                if (m < a.M && n < a.N)
                    finish4<E, OUT>(a, m, n, int(a.N - n < 4 ? a.N - n : 4), x, y);
            }
            wave_sync();
        }
    }

    // Order LDS accesses of one wave's lanes among themselves.
    static __device__ __forceinline__ void wave_sync() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }

    // Workgroups go round robin over the 8 XCDs: XCD x takes a contiguous run of the tile order,
    // and that order walks bands of 8 token tiles, so the tiles an XCD works on at one time share
    // rows of both operands in its L2.
    static __device__ __forceinline__ void tile_of(const ProductArgs &a, int &tm, int &tn) {
        const int total = a.tiles_m * a.tiles_n, id = blockIdx.x;
        const int per = total / 8, extra = total % 8, x = id % 8;
        const int t = x * per + (x < extra ? x : extra) + id / 8;
        constexpr int kBand = 8;
        const int band = t / (kBand * a.tiles_n), first = band * kBand;
        const int height = a.tiles_m - first < kBand ? a.tiles_m - first : kBand;
        const int in = t - first * a.tiles_n;
        tm = first + in % height;
        tn = in / height;
    }
};

template <class E, int BM, int BN, int WM, int WN, int MF, bool DUAL, bool ALIGNED, Out OUT>
__global__ __launch_bounds__(64 * WM * WN) void dense_tile_kernel(ProductArgs a) {
    using K = TileKernel<E, BM, BN, WM, WN, MF, DUAL, ALIGNED, OUT>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
