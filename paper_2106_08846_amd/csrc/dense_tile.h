// The tiled matrix-core products behind the dense entry points:
//   P[m][n] = sum over k of A[m][k] B[n][k],
// rows of A ("tokens") and of B ("channels") contiguous along k.  With DUAL, B is two matrices of
// the same shape and every token meets both (the gate and up projections).
//
// A workgroup makes a BM x BN tile of P; DUAL interleaves 16 rows of either matrix in the tile's BN
// rows, so that one lane holds the gate and the up value of the same outputs.  A lane's operand of
// one matrix instruction is 16 consecutive bytes of one row: 8 bf16 for 16x16x32 or 16 int8 for
// 16x16x64.  (32x32 instructions move the same bytes per product and ran the 8192^3 product 5%
// slower.)  fp32 operands are split into three bf16 pieces on their way into LDS, see Pieces.
//
// Here: what the tile kernels share, and the kernel that takes its operands through registers into
// LDS: for rows that start on no 16-byte boundary, and for fp32.  Rows on 16-byte boundaries go
// straight into LDS in dense_ring.h.
#pragma once

#include <type_traits>

#include "dense_math.h"

namespace bsr {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// One matrix-instruction step over a 16-byte chunk of 16 rows each.  fp32: the four values of a
// chunk go to four 16x16x4 instructions, which is the same sum with its terms in another order.
template <class E> struct Mma;
template <> struct Mma<bf16> {
    using Acc = f32x4;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mma<int8_t> {
    using Acc = i32x4;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    }
};
template <> struct Mma<float> {
    using Acc = f32x4;
    static __device__ __forceinline__ Acc step(i32x4 a, i32x4 b, Acc c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};

// fp32 values as sums of three bf16 pieces, x = h + m + l: h is x rounded to bf16, m the remainder
// rounded, l what is left, which has 8 significant bits (|m| <= 2^-9 |x|, |l| <= 2^-18 |x|; exact
// while l does not underflow, |x| >= 2^-100).  A product x y is formed from the six cross terms down
// to 2^-18 |x y| (hh, hm, mh, hl, lh, mm), each exact in fp32; the three left out are together below
// 2^-25.9 |x y|, a quarter of fp32's own rounding.  Six bf16 instructions take 96 cycles for what
// the fp32 instructions need 256 for.  An infinite operand (or one that rounds to infinity in bf16,
// from 2^128 (1 - 2^-9) on) gives NaN.
struct Pieces {
    bf16x4 h, m, l;
};
__device__ __forceinline__ Pieces split(f32x4 x) {
    Pieces p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p.h[i] = static_cast<__bf16>(x[i]);
        const float r = x[i] - static_cast<float>(p.h[i]);
        p.m[i] = static_cast<__bf16>(r);
        p.l[i] = static_cast<__bf16>(r - static_cast<float>(p.m[i]));
    }
    return p;
}

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

constexpr int kMF = 16;           // rows and columns of a matrix instruction
constexpr int kChunk = 16;        // bytes of a row per lane and instruction

struct Source {   // one operand's rows as a workgroup reads them
    const char *base;     // first row of the tile
    int64_t pitch;
    int rows;             // rows that exist, at least 1
};

// The 16 bytes at byte kb of row `row`, those from Kb on and those of a row that does not exist
// being zero.  ALIGNED: rows start on 16-byte boundaries and Kb is a multiple of 16, so chunks are
// loaded whole through a range-checked buffer load; otherwise byte-aligned loads, with the last
// chunk of a row put together from what it has.
template <class E, bool ALIGNED>
__device__ __forceinline__ i32x4 load_chunk(const Source &s, int row, int kb, int Kb) {
    if constexpr (ALIGNED) {
        // Every existing row ends at or before byte (rows - 1) * pitch + Kb; a row past the end is
        // out of that range by itself, a chunk past Kb is sent there.
        const unsigned bytes = unsigned((s.rows - 1) * s.pitch) + unsigned(Kb);
        const unsigned off = kb < Kb ? unsigned(row) * unsigned(s.pitch) + unsigned(kb) : 0x80000000u;
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

// The tile of this workgroup.  Workgroups go round robin over the 8 XCDs: XCD x takes a contiguous
// run of the tile order, and that order walks bands of 8 token tiles, so the tiles an XCD works on
// at one time share rows of both operands in its L2.
__device__ __forceinline__ void tile_of(const ProductArgs &a, int &tm, int &tn) {
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

// Order LDS accesses of one wave's lanes among themselves.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A wave's NN x NM accumulators (channels x tokens, 16 x 16 each) to the outputs, 16 tokens at a time
// through the wave's own LDS, so that consecutive lanes finish consecutive channels of a token.
// m0, n0: the wave's first token and channel.
constexpr int epilogue_bytes(int NN) { return kMF * (NN * kMF + 4) * 4; }
template <class E, Out OUT, int NN, int NM, class Acc>
__device__ __forceinline__ void epilogue(const ProductArgs &a, const Acc (&acc)[NN][NM], float *mine,
                                         int64_t m0, int64_t n0) {
    constexpr bool kDual = OUT == Out::kGated;
    constexpr int kPitch = NN * kMF + 4;
    constexpr int kQuads = NN * kMF / (kDual ? 8 : 4);
    const int lane = threadIdx.x & 63, fr = lane % kMF, fc = lane / kMF;
#pragma unroll
    for (int i = 0; i < NM; ++i) {
#pragma unroll
        for (int j = 0; j < NN; ++j) {      // lane: token fr, channels 4 fc .. + 3
            i32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const auto x = acc[j][i][e];
                v[e] = __builtin_bit_cast(int, x);
            }
            *reinterpret_cast<i32x4 *>(mine + fr * kPitch + j * kMF + 4 * fc) = v;
        }
        wave_sync();
#pragma unroll 1
        for (int e = lane; e < kMF * kQuads; e += 64) {
            const int t = e / kQuads, quad = e % kQuads;
            const int64_t m = m0 + i * kMF + t, n = n0 + quad * 4;
            const float *p = mine + t * kPitch;
            i32x4 x, y = {0, 0, 0, 0};
            if constexpr (kDual) {
                const int pair = quad / (kMF / 4), r = quad % (kMF / 4) * 4;
                x = *reinterpret_cast<const i32x4 *>(p + pair * 2 * kMF + r);
                y = *reinterpret_cast<const i32x4 *>(p + pair * 2 * kMF + kMF + r);
            } else {
                x = *reinterpret_cast<const i32x4 *>(p + quad * 4);
            }
            if (m < a.M && n < a.N)
                finish4<E, OUT>(a, m, n, int(a.N - n < 4 ? a.N - n : 4), x, y);
        }
        wave_sync();
    }
}

// BM x BN tile, WM x WN waves, operands through registers.  A step of the contraction takes 128
// bytes of every row (64 bf16, 128 int8, 32 fp32): its chunks are loaded one step before they are
// written into LDS and two before they are used, and written between the halves of a step's matrix
// instructions (10% faster at 8192^3 than loading and writing the next step around all of them).
template <class E, int BM, int BN, int WM, int WN, bool ALIGNED, Out OUT> struct TileKernel {
    static constexpr bool kDual = OUT == Out::kGated;
    static constexpr bool kSplit = sizeof(E) == 4;       // fp32 in three pieces
    static constexpr int kPlanes = kSplit ? 3 : 1;
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int TM = BM / WM, TN = BN / WN;     // a wave's tokens and channels
    static constexpr int NM = TM / kMF, NN = TN / kMF;
    static constexpr int kStepBytes = 128;
    static constexpr int kRowChunks = kStepBytes / kChunk;
    static constexpr int kRowBytes = kSplit ? 64 : 128;  // of a row (and piece) in LDS
    static constexpr int kSteps = kRowBytes / 64;        // matrix-instruction steps
    static constexpr int kRowsPerPass = kThreads / kRowChunks;
    static constexpr int LA = BM / kRowsPerPass, LB = BN / kRowsPerPass;   // chunks per thread
    static constexpr int kPlaneBytes = (BM + BN) * kRowBytes;
    static constexpr int kStageBytes = kPlanes * kPlaneBytes;
    static constexpr int kEpiBytes = WM * WN * epilogue_bytes(NN);
    static constexpr int kLds = 2 * kStageBytes > kEpiBytes ? 2 * kStageBytes : kEpiBytes;
    static constexpr int kTileN = kDual ? BN / 2 : BN;   // channels per tile
    using M_ = Mma<typename std::conditional<kSplit, bf16, E>::type>;
    using Acc = typename M_::Acc;
    static_assert(BM % kRowsPerPass == 0 && BN % kRowsPerPass == 0, "whole passes");
    static_assert(!kDual || NN % 2 == 0, "gate and up blocks in pairs");
    static_assert(kLds <= 160 * 1024, "LDS of a CU");

    // LDS position of 16-byte chunk c of a row: the chunks of a row are permuted by its number, so
    // that a wave's reads of 16 rows spread over all banks (no conflicts counted).
    static __device__ __forceinline__ int swizzled(int row, int c) {
        return kRowBytes == 128 ? c ^ ((row >> 1) & 7) : c ^ ((row >> 2) & 3);
    }
    // Chunk c (of the source row) of row `row` into the stage at p.
    static __device__ __forceinline__ void put_chunk(char *p, int row, int c, i32x4 v) {
        if constexpr (kSplit) {
            const Pieces s = split(__builtin_bit_cast(f32x4, v));
            char *q = p + row * kRowBytes + swizzled(row, c >> 1) * kChunk + (c & 1) * 8;
            *reinterpret_cast<bf16x4 *>(q) = s.h;
            *reinterpret_cast<bf16x4 *>(q + kPlaneBytes) = s.m;
            *reinterpret_cast<bf16x4 *>(q + 2 * kPlaneBytes) = s.l;
        } else {
            *reinterpret_cast<i32x4 *>(p + row * kRowBytes + swizzled(row, c) * kChunk) = v;
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
        const Source sb1{kDual ? a.B1 + n0 * a.ldb1 : nullptr, a.ldb1, rows_n};

        const int c = tid & (kRowChunks - 1), r0 = tid / kRowChunks;
        const int wave_row = wave * (64 / kRowChunks);      // first row of this wave in a pass
        i32x4 ra[LA], rb[LB];
        auto load = [&](int step) {
            const int kb = step * kStepBytes + c * kChunk;
#pragma unroll
            for (int i = 0; i < LA; ++i)
                ra[i] = load_chunk<E, ALIGNED>(sa, i * kRowsPerPass + r0, kb, a.Kb);
#pragma unroll
            for (int i = 0; i < LB; ++i) {
                const int row = i * kRowsPerPass + r0;
                if constexpr (kDual) {
                    // row = (pair * 2 + which) * 16 + r stands for channel pair * 16 + r
                    const int first = i * kRowsPerPass + wave_row;      // uniform
                    const int channel = row / (2 * kMF) * kMF + row % kMF;
                    const Source &s = (first / kMF) & 1 ? sb1 : sb0;
                    rb[i] = load_chunk<E, ALIGNED>(s, channel, kb, a.Kb);
                } else {
                    rb[i] = load_chunk<E, ALIGNED>(sb0, row, kb, a.Kb);
                }
            }
        };
        auto put = [&](int buf) {
            char *p = lds + buf * kStageBytes;
#pragma unroll
            for (int i = 0; i < LA; ++i) put_chunk(p, i * kRowsPerPass + r0, c, ra[i]);
#pragma unroll
            for (int i = 0; i < LB; ++i) put_chunk(p + BM * kRowBytes, i * kRowsPerPass + r0, c, rb[i]);
        };

        Acc acc[NN][NM] = {};
        const int fr = lane % kMF, fc = lane / kMF;
        const int steps = (a.Kb + kStepBytes - 1) / kStepBytes;
        load(0);
        put(0);
        if (steps > 1) load(1);
        for (int s = 0; s < steps; ++s) {
            __syncthreads();
            const char *pa = lds + (s & 1) * kStageBytes + (wm * TM + fr) * kRowBytes;
            const char *pb = lds + (s & 1) * kStageBytes + (BM + wn * TN + fr) * kRowBytes;
            i32x4 fa[kPlanes][NM], fb[kPlanes][NN];
            auto fetch = [&](int k) {
                const int at = swizzled(fr, k * 4 + fc) * kChunk;
#pragma unroll
                for (int p = 0; p < kPlanes; ++p) {
#pragma unroll
                    for (int i = 0; i < NM; ++i)
                        fa[p][i] = *reinterpret_cast<const i32x4 *>(pa + p * kPlaneBytes +
                                                                   i * kMF * kRowBytes + at);
#pragma unroll
                    for (int j = 0; j < NN; ++j)
                        fb[p][j] = *reinterpret_cast<const i32x4 *>(pb + p * kPlaneBytes +
                                                                   j * kMF * kRowBytes + at);
                }
            };
            // Piece x of B with piece y of A.
            auto multiply = [&](int x, int y) {
#pragma unroll
                for (int j = 0; j < NN; ++j)
#pragma unroll
                    for (int i = 0; i < NM; ++i) acc[j][i] = M_::step(fb[x][j], fa[y][i], acc[j][i]);
            };
            auto next = [&] {
                if (s + 1 < steps) put((s + 1) & 1);
                if (s + 2 < steps) load(s + 2);
            };
            fetch(0);
            if constexpr (kSplit) {
                multiply(0, 2);
                multiply(2, 0);
                next();
                multiply(1, 1);
                multiply(0, 1);
                multiply(1, 0);
                multiply(0, 0);
            } else {
                multiply(0, 0);
                next();
                fetch(1);
                multiply(0, 0);
            }
        }
        __syncthreads();
        epilogue<E, OUT, NN, NM>(a, acc, reinterpret_cast<float *>(lds + wave * epilogue_bytes(NN)),
                                 m0 + wm * TM, n0 + wn * (kDual ? TN / 2 : TN));
    }
};

template <class E, int BM, int BN, int WM, int WN, bool ALIGNED, Out OUT>
__global__ __launch_bounds__(64 * WM * WN) void dense_tile_kernel(ProductArgs a) {
    using K = TileKernel<E, BM, BN, WM, WN, ALIGNED, OUT>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
