// The tiled matrix-core products behind the dense entry points:
//   P[m][n] = sum over k of A[m][k] B[n][k],
// rows of A ("tokens") and of B ("channels") contiguous along k.  With DUAL, B is two matrices of
// the same shape and every token meets both (the gate and up projections).
//
// A workgroup makes a BM x BN tile of P; DUAL interleaves 16 rows of either matrix in the tile's BN
// rows, so that one lane holds the gate and the up value of the same outputs.  A lane's operand of
// one matrix instruction is 16 consecutive bytes of one row: 8 bf16 for 16x16x32 or 16 int8 for
// 16x16x64.  (32x32 instructions move the same bytes per product and ran the 8192^3 product 5%
// slower.)
//
// Here: what the tile kernels share, and the one for bf16 and int8 rows that start on no 16-byte
// boundary.  Rows on 16-byte boundaries go straight into LDS in dense_ring.h; fp32 is in
// dense_split.h.
#pragma once

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

// What becomes of the product.
enum class Out { kStore, kScale, kGated };

struct ProductArgs {
    const char *A, *B0, *B1;      // B1: DUAL, column operands
    int64_t lda, ldb0, ldb1;      // row pitches in bytes
    int64_t M, N;                 // tokens; channels (of each matrix)
    int Kb;                       // bytes of a row that are summed over
    int rows_k, half;             // column operands: rows of each matrix, and the step from which on
                                  // the second one (B1) is taken
    int tiles_m, tiles_n;
    int slice;                    // kStore: steps of the contraction per workgroup, blockIdx.y counting
                                  // slices whose sums go to out + blockIdx.y * M * N; 0: all of them
    // epilogue
    const float *sx, *s0, *s1;    // scales of tokens and channels (int8)
    const float *b0, *b1;         // biases or NULL
    void *out, *out2;             // kStore: rows from `split` on go to out2; `limit` of each exist
    float *G, *U;                 // kGated: pre-activations or NULL
    int64_t ldo, ldp, split, limit;
    int out_bf16, act;
    const char *A1;               // column operands: A's second matrix, of A's pitch (last: beside A it
                                  // made a training step of 100 x 1000 x 4000 1 us longer, of 49)
};

// 4 consecutive outputs, of which the first `n` exist.  PAST: stored past the caches, so that the
// operands which other workgroups still read keep their place.
template <bool PAST>
__device__ __forceinline__ void store4(void *base, int64_t at, bool as_bf16, f32x4 v, int n) {
    if (as_bf16) {
        bf16x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = static_cast<__bf16>(v[i]);
        __bf16 *p = static_cast<__bf16 *>(base) + at;
        if (PAST && n >= 4) {
            typedef unsigned Words __attribute__((ext_vector_type(2), aligned(2)));
            Words w;
            __builtin_memcpy(&w, &h, 8);
            __builtin_nontemporal_store(w, reinterpret_cast<Words *>(p));
        } else if (n >= 4) {
            __builtin_memcpy(p, &h, 8);
        } else {
            for (int i = 0; i < n; ++i) p[i] = h[i];
        }
    } else {
        float *p = static_cast<float *>(base) + at;
        if (PAST && n >= 4) {
            typedef float Floats __attribute__((ext_vector_type(4), aligned(4)));
            __builtin_nontemporal_store(Floats(v), reinterpret_cast<Floats *>(p));
        } else if (n >= 4) {
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

// What four channels from n on (`cnt` of which exist) bring to every token's outputs.
template <class E, Out OUT> struct ChannelQuad {
    f32x4 s0, s1, b0, b1;
    __device__ __forceinline__ ChannelQuad(const ProductArgs &a, int64_t n, int cnt) {
        if constexpr (OUT != Out::kStore) {
            if constexpr (sizeof(E) == 1) {
                s0 = load4(a.s0, n, cnt, 0.0f);
                if constexpr (OUT == Out::kGated) s1 = load4(a.s1, n, cnt, 0.0f);
            }
            b0 = b1 = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (a.b0) b0 = load4(a.b0, n, cnt, 0.0f);
            if (OUT == Out::kGated && a.b1) b1 = load4(a.b1, n, cnt, 0.0f);
        }
    }
};

// Four outputs of token m from channel n on (`cnt` of them exist): `p`, and for kGated `q`, hold
// the products (int8: as integers).  Every operation rounds, as the 8-bit product is defined: nothing is
// fused, so that the results do not depend on the kernel.
template <class E, Out OUT, bool PAST>
__device__ __forceinline__ void finish4(const ProductArgs &a, const ChannelQuad<E, OUT> &of, int64_t m,
                                        int64_t n, int cnt, i32x4 p, i32x4 q) {
#pragma clang fp contract(off)
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
        if (a.slice > 0) {
            store4<false>(a.out, (blockIdx.y * a.M + m) * a.N + n, false, x, cnt);
            return;
        }
        const int64_t row = m < a.split ? m : m - a.split;
        if (row < a.limit)
            store4<PAST>(m < a.split ? a.out : a.out2, row * a.ldo + n, a.out_bf16, x, cnt);
        return;
    }
    if constexpr (sizeof(E) == 1) {
        const float s = a.sx[m];
        x = x * s * of.s0;
        if constexpr (OUT == Out::kGated) y = y * s * of.s1;
    }
    if (a.b0) x += of.b0;
    if constexpr (OUT == Out::kScale) {
        store4<PAST>(a.out, m * a.ldo + n, a.out_bf16, x, cnt);
    } else {
        if (a.b1) y += of.b1;
        f32x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = activate_by(a.act, x[i]) * y[i];
        store4<PAST>(a.out, m * a.ldo + n, a.out_bf16, h, cnt);
        if (a.G) {
            store4<PAST>(a.G, m * a.ldp + n, false, x, cnt);
            store4<PAST>(a.U, m * a.ldp + n, false, y, cnt);
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

// One lane's view of a row: the 16-byte chunk at byte `col` of it, and those at `col` plus whole steps.
// Rows past the end stand for the last one: what they give reaches only outputs that do not exist.
//
// kAligned: rows start on 16-byte boundaries and Kb is a multiple of 16, so chunks are loaded whole
//   through a range-checked buffer load.
// Otherwise the last chunk of a row is put together from what it has, and the others are
// kBytes: loaded with one byte-aligned 16-byte load, or
// kShifted: shifted out of the five aligned dwords that hold them (none of which lies outside the
//   row), which spares the memory pipe taking the load apart but loads and computes more: one token
//   through 12288 x 8191 int8 takes 38 us this way and 69 with byte-aligned loads, 4096 tokens through
//   4096 x 4095 in tiles 152 us and 107.
enum class Load { kAligned, kBytes, kShifted };
template <class E, Load LOAD> struct RowChunks {
    const char *base;     // uniform
    unsigned bytes, off;
    unsigned shift;       // kShifted: bytes from the dword at `off` to the chunk

    __device__ __forceinline__ void set(const Source &s, int row, int col, int Kb) {
        base = s.base;
        bytes = unsigned((s.rows - 1) * s.pitch) + unsigned(Kb);
        off = unsigned(row < s.rows ? row : s.rows - 1) * unsigned(s.pitch) + unsigned(col);
        shift = 0;
        if constexpr (LOAD == Load::kShifted) {
            const unsigned low = unsigned(reinterpret_cast<uintptr_t>(base)) & 3u;
            base -= low;
            shift = (off + low) & 3u;
            off = (off + low) & ~3u;
        }
    }
    // The chunk `kb` bytes further on, `left` = Kb - col - kb bytes of which are left in the row; zeros
    // past its end.  kb is a multiple of 4.
    __device__ __forceinline__ i32x4 load(int kb, int left) const {
        if constexpr (LOAD == Load::kAligned) {
            const unsigned at = left > 0 ? off + unsigned(kb) : 0x80000000u;    // out of range: zeros
            return __builtin_bit_cast(
                i32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer_rsrc(base, bytes), at, 0, 0));
        } else {
            i32x4 v = {0, 0, 0, 0};
            const char *p = base + (off + unsigned(kb));
            if (left >= kChunk && LOAD == Load::kBytes) {
                __builtin_memcpy(&v, p, kChunk);
            } else if (left >= kChunk) {
                typedef int i32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));
                const i32x4 w = *reinterpret_cast<const i32x4_by4 *>(p);
                const int next = *reinterpret_cast<const int *>(p + (shift ? 16 : 12));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] = int(__builtin_amdgcn_alignbyte(unsigned(i < 3 ? w[i + 1] : next),
                                                          unsigned(w[i]), shift));
            } else if (left > 0) {
                const E *e = reinterpret_cast<const E *>(p + shift);
                const int n = left / int(sizeof(E));
                E tail[kChunk / sizeof(E)] = {};
#pragma unroll
                for (int i = 0; i < int(kChunk / sizeof(E)); ++i)
                    if (i < n) tail[i] = e[i];
                __builtin_memcpy(&v, tail, kChunk);
            }
            return v;
        }
    }
};

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

// The steps of the contraction that this workgroup sums: `steps` from `first` on, of `total`.
struct Slice {
    int first, steps;
    __device__ __forceinline__ Slice(const ProductArgs &a, int total) {
        first = a.slice > 0 ? int(blockIdx.y) * a.slice : 0;
        steps = a.slice > 0 && total - first > a.slice ? a.slice : total - first;
    }
};

// The rows of both operands that a workgroup's tile takes: BM tokens, kTileN channels of each of B's
// matrices.
template <int BM, int kTileN, bool DUAL> struct TileRows {
    int64_t m0, n0;
    Source a, b0, b1;

    __device__ __forceinline__ explicit TileRows(const ProductArgs &p) {
        int tm, tn;
        tile_of(p, tm, tn);
        m0 = int64_t(tm) * BM;
        n0 = int64_t(tn) * kTileN;
        const int64_t left_m = p.M - m0, left_n = p.N - n0;
        const int rows_n = int(left_n < kTileN ? left_n : kTileN);
        a = Source{p.A + m0 * p.lda, p.lda, int(left_m < BM ? left_m : BM)};
        b0 = Source{p.B0 + n0 * p.ldb0, p.ldb0, rows_n};
        b1 = DUAL ? Source{p.B1 + n0 * p.ldb1, p.ldb1, rows_n} : b0;
    }
    // Row `row` of the tile's B is row `channel(row)` of this source; `first` is the first row that
    // the wave's lanes ask for (uniform; at most 16 rows, from a multiple of their number on).  DUAL:
    // row (pair * 2 + which) * 16 + r stands for channel pair * 16 + r.
    __device__ __forceinline__ const Source &b(int first) const {
        return DUAL && ((first / kMF) & 1) ? b1 : b0;
    }
    static __device__ __forceinline__ int channel(int row) {
        return DUAL ? row / (2 * kMF) * kMF + row % kMF : row;
    }
};

// LDS layout of rows of 64 bytes: two rows to a line of 128, whose 16-byte chunks are permuted by the
// line's number.  A wave's read of 16 rows then meets every bank once in each of the groups of 16
// lanes that a 16-byte read is served in (lanes 0-3, 12-15, 20-23, 24-27 and so on); permuting each
// row's four chunks by row / 4 instead gave two-way conflicts, measured as twice the LDS cycles.
__device__ __forceinline__ int half_row_at(int row, int c) {
    const int line = row >> 1;
    return line * 128 + ((((row & 1) << 2) | c) ^ (line & 7)) * kChunk;
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
template <class E, Out OUT, int NN, int NM, bool PAST = false, class Acc>
__device__ __forceinline__ void epilogue(const ProductArgs &a, const Acc (&acc)[NN][NM], float *mine,
                                         int64_t m0, int64_t n0) {
    constexpr bool kDual = OUT == Out::kGated;
    constexpr int kPitch = NN * kMF + 4;
    constexpr int kQuads = NN * kMF / (kDual ? 8 : 4);      // of a token; a lane keeps its own
    static_assert(64 % kQuads == 0, "whole tokens per pass");
    const int lane = threadIdx.x & 63, fr = lane % kMF, fc = lane / kMF;
    const int quad = lane % kQuads;
    const int64_t n = n0 + quad * 4;
    const int cnt = a.N - n < 4 ? int(a.N - n) : 4;
    const ChannelQuad<E, OUT> of(a, n, cnt);                // nothing where cnt <= 0
    const int pair = quad / (kMF / 4), r = quad % (kMF / 4) * 4;
    const int at = kDual ? pair * 2 * kMF + r : quad * 4;
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
        for (int t = lane / kQuads; t < kMF; t += 64 / kQuads) {
            const int64_t m = m0 + i * kMF + t;
            const float *p = mine + t * kPitch + at;
            const i32x4 x = *reinterpret_cast<const i32x4 *>(p);
            i32x4 y = {0, 0, 0, 0};
            if constexpr (kDual) y = *reinterpret_cast<const i32x4 *>(p + kMF);
            if (m < a.M && cnt > 0) finish4<E, OUT, PAST>(a, of, m, n, cnt, x, y);
        }
        wave_sync();
    }
}

// BM x BN tile, WM x WN waves, for bf16 and int8 rows that start on no 16-byte boundary: operands go
// through registers into LDS.  A step of the contraction takes 128 bytes of every row (64 bf16, 128
// int8): its chunks are loaded HELD steps before they are written into LDS and HELD + 1 before they
// are used (small tiles, whose steps are shorter than a load, hold three), and written between the
// halves of a step's matrix instructions (10% faster at 8192^3 than around all of them).
template <class E, int BM, int BN, int WM, int WN, int HELD, Out OUT> struct TileKernel {
    static constexpr bool kDual = OUT == Out::kGated;
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int TM = BM / WM, TN = BN / WN;     // a wave's tokens and channels
    static constexpr int NM = TM / kMF, NN = TN / kMF;
    static constexpr int kRowBytes = 128;
    static constexpr int kRowChunks = kRowBytes / kChunk;
    static constexpr int kRowsPerPass = kThreads / kRowChunks;
    static constexpr int LA = BM / kRowsPerPass, LB = BN / kRowsPerPass;   // chunks per thread
    static constexpr int kStageBytes = (BM + BN) * kRowBytes;
    static constexpr int kEpiBytes = WM * WN * epilogue_bytes(NN);
    static constexpr int kLds = 2 * kStageBytes > kEpiBytes ? 2 * kStageBytes : kEpiBytes;
    static constexpr int kTileN = kDual ? BN / 2 : BN;   // channels per tile
    using M_ = Mma<E>;
    using Acc = typename M_::Acc;
    static_assert(BM % kRowsPerPass == 0 && BN % kRowsPerPass == 0, "whole passes");
    static_assert(!kDual || NN % 2 == 0, "gate and up blocks in pairs");
    static_assert(kLds <= 160 * 1024, "LDS of a CU");

    // LDS position of 16-byte chunk c of a row: the chunks of a row are permuted by its number, so
    // that a wave's reads of 16 rows spread over all banks (no conflicts counted).
    static __device__ __forceinline__ int swizzled(int row, int c) { return c ^ ((row >> 1) & 7); }

    static __device__ __forceinline__ void run(const ProductArgs &a, char *lds) {
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
        const int wm = wave % WM, wn = wave / WM;
        const TileRows<BM, kTileN, kDual> rows(a);
        const int c = tid & (kRowChunks - 1), r0 = tid / kRowChunks;
        const int wave_row = wave * (64 / kRowChunks);      // first row of this wave in a pass
        struct Held {                        // a step's chunks of this thread
            i32x4 a[LA], b[LB];
        };
        Held held[HELD];                     // step k in held[k % HELD], its place in LDS k % 2
        RowChunks<E, Load::kBytes> ca[LA], cb[LB];
#pragma unroll
        for (int i = 0; i < LA; ++i) ca[i].set(rows.a, i * kRowsPerPass + r0, c * kChunk, a.Kb);
#pragma unroll
        for (int i = 0; i < LB; ++i)
            cb[i].set(rows.b(i * kRowsPerPass + wave_row), rows.channel(i * kRowsPerPass + r0),
                      c * kChunk, a.Kb);
        auto load = [&](int step, Held &h) { // zeros from Kb on
            const int kb = step * kRowBytes, left = a.Kb - c * kChunk - kb;
#pragma unroll
            for (int i = 0; i < LA; ++i) h.a[i] = ca[i].load(kb, left);
#pragma unroll
            for (int i = 0; i < LB; ++i) h.b[i] = cb[i].load(kb, left);
        };
        auto put = [&](int buf, const Held &h) {
            char *p = lds + buf * kStageBytes;
#pragma unroll
            for (int i = 0; i < LA + LB; ++i) {
                const int row = (i < LA ? i : i - LA) * kRowsPerPass + r0;
                *reinterpret_cast<i32x4 *>(p + (i < LA ? 0 : BM * kRowBytes) + row * kRowBytes +
                                           swizzled(row, c) * kChunk) = i < LA ? h.a[i] : h.b[i - LA];
            }
        };

        Acc acc[NN][NM] = {};
        const int fr = lane % kMF, fc = lane / kMF;
        const int steps = (a.Kb + kRowBytes - 1) / kRowBytes;
#pragma unroll
        for (int k = 0; k < HELD; ++k) load(k, held[k]);
        put(0, held[0]);
        load(HELD, held[0]);
        // Step s, whose successor waits in h.
        auto step = [&](int s, Held &h) {
            __syncthreads();
            const char *pa = lds + (s & 1) * kStageBytes + (wm * TM + fr) * kRowBytes;
            const char *pb = lds + (s & 1) * kStageBytes + (BM + wn * TN + fr) * kRowBytes;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = swizzled(fr, k * 4 + fc) * kChunk;
                i32x4 fa[NM], fb[NN];
#pragma unroll
                for (int i = 0; i < NM; ++i)
                    fa[i] = *reinterpret_cast<const i32x4 *>(pa + i * kMF * kRowBytes + at);
#pragma unroll
                for (int j = 0; j < NN; ++j)
                    fb[j] = *reinterpret_cast<const i32x4 *>(pb + j * kMF * kRowBytes + at);
#pragma unroll
                for (int j = 0; j < NN; ++j)
#pragma unroll
                    for (int i = 0; i < NM; ++i) acc[j][i] = M_::step(fb[j], fa[i], acc[j][i]);
                if (k == 0) {
                    put((s + 1) & 1, h);
                    load(s + 1 + HELD, h);
                }
            }
        };
        for (int s = 0; s < steps;) {
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                step(s, held[(k + 1) % HELD]);
                if (++s >= steps) break;
            }
        }
        __syncthreads();
        epilogue<E, OUT, NN, NM>(a, acc, reinterpret_cast<float *>(lds + wave * epilogue_bytes(NN)),
                                 rows.m0 + wm * TM, rows.n0 + wn * (kDual ? TN / 2 : TN));
    }
};

template <class E, int BM, int BN, int WM, int WN, int HELD, Out OUT>
__global__ __launch_bounds__(64 * WM * WN) void dense_tile_kernel(ProductArgs a) {
    using K = TileKernel<E, BM, BN, WM, WN, HELD, OUT>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
