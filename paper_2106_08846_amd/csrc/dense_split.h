// The tiled product (dense_tile.h) of fp32 operands, on bf16 matrix instructions.
//
// fp32 values as sums of three bf16 pieces, x = h + m + l: h is x rounded to bf16, m the remainder
// rounded, l what is left, which has 8 significant bits (|m| <= 2^-9 |x|, |l| <= 2^-18 |x|; exact
// while l does not underflow, |x| >= 2^-100).  A product x y is formed from the six cross terms down
// to 2^-18 |x y| (hh, hm, mh, hl, lh, mm), each exact in fp32; the three left out are together below
// 2^-25.9 |x y|, a quarter of fp32's own rounding.  Six bf16 instructions take 96 cycles for what
// the fp32 instructions need 256 for.
//
// The ends of the range.  An operand that rounds to infinity (from 2^128 (1 - 2^-9) on) has l = NaN, which
// reaches all its outputs: a tile with a NaN among its sums is made again, with h clamped to the largest
// bf16 and the rest in m (|m| <= 2^-8 |x| then, and what is left out is below 2^-25).  The other outputs
// of that tile come out the same.  Clamping always would cost 2 to 4% (one instruction a value; 1000 x
// 768 x 1531 trains in 154 us with it, 148 without); so only tiles with such operands, infinities or NaN
// take twice as long.  An infinite operand gives NaN.  Pieces below 2^-126 may be lost, at most 2^-125 of
// an operand.  h may be larger than x, so a sum with a term within 2^-8 of fp32's largest value may
// overflow.
#pragma once

#include <type_traits>

#include "dense_tile.h"

namespace bsr {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kLargestBf16 = 0x1.fep127f;

// The next piece of eight values: four packed conversions; what is left stays in x.  CLAMP: to the
// largest bf16.
template <bool CLAMP> __device__ __forceinline__ i32x4 next_piece(f32x8 &x) {
    auto in_range = [](float v) {
        return CLAMP ? __builtin_amdgcn_fmed3f(v, -kLargestBf16, kLargestBf16) : v;
    };
    i32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 pair = {in_range(x[2 * i]), in_range(x[2 * i + 1])};
        const bf16x2 h = __builtin_convertvector(pair, bf16x2);
        const unsigned u = __builtin_bit_cast(unsigned, h);
        p[i] = int(u);
        x[2 * i] -= __uint_as_float(u << 16);
        x[2 * i + 1] -= __uint_as_float(u & 0xffff0000u);
    }
    return p;
}

// BM x BN tile, WM x WN waves.  A step of the contraction takes 32 fp32 values of every row; they are
// split on their way from registers into LDS, where each piece has a plane of 64-byte rows.  LDS
// holds a ring of three steps.  While the 6 NN NM matrix instructions of step s run, the fragments of
// step s + 1 are read into the registers of those that have been used for the last time, step s + 2
// is split (ten vector instructions beside every few matrix instructions) and written, and step s + 5
// is loaded: three steps wait in registers, since a step of a small tile is shorter than a load.  The
// product of the middle pieces comes first, so that the first pieces, read last, have time to arrive;
// the product of the first pieces comes last, so that the small terms are not lost to it (a row of X
// that picks out one weight gives that weight, exactly).
//
// At 4096^3 (MI355X) a step of 128 x 128 takes 1.3 us, of which the matrix instructions alone are 0.7:
// the split's vector instructions add their own time to them (0.4 us) rather than run beside them.
template <int BM, int BN, int WM, int WN, bool ALIGNED, Out OUT> struct SplitKernel {
    static constexpr bool kDual = OUT == Out::kGated;
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int TM = BM / WM, TN = BN / WN;
    static constexpr int NM = TM / kMF, NN = TN / kMF;
    static constexpr int kStepBytes = 128;               // of a row of fp32
    static constexpr int kRowBytes = 64;                 // of a row of one piece in LDS
    static constexpr int kRowsPerPass = kThreads / 4;    // four lanes, 8 values each, to a row
    static constexpr int L = (BM + BN) / kRowsPerPass;   // the tile's rows: A's, then B's
    static constexpr int kPlaneBytes = (BM + BN) * kRowBytes;
    static constexpr int kStageBytes = 3 * kPlaneBytes;
    static constexpr int kEpiBytes = WM * WN * epilogue_bytes(NN);
    static constexpr int kTileLds = 3 * kStageBytes > kEpiBytes ? 3 * kStageBytes : kEpiBytes;
    static constexpr int kLds = kTileLds + WM * WN * 4;  // a flag for each wave
    static constexpr int kTileN = kDual ? BN / 2 : BN;
    using M_ = Mma<bf16>;
    using Acc = typename M_::Acc;
    static_assert((BM + BN) % kRowsPerPass == 0 && BM % kMF == 0, "whole passes and groups");
    static_assert(!kDual || NN % 2 == 0, "gate and up blocks in pairs");
    static_assert(kLds <= 160 * 1024, "LDS of a CU");

    static __device__ __forceinline__ void pin() { asm volatile("" ::: "memory"); }

    static __device__ __forceinline__ void run(const ProductArgs &a, char *lds) {
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
        const int wm = wave % WM, wn = wave / WM;
        const TileRows<BM, kTileN, kDual> rows(a);
        const int c = tid & 3, r0 = tid >> 2;
        struct Held {                        // a step's values of this thread
            f32x8 v[L];
        };
        Held held[3];                        // step k in held[k % 3], its place in LDS slot k % 3
        RowChunks<float, ALIGNED ? Load::kAligned : Load::kBytes> chunks[L];
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int first = i * kRowsPerPass + wave * 16, row = i * kRowsPerPass + r0;
            if (first < BM)           // uniform
                chunks[i].set(rows.a, row, c * 2 * kChunk, a.Kb);
            else
                chunks[i].set(rows.b(first - BM), rows.channel(row - BM), c * 2 * kChunk, a.Kb);
        }
        const Slice slice(a, (a.Kb + kStepBytes - 1) / kStepBytes);
        const int end = min(a.Kb, (slice.first + slice.steps) * kStepBytes);
        auto load = [&](int step, Held &h) { // zeros from the slice's end on
            const int kb = (slice.first + step) * kStepBytes, left = end - c * 2 * kChunk - kb;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                i32x4 v[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) v[q] = chunks[i].load(kb + q * kChunk, left - q * kChunk);
                __builtin_memcpy(&h.v[i], v, sizeof v);
            }
        };
        // Piece x of this thread's i-th row into the stage at p.
        const int put_at = half_row_at(r0, c);
        auto put = [&](char *p, int i, int x, i32x4 v) {
            *reinterpret_cast<i32x4 *>(p + x * kPlaneBytes + i * kRowsPerPass * kRowBytes + put_at) = v;
        };

        Acc acc[NN][NM] = {};
        const int fr = lane % kMF, fc = lane / kMF;
        const int at_a = wm * TM * kRowBytes + half_row_at(fr, fc);
        const int at_b = (BM + wn * TN) * kRowBytes + half_row_at(fr, fc);
        // The sums of the tile, with first pieces clamped or not.
        auto sum = [&](auto clamp) {
            i32x4 fa[3][NM], fb[3][NN];
            auto fetch_a = [&](const char *p, int x) {
#pragma unroll
                for (int i = 0; i < NM; ++i)
                    fa[x][i] = *reinterpret_cast<const i32x4 *>(p + x * kPlaneBytes + at_a +
                                                               i * kMF * kRowBytes);
            };
            auto fetch_b = [&](const char *p, int x) {
#pragma unroll
                for (int j = 0; j < NN; ++j)
                    fb[x][j] = *reinterpret_cast<const i32x4 *>(p + x * kPlaneBytes + at_b +
                                                               j * kMF * kRowBytes);
            };
            auto piece = [](f32x8 &v, int x) {
                return x == 0 ? next_piece<decltype(clamp)::value>(v) : next_piece<false>(v);
            };
            auto put_all = [&](char *p, Held &h) {
#pragma unroll
                for (int i = 0; i < L; ++i)
#pragma unroll
                    for (int x = 0; x < 3; ++x) put(p, i, x, piece(h.v[i], x));
            };
            load(0, held[0]);
            load(1, held[1]);
            load(2, held[2]);
            put_all(lds, held[0]);
            load(3, held[0]);
            put_all(lds + kStageBytes, held[1]);
            load(4, held[1]);
            __syncthreads();
#pragma unroll
            for (int x = 0; x < 3; ++x) {
                fetch_a(lds, x);
                fetch_b(lds, x);
            }
            // Step s, s % 3 = SLOT.
            auto step = [&](int s, auto slot) {
                constexpr int kSlot = decltype(slot)::value;
                const char *p = lds + (kSlot + 1) % 3 * kStageBytes;
                char *to = lds + (kSlot + 2) % 3 * kStageBytes;
                Held &h = held[(kSlot + 2) % 3];
                // Six products of NN groups of NM instructions: piece kB of B with piece kA of A.
                constexpr int kB[6] = {1, 0, 2, 0, 1, 0}, kA[6] = {1, 2, 0, 1, 0, 0};
                constexpr int kCuts = 3 * L, kCutSlots = 4 * NN;     // the split: in the first four
#pragma unroll
                for (int g = 0; g < 6 * NN; ++g) {
                    const int w = g / NN, j = g % NN;
#pragma unroll
                    for (int i = 0; i < NM; ++i)
                        acc[j][i] = M_::step(fb[kB[w]][j], fa[kA[w]][i], acc[j][i]);
#pragma unroll
                    for (int q = 0; q < kCuts; ++q)
                        if (q * kCutSlots / kCuts == g) put(to, q / 3, q % 3, piece(h.v[q / 3], q % 3));
                    if (j == NN - 1) {
                        if (w == 1) fetch_a(p, 2);
                        if (w == 2) fetch_b(p, 2);
                        if (w == 3) fetch_a(p, 1);
                        if (w == 4) {
                            pin();
                            load(s + 5, h);
                            fetch_b(p, 1);
                        }
                        if (w == 5) {
                            fetch_b(p, 0);
                            fetch_a(p, 0);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                pin();
                // This wave's writes of step s + 2 are older than its last NM + NN reads: done.
                __builtin_amdgcn_s_waitcnt(0xc07f | ((NM + NN) << 8));
                __builtin_amdgcn_s_barrier();
                pin();
            };
            // Whole rounds of three: steps past the end multiply zeros.
            for (int s = 0; s < slice.steps; s += 3) {
                step(s, std::integral_constant<int, 0>{});
                step(s + 1, std::integral_constant<int, 1>{});
                step(s + 2, std::integral_constant<int, 2>{});
            }
        };
        sum(std::false_type{});
        bool lost = false;                   // a sum is NaN
#pragma unroll
        for (int j = 0; j < NN; ++j)
#pragma unroll
            for (int i = 0; i < NM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) lost |= acc[j][i][e] != acc[j][i][e];
        int *flags = reinterpret_cast<int *>(lds + kTileLds);
        const int any = __any(lost);
        if (lane == 0) flags[wave] = any;
        __syncthreads();
        int again = 0;
#pragma unroll
        for (int w = 0; w < WM * WN; ++w) again |= flags[w];
        if (uniform(again)) {
#pragma unroll
            for (int j = 0; j < NN; ++j)
#pragma unroll
                for (int i = 0; i < NM; ++i) acc[j][i] = Acc{};
            sum(std::true_type{});
            __syncthreads();
        }
        epilogue<float, OUT, NN, NM>(a, acc, reinterpret_cast<float *>(lds + wave * epilogue_bytes(NN)),
                                     rows.m0 + wm * TM, rows.n0 + wn * (kDual ? TN / 2 : TN));
    }
};

template <int BM, int BN, int WM, int WN, bool ALIGNED, Out OUT>
__global__ __launch_bounds__(64 * WM * WN) void dense_split_kernel(ProductArgs a) {
    using K = SplitKernel<BM, BN, WM, WN, ALIGNED, OUT>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
