// The product of 8-bit floating-point matrices (f8_product.h) in tiles.  LDS holds two stages of one block
// of 128 columns each, with the block's scales.
//
// A wave's order of work in a block: token fragment i meets the channel fragments j in turn.  The sums of
// (i, j) are added to the outputs while the matrix unit forms those of the next pair.  A token fragment is
// read from LDS two i before its use, a channel fragment over the last two i of the block before, so the
// reads of a block end two i before its products do (kDepth; one i in the tile with the least registers left):
// there every wave waits for the next block's data and meets the others, and the loads of the block after
// that go into the stage that is free from then on.  They have most of a block's products to arrive.
//
// DIRECT (rows on 16-byte boundaries): codes go straight from memory into LDS.  Otherwise they go through
// registers, loaded byte-aligned at the same point and written shortly before the next meeting (128 x 4096 x
// 4095 takes 26 us so in one part, 34 where the codes are shifted out of aligned words).
//
// PARTS: so many groups of WM x WN waves share out the blocks of a contraction, each with stages of its own,
// and add their sums at the end.
//
// MI355X, 8192^3: bf16 output 447 to 474 us, card by card (2.3 to 2.5 Pflop/s, at the 1.9 GHz that the power
// leaves; matrix and vector instructions take 61% and 41% of the cycles and hardly overlap; the library's
// product with one scale takes 339).  fp32
// output 1.35 Pflop/s, and with a scale for each row of B 1.16: there the vector instructions (12 and 15 to
// four matrix instructions) and the matrix instructions take turns (with a scale for each row 43% and 45% of
// the cycles).
#pragma once

#include <type_traits>

#include "f8_product.h"

namespace bsr {

template <int BM, int BN, int WM, int WN, int XF, bool WROWS, bool WIDE, bool DIRECT, int PARTS = 1>
struct F8RingKernel {
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves * PARTS;    // kWaves: of a part
    static constexpr int TM = BM / WM, TN = BN / WN;
    static constexpr int NM = TM / kMF, NN = TN / kMF;
    static constexpr int kRowBytes = kF8Block;
    // A load of a wave is 8 rows of 128 bytes.  Scales: 64 of a load, in as many loads for either operand.
    static constexpr int PA = BM / 8 / kWaves, PB = BN / 8 / kWaves;
    static constexpr int kScaleLoadsX = BM / 64, kScaleLoadsW = WROWS ? BN / 64 : 1;
    static constexpr int kScaleAt = (BM + BN) * kRowBytes, kScaleWAt = kScaleAt + BM * 4;
    static constexpr int kStageBytes = kScaleWAt + kScaleLoadsW * 256;
    static constexpr int kStages = 2;        // four are no faster, not in the smallest tile either
    static constexpr int kEpiBytes = kWaves * epilogue_bytes(NN);
    static constexpr int kPartBytes = kStages * kStageBytes;
    static constexpr int kLds = PARTS * kPartBytes > kEpiBytes ? PARTS * kPartBytes : kEpiBytes;
    // Parts hand their sums over through the stages, behind the epilogue's own LDS.
    static constexpr int kSumBytes = NM * NN * 16 * 64 * kWaves;
    static_assert(kLds >= (PARTS > 1 ? kEpiBytes + (PARTS - 1) * kSumBytes : 0), "room for the parts' sums");
    static constexpr int kTileN = BN;
    // How many i ahead token fragments are read.  256 x 256 with widened codes and a scale for each row of B takes
    // more than the 256 registers of a wave (nine go to memory, two ahead 25), and still gains on two rounds of
    // half the tile: 8192 x 2048 x 6144 191 us and 205, 4096 x 4096 x 4096 121 and 133, 8192^3 922 and 966.
    static constexpr int kDepth = WIDE && WROWS && BM * BN > 192 * 256 ? 1 : 2;
    static_assert(DIRECT || kDepth == 2, "codes on their way through registers are put in place two i ahead");
    static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && BM % 64 == 0, "whole loads");
    static_assert(kScaleLoadsX + kScaleLoadsW <= kWaves, "one scale load of a wave");
    static_assert(kF8Block % TN == 0 && NM >= 2, "one scale of B for a wave's channels");
    static_assert(kLds <= 160 * 1024, "LDS of a CU");

    typedef __attribute__((address_space(3))) char lds_char;
    typedef __attribute__((address_space(3))) void lds_void;

    static __device__ __forceinline__ int swizzled(int row, int c) { return c ^ ((row >> 1) & 7); }
    static __device__ __forceinline__ void pin() { asm volatile("" ::: "memory"); }

    static __device__ __forceinline__ void run(const F8Args &args, char *lds) {
        const ProductArgs &a = args.p;
        const int lane = threadIdx.x & 63, part = uniform(threadIdx.x >> 6) / kWaves;
        const int wave = uniform(threadIdx.x >> 6) % kWaves;
        const int wm = wave % WM, wn = wave / WM;
        char *const all = lds;
        lds += part * kPartBytes;
        const TileRows<BM, kTileN, false> rows(a);
        const Source &sa = rows.a, &sb = rows.b0;
        constexpr unsigned kOut = 0x80000000u;      // out of every range: loads zeros
        // The last row's end is rounded up to the dword that holds it, which the range check would drop.
        const auto end = [&](const Source &s) {
            return (unsigned((s.rows - 1) * s.pitch) + unsigned(a.Kb) + 3u) & ~3u;
        };
        const auto rsa = buffer_rsrc(sa.base, end(sa)), rsb = buffer_rsrc(sb.base, end(sb));
        // A lane's place in a load's 8 rows, and the chunk of the row that belongs there, the same for all of
        // its loads (a multiple of 16 rows apart).  Rows that do not exist begin past the range's end.
        static_assert(kWaves % 2 == 0, "loads of a wave a multiple of 16 rows apart");
        const int row0 = wave * 8 + (lane >> 3), c0 = swizzled(row0, lane & 7) * kChunk;
        const unsigned oa = unsigned(row0) * unsigned(sa.pitch) + c0;
        const unsigned ob = unsigned(row0) * unsigned(sb.pitch) + c0;
        const int64_t left_m = a.M - rows.m0, left_n = a.N - rows.n0;
        const int w_first = int(WROWS ? 0 : rows.n0 / kF8Block);
        const float *sx = args.sx + rows.m0, *sw = args.sw + (WROWS ? rows.n0 : w_first);
        const unsigned bytes_x = unsigned(left_m < BM ? left_m : BM) * 4;
        const unsigned bytes_w = WROWS ? unsigned(left_n < BN ? left_n : BN) * 4
                                       : unsigned((a.N - 1) / kF8Block - w_first + 1 < (BN + 127) / 128
                                                      ? (a.N - 1) / kF8Block - w_first + 1
                                                      : (BN + 127) / 128) * 4;
        // Part p takes every PARTS-th block from p on; blocks past the end are zeros.
        const int blocks = (a.Kb + kRowBytes - 1) / kRowBytes, steps = (blocks + PARTS - 1) / PARTS;
        // A step's loads in pieces, by number: codes of A (DIRECT), of B, then scales, as many in every wave (some
        // load the same scales).  Steps past the end load zeros, scales too: a part that has no block there
        // adds 0, also where sx sw is infinite.
        constexpr int kCodes = DIRECT ? PA + PB : 0, kPieces = kCodes + 1;
        auto load = [&](int step, int piece) {
            const int block = step * PARTS + part, kb = block * kRowBytes;
            lds_char *stage = (lds_char *)lds + (step & 1) * kStageBytes;
            if (piece < kCodes) {
                const bool of_a = piece < PA, in = kb + c0 < a.Kb;
                const int i = of_a ? piece : piece - PA;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    of_a ? rsa : rsb,
                    (lds_void *)(stage + (of_a ? 0 : BM * kRowBytes) + (i * kWaves + wave) * 1024), 16,
                    in ? (of_a ? oa : ob) : kOut, kb + i * kWaves * 8 * int(of_a ? sa.pitch : sb.pitch), 0, 0);
                return;
            }
            const int n = wave % (kScaleLoadsX + kScaleLoadsW);
            const bool of_x = n < kScaleLoadsX, in = block < blocks;
            const int64_t row = in ? block : 0;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                of_x ? buffer_rsrc(sx + row * args.ldsx, bytes_x) : buffer_rsrc(sw + row * args.ldsw, bytes_w),
                (lds_void *)(stage + kScaleAt + n * 256), 4,
                in ? (of_x ? n : n - kScaleLoadsX) * 256 + lane * 4 : kOut, 0, 0, 0);
        };
        // !DIRECT: the codes of a step on their way through registers, in the same places.  Rows that do not
        // exist stand for the last one: they reach only outputs that do not exist.
        i32x4 held[DIRECT ? 1 : PA + PB];
        RowChunks<int8_t, Load::kBytes> chunk[DIRECT ? 1 : PA + PB];
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < PA + PB; ++i)
                chunk[i].set(i < PA ? sa : sb, row0 + (i < PA ? i : i - PA) * kWaves * 8, c0, a.Kb);
        }
        auto take = [&](int step) {
            if (step >= steps) return;
            const int kb = (step * PARTS + part) * kRowBytes;
            if (kb + kRowBytes <= a.Kb) {
#pragma unroll
                for (int i = 0; i < PA + PB; ++i) held[i] = chunk[i].load(kb, kChunk);
            } else {
#pragma unroll
                for (int i = 0; i < PA + PB; ++i) held[i] = chunk[i].load(kb, a.Kb - c0 - kb);
            }
        };
        auto put = [&](int step) {
            if (step >= steps) return;
            char *p = lds + (step & 1) * kStageBytes + wave * 1024 + lane * kChunk;
#pragma unroll
            for (int i = 0; i < PA + PB; ++i)
                *reinterpret_cast<i32x4 *>(p + (i < PA ? i : i - PA) * kWaves * 1024 +
                                           (i < PA ? 0 : BM * kRowBytes)) = held[i];
        };
        // What lies beyond a row's end in its last chunk, replaced by zeros.
        const int tail = DIRECT ? a.Kb % kChunk : 0;
        auto clear_tail = [&](int step) {
            char *p = lds + (step & 1) * kStageBytes;
            const int c = a.Kb % kRowBytes / kChunk;
            if (step * PARTS + part == blocks - 1)
                for (int row = wave * 64 + lane; row < BM + BN; row += 64 * kWaves) {
                    i32x4 *at = reinterpret_cast<i32x4 *>(p + row * kRowBytes + swizzled(row, c) * kChunk);
                    *at = first_bytes(*at, tail);
                }
            __syncthreads();
        };
        // This wave's reads of the stage are done and the next block's loads are there, for every wave.
        auto meet = [&](int next) {
            pin();
            __builtin_amdgcn_s_waitcnt(0x0070);          // vmcnt(0) lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
            pin();
            if (tail && next == steps - 1) clear_tail(next);
        };

        f32x4 acc[NN][NM] = {};
        const int fr = lane % kMF, fc = lane / kMF;
        const int at_lo = fr * kRowBytes + swizzled(fr, fc) * kChunk;
        const int at_hi = fr * kRowBytes + swizzled(fr, fc + 4) * kChunk;
        const auto fetch = [&](const char *p) {
            return join_chunks(*reinterpret_cast<const i32x4 *>(p + at_lo),
                               *reinterpret_cast<const i32x4 *>(p + at_hi));
        };
        const auto fetch_a = [&](const char *stage, int i) { return fetch(stage + (wm * TM + i * kMF) * kRowBytes); };
        const auto fetch_b = [&](const char *stage, int j) {
            return fetch(stage + (BM + wn * TN + j * kMF) * kRowBytes);
        };
        const auto fetch_sx = [&](const char *stage, int i) {
            return reinterpret_cast<const float *>(stage + kScaleAt)[wm * TM + i * kMF + fr];
        };
        // Of four channels of a fragment, or of all the wave's.
        using WScale = std::conditional_t<WROWS, f32x4, float>;
        constexpr int kWScales = WROWS ? NN : 1;
        const auto fetch_sw = [&](const char *stage, int j) {
            const float *s = reinterpret_cast<const float *>(stage + kScaleWAt);
            if constexpr (WROWS)
                return *reinterpret_cast<const f32x4 *>(s + wn * TN + j * kMF + 4 * fc);
            else
                return s[wn * TN / kF8Block];
        };
        const auto add = [](f32x4 &out, const f32x4 &sum, const WScale &of) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (WROWS)
                    out[e] = fmaf(sum[e], of[e], out[e]);
                else
                    out[e] = fmaf(sum[e], of, out[e]);
            }
            // Here, and not after the loads and products that follow, which would keep every pair's sums.
            asm volatile("" : "+v"(out));
        };
        // Where in a block's products each piece is issued: with every second product from the meeting on
        // (all at once behind it, waves wait to issue them: 8192^3 475 us, 455 so), closer where a block has
        // few products.  The first kFirst come before the block ends, the others in the next.
        constexpr int kSlots = NM * NN, kApart = 2 * kPieces <= kSlots ? 2 : 1;
        constexpr int kPerSlot = (kPieces + kSlots - 1) / kSlots;
        constexpr int kBeforeEnd = (kDepth * NN + kApart - 1) / kApart * kPerSlot;
        constexpr int kFirst = kBeforeEnd < kPieces ? kBeforeEnd : kPieces;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) load(0, i);
        if constexpr (!DIRECT) take(0), put(0);
        meet(0);
#pragma unroll
        for (int i = 0; i < kFirst; ++i) load(1, i);
        if constexpr (!DIRECT) take(1);
        i32x8 fa[kDepth];
        // Channel fragments have two sets of registers where they fit, and the next block's are read over
        // the last two i (8192^3 446 us, 455 with one set); in one set each is replaced as its last product
        // is issued.
        constexpr int kSets = WIDE || !DIRECT || (WROWS && BM * BN > 192 * 256) ? 1 : 2;
        F8Fragment<BSR_E4M3, WIDE> fb[kSets][NN];
        float sxi[kDepth];
        WScale swj[kWScales];
#pragma unroll
        for (int j = 0; j < NN; ++j) fb[0][j].set(fetch_b(lds, j));
#pragma unroll
        for (int j = 0; j < kWScales; ++j) swj[j] = fetch_sw(lds, j);
#pragma unroll
        for (int i = 0; i < kDepth; ++i) fa[i] = fetch_a(lds, i), sxi[i] = fetch_sx(lds, i);
        // The sums that wait to be added to the outputs, and their scales.
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        WScale of{};
        // Block s, whose channel fragments are in the given set of registers.
        auto block = [&](int s, auto set) {
            constexpr int kMine = decltype(set)::value;
            F8Fragment<BSR_E4M3, WIDE>(&mine)[NN] = fb[kMine], (&next_b)[NN] = fb[kSets - 1 - kMine];
            const char *now = lds + (s & 1) * kStageBytes, *then = lds + ((s + 1) & 1) * kStageBytes;
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                if constexpr (!DIRECT)
                    if (i == (NM > 2 ? NM - 3 : 0)) put(s + 1);
                if (i == NM - kDepth) {
                    meet(s + 1);
                    if constexpr (!DIRECT) take(s + 2);
                }
                F8Fragment<XF, WIDE> x;
                x.set(fa[i % kDepth]);
                const float scale = sxi[i % kDepth];
                const char *from = i + kDepth < NM ? now : then;
                const int next = (i + kDepth) % NM;
#pragma unroll
                for (int j = 0; j < NN; ++j) {
                    const f32x4 more = block_sums<XF>(mine[j], x);
                    const int slot = (i + kDepth) % NM * NN + j;
#pragma unroll
                    for (int p = 0; p < kPieces; ++p)
                        if (p / kPerSlot * kApart == slot) load(i < NM - kDepth ? s + 1 : s + 2, p);
                    __builtin_amdgcn_sched_barrier(0);
                    add(acc[j > 0 ? j - 1 : NN - 1][j > 0 ? i : i > 0 ? i - 1 : NM - 1], sum, of);
                    sum = more;
                    if (WROWS || j == 0) of = swj[WROWS ? j : 0] * scale;
                    // a widened fragment leaves its codes' registers at once
                    if (j == (WIDE ? 0 : NN - 1))
                        fa[i % kDepth] = fetch_a(from, next), sxi[i % kDepth] = fetch_sx(from, next);
                    if constexpr (kSets == 1) {
                        if (i == NM - 1) next_b[j].set(fetch_b(then, j));
                    } else {
                        constexpr int kEvery = NN > 1 ? 2 : 1;
                        const int at = (i - (NM - 2)) * NN + j;
                        if (i >= NM - 2 && at % kEvery == 0 && at / kEvery < NN)
                            next_b[at / kEvery].set(fetch_b(then, at / kEvery));
                    }
                    if (i == NM - 1 && j < kWScales) swj[j] = fetch_sw(then, j);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        using std::integral_constant;
        if constexpr (kSets == 1) {
            for (int s = 0; s < steps; ++s) block(s, integral_constant<int, 0>{});
        } else {
            int s = 0;
            for (; s + 1 < steps; s += 2) {
                block(s, integral_constant<int, 0>{});
                block(s + 1, integral_constant<int, 1>{});
            }
            if (s < steps) block(s, integral_constant<int, 0>{});
        }
        add(acc[NN - 1][NM - 1], sum, of);
        __builtin_amdgcn_s_waitcnt(0x0070);      // loads past the end, before LDS is used again
        __syncthreads();
        if constexpr (PARTS > 1) {               // the first part adds the others' sums, in order
            f32x4 *sums = reinterpret_cast<f32x4 *>(all + kEpiBytes) + wave * 64 + lane;
            constexpr int kStride = 64 * kWaves;
            if (part > 0) {
#pragma unroll
                for (int j = 0; j < NN; ++j)
#pragma unroll
                    for (int i = 0; i < NM; ++i)
                        sums[((part - 1) * NN * NM + j * NM + i) * kStride] = acc[j][i];
            }
            __syncthreads();
            if (part > 0) return;
#pragma unroll
            for (int p = 0; p < PARTS - 1; ++p)
#pragma unroll
                for (int j = 0; j < NN; ++j)
#pragma unroll
                    for (int i = 0; i < NM; ++i) acc[j][i] += sums[(p * NN * NM + j * NM + i) * kStride];
        }
        // Past the caches: 9616 x 768 x 656 with bf16 output takes 14.5 us through them and 12.3 so, 4096 x 1024
        // x 1024 with fp32 output 17.8 and 16.1.
        epilogue<bf16, Out::kScale, NN, NM, true>(
            a, acc, reinterpret_cast<float *>(lds + wave * epilogue_bytes(NN)), rows.m0 + wm * TM,
            rows.n0 + wn * TN);
    }
};

template <int BM, int BN, int WM, int WN, int XF, bool WROWS, bool WIDE, bool DIRECT, int PARTS = 1>
__global__ __launch_bounds__(64 * WM * WN * PARTS) void f8_ring_kernel(F8Args a) {
    using K = F8RingKernel<BM, BN, WM, WN, XF, WROWS, WIDE, DIRECT, PARTS>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
