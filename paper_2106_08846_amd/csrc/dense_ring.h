// The tiled product (dense_tile.h) for bf16 and int8 rows on 16-byte boundaries: global memory goes
// straight into LDS, several steps deep.
//
// A step of the contraction takes 64 bytes of every row: one 16-byte operand chunk per lane, one
// matrix instruction per pair of fragments.  LDS holds a ring of RING steps.  While the matrix
// instructions of step s run, their operands for step s + 1 are read from the ring into the
// registers that step s frees one by one, and step s + RING - 1 is being written into the place of
// step s - 1, which every wave had read by the last barrier.  So no wave waits for LDS after a
// barrier, and a load has RING - 2 whole steps to arrive: two of 1000 cycles for the largest tile,
// more and shorter ones for the small tiles.
//
// One workgroup of 256 x 256 outputs fills a CU: 8 waves of 128 x 64, 128 KB of LDS.  At 8192^3
// (MI355X) it runs at 1.23-1.27 Pflop/s in bf16 and 2.4 Pop/s in int8, within 6% of the library
// products on the same card; the matrix units are busy 60-68% of the cycles, at the 1.6-1.8 GHz that
// the card's power leaves them.
// COLS_A, COLS_B (bf16): the operand's rows lie along the outputs instead, k after k: an operand of a
// gradient, as it is in memory.  A step is then 32 of its rows, cut to the tile's columns, and the
// fragments are read from LDS with the transposing read (ds_read_b64_tr_b16), which gives a lane four
// k of its column.
#pragma once

#include "dense_tile.h"

namespace bsr {

template <class E, int BM, int BN, int WM, int WN, int RING, Out OUT, bool COLS_A = false,
          bool COLS_B = false>
struct RingKernel {
    static constexpr bool kDual = OUT == Out::kGated;
    static constexpr int kWaves = WM * WN;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int TM = BM / WM, TN = BN / WN;
    static constexpr int NM = TM / kMF, NN = TN / kMF;
    static constexpr int kRowBytes = 64;
    // Each wave loads groups of 16 rows (64 lanes of 16 bytes).  A tile height that does not give
    // every wave the same number of groups is rounded up in LDS; those rows are loaded as zeros.
    static constexpr int PA = (BM / 16 + kWaves - 1) / kWaves, PB = (BN / 16 + kWaves - 1) / kWaves;
    static constexpr int kRowsA = PA * kWaves * 16, kRowsB = PB * kWaves * 16;
    static constexpr int kStageBytes = (kRowsA + kRowsB) * kRowBytes;
    static constexpr int kEpiBytes = kWaves * epilogue_bytes(NN);
    static constexpr int kLds = RING * kStageBytes > kEpiBytes ? RING * kStageBytes : kEpiBytes;
    static constexpr int kTileN = kDual ? BN / 2 : BN;
    using M_ = Mma<E>;
    using Acc = typename M_::Acc;
    static_assert(BM % 16 == 0 && BN % 16 == 0 && TM % kMF == 0 && TN % kMF == 0, "whole blocks");
    static_assert(!kDual || (NN % 2 == 0 && kWaves % 2 == 0), "gate and up blocks in pairs");
    static_assert(kLds <= 160 * 1024, "LDS of a CU");
    static constexpr int kAhead = (RING - 3) * (PA + PB);   // loads in flight across a barrier
    static_assert(RING >= 4 && kAhead < 64, "vmcnt");

    static_assert(!COLS_A || COLS_B, "as the gradients have them");
    static_assert(!COLS_B || (sizeof(E) == 2 && !kDual), "bf16 gradients");

    typedef __attribute__((address_space(3))) char lds_char;
    typedef __attribute__((address_space(3))) void lds_void;

    // Keep the compiler from moving memory accesses across.
    static __device__ __forceinline__ void pin() { asm volatile("" ::: "memory"); }
    // All but this wave's last N loads into LDS have arrived.
    template <int N> static __device__ __forceinline__ void wait_loads() {
        pin();
        __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);   // vmcnt(N)
    }

    // A column operand in LDS: ROWS columns of 32 k, row k in ROWS * 2 bytes, whose 32-byte segments
    // are permuted by fold(k), so that the rows a transposing read takes together (4 of every 8) lie on
    // different banks.
    template <int ROWS> struct Columns {
        static constexpr int kPitch = ROWS * 2;                  // 128 bytes or more
        static constexpr int kChunks = kPitch / kChunk;
        static __device__ __forceinline__ int fold(int k) {
            const int eight = (k >> 3) & 1;
            return kPitch >= 256 ? (k & 3) | eight << 2 : ((k >> 1) & 1) | eight << 1;
        }
        // The chunk that belongs at 16-byte place `at` of the step: row k, column chunk c.
        static __device__ __forceinline__ void place(int at, int &k, int &c) {
            k = at / kChunks;
            c = (at % kChunks) ^ (fold(k) << 1);
        }
        // The 16 columns from 16 * segment on: k = 8 (lane / 16) .. + 7 of column lane % 16.
        static __device__ __forceinline__ i32x4 fetch(const char *p, int lane, int segment) {
            const int j = lane & 15, k = (lane >> 4) * 8 + (j >> 2);
            const char *q = p + k * kPitch + (segment ^ fold(k)) * 32 + (j & 3) * 8;
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(q));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(q + 4 * kPitch));
            i32x4 v;
            __builtin_memcpy(&v, &lo, 8);
            __builtin_memcpy(reinterpret_cast<char *>(&v) + 8, &hi, 8);
            return v;
        }
    };
    // Where a column operand's step comes from: `rows` rows of one matrix, or of two, the second from
    // step `half` on; their columns from the tile's first on.
    struct ColumnSource {
        const char *base[2];
        int64_t pitch[2];
        int rows, half;
        unsigned width;           // bytes of a row from the tile's first column on, whole chunks (the
                                  // range check drops a dword that ends outside)
        // Descriptor (buffer_rsrc's four words) of the step's rows, as far as they exist.
        __device__ __forceinline__ i32x4 rsrc(int s, unsigned &ld) const {
            const int which = s >= half, k = (s - (which ? half : 0)) * 32, left = rows - k;
            const int64_t step_ld = which ? pitch[1] : pitch[0];
            const char *p = (which ? base[1] : base[0]) + k * step_ld;
            ld = unsigned(step_ld);
            const unsigned bytes = left > 0 ? unsigned((left < 32 ? left : 32) - 1) * ld + width : 0u;
            const uint64_t at = reinterpret_cast<uint64_t>(p);
            return i32x4{int(at), int(at >> 32) & 0xffff, int(bytes), 0x00020000};
        }
    };

    // 16 bytes a lane from `off` of the descriptor's range into the 1024 at `to`.  Written as an
    // instruction because the compiler waits for every load into LDS that it knows of before it reads
    // LDS with the transposing read, which would leave one step in flight; wait_loads does the waiting.
    // It has no result register, and no compiler-made wait depends on it.
    static __device__ __forceinline__ void load_unseen(i32x4 rsrc, lds_char *to, unsigned off) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"(unsigned(reinterpret_cast<uintptr_t>(to))), "v"(off), "s"(rsrc)
                     : "memory", "m0");
    }

    static __device__ __forceinline__ void run(const ProductArgs &a, char *lds) {
        const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
        const int wm = wave % WM, wn = wave / WM;
        const TileRows<BM, kTileN, kDual> rows(a);
        // Offsets from `kOut` on are out of every range and load zeros.
        constexpr unsigned kOut = 0x80000000u;
        // A group's 1024 bytes in LDS are written in lane order, so a lane loads what belongs in its
        // place there.
        //
        // Rows: group g holds rows 16 g .. (gated: gate rows where g is even, up rows where it is odd; a
        // wave's groups g = i * kWaves + wave are all of one kind), and a lane's place is line lane / 8,
        // position lane % 8 of half_row_at's layout.
        const bool up = kDual && (wave & 1);
        const Source &sa = rows.a, &sb = up ? rows.b1 : rows.b0;
        const unsigned bytes_a = unsigned((sa.rows - 1) * sa.pitch) + unsigned(a.Kb);
        const auto rsa = buffer_rsrc(sa.base, bytes_a);
        const auto rsb = buffer_rsrc(sb.base, unsigned((sb.rows - 1) * sb.pitch) + unsigned(a.Kb));
        const uint64_t base_a = reinterpret_cast<uint64_t>(sa.base);
        const i32x4 words_a = {int(base_a), int(base_a >> 32) & 0xffff, int(bytes_a), 0x00020000};
        const int place = (lane & 7) ^ (lane >> 3), row = (lane >> 3) * 2 + (place >> 2), c = place & 3;
        unsigned oa[PA], ob[PB];
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int r = (i * kWaves + wave) * 16 + row;
            oa[i] = r < sa.rows ? unsigned(r) * unsigned(sa.pitch) + c * kChunk : kOut;
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int g = i * kWaves + wave, r = (kDual ? g >> 1 : g) * 16 + row;
            ob[i] = r < sb.rows ? unsigned(r) * unsigned(sb.pitch) + c * kChunk : kOut;
        }
        // Columns: the operand's matrices from the tile's first column on.
        const ColumnSource ca{{a.A + rows.m0 * 2, a.A1 + rows.m0 * 2}, {a.lda, a.lda}, a.rows_k, a.half,
                              unsigned((a.M - rows.m0 + 7) / 8) * kChunk};
        const ColumnSource cb{{a.B0 + rows.n0 * 2, a.B1 + rows.n0 * 2}, {a.ldb0, a.ldb1}, a.rows_k,
                              a.half, unsigned((a.N - rows.n0 + 7) / 8) * kChunk};
        using ColsA = Columns<kRowsA>;
        using ColsB = Columns<kRowsB>;

        const Slice slice(a, (a.Kb + kRowBytes - 1) / kRowBytes);
        auto load = [&](int step) {
            const int s = slice.first + step;
            const int kb = s * kRowBytes;
            const bool in = kb + c * kChunk < a.Kb;      // chunks past the row's end: zeros
            lds_char *to = (lds_char *)lds + (step % RING) * kStageBytes + wave * 1024;
            auto columns = [&](auto cols, const ColumnSource &src, lds_char *at, int tile, int groups) {
                unsigned ld;
                const i32x4 rsrc = src.rsrc(s, ld);
#pragma unroll
                for (int i = 0; i < groups; ++i) {
                    int k, chunk;
                    cols.place((i * kWaves + wave) * 64 + lane, k, chunk);
                    load_unseen(rsrc, at + i * kWaves * 1024,
                                chunk * 8 < tile ? __umul24(unsigned(k), ld) + unsigned(chunk) * kChunk : kOut);
                }
            };
            if constexpr (COLS_A) {
                columns(ColsA{}, ca, to, BM, PA);
            } else {
#pragma unroll
                for (int i = 0; i < PA; ++i) {
                    const unsigned off = in ? oa[i] + kb : kOut;
                    if constexpr (COLS_B)
                        load_unseen(words_a, to + i * kWaves * 1024, off);
                    else
                        __builtin_amdgcn_raw_ptr_buffer_load_lds(
                            rsa, (lds_void *)(to + i * kWaves * 1024), 16, off, 0, 0, 0);
                }
            }
            to += kRowsA * kRowBytes;
            if constexpr (COLS_B) {
                columns(ColsB{}, cb, to, BN, PB);
            } else {
#pragma unroll
                for (int i = 0; i < PB; ++i)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(
                        rsb, (lds_void *)(to + i * kWaves * 1024), 16, in ? ob[i] + kb : kOut, 0, 0, 0);
            }
        };

        Acc acc[NN][NM] = {};
        const int fr = lane % kMF, fc = lane / kMF;
        const int at_a = wm * TM * kRowBytes + half_row_at(fr, fc);
        const int at_b = (kRowsA + wn * TN) * kRowBytes + half_row_at(fr, fc);
        auto fetch_a = [&](const char *p, int i) {
            if constexpr (COLS_A) return ColsA::fetch(p, lane, wm * NM + i);
            return *reinterpret_cast<const i32x4 *>(p + at_a + i * kMF * kRowBytes);
        };
        auto fetch_b = [&](const char *p, int j) {
            if constexpr (COLS_B) return ColsB::fetch(p + kRowsA * kRowBytes, lane, wn * NN + j);
            return *reinterpret_cast<const i32x4 *>(p + at_b + j * kMF * kRowBytes);
        };
        i32x4 fa[NM], fb[2][NN];
        const int steps = slice.steps;
#pragma unroll
        for (int s = 0; s < RING - 1; ++s) load(s);
        wait_loads<kAhead>();          // steps 0 and 1 are there
        __builtin_amdgcn_s_barrier();
        pin();
#pragma unroll
        for (int j = 0; j < NN; ++j) fb[0][j] = fetch_b(lds, j);
#pragma unroll
        for (int i = 0; i < NM; ++i) fa[i] = fetch_a(lds, i);
        auto step = [&](int s, const i32x4 (&now)[NN], i32x4 (&then)[NN]) {
            const char *p = lds + ((s + 1) % RING) * kStageBytes;
#pragma unroll
            for (int i = 0; i < NM; ++i) {
#pragma unroll
                for (int j = 0; j < NN; ++j) acc[j][i] = M_::step(now[j], fa[i], acc[j][i]);
                fa[i] = fetch_a(p, i);
                if (i == 0) load(s + RING - 1);
                // the channels' fragments, spread over the rest of the step
#pragma unroll
                for (int j = 0; j < NN; ++j)
                    if (j * NM / NN == i) then[j] = fetch_b(p, j);
                __builtin_amdgcn_sched_barrier(0);
            }
            wait_loads<kAhead>();      // step s + 2 is there
            __builtin_amdgcn_s_barrier();
            pin();
        };
        int s = 0;
        for (; s + 1 < steps; s += 2) {
            step(s, fb[0], fb[1]);
            step(s + 1, fb[1], fb[0]);
        }
        if (s < steps) step(s, fb[0], fb[1]);
        wait_loads<0>();               // what was loaded past the end, before LDS is used again
        __syncthreads();
        // The tiles that large products take write more than the L2s hold, and store past them: a gated
        // int8 block of 2048 tokens, 4096 to 10240 features, takes 175 us with plain stores and 168 so,
        // an int8 product of 8192^3 466 and 457.  The smaller tiles' outputs stay for the kernel that
        // reads them next (the fp32 gradients of 1000 tokens, 768 features and 1531 hidden units: 150
        // us past the caches, 146 through them).
        constexpr bool kPast = BM * BN >= 192 * 256;
        epilogue<E, OUT, NN, NM, kPast>(a, acc, reinterpret_cast<float *>(lds + wave * epilogue_bytes(NN)),
                                        rows.m0 + wm * TM, rows.n0 + wn * (kDual ? TN / 2 : TN));
    }
};

template <class E, int BM, int BN, int WM, int WN, int RING, Out OUT, bool COLS_A = false,
          bool COLS_B = false>
__global__ __launch_bounds__(64 * WM * WN) void dense_ring_kernel(ProductArgs a) {
    using K = RingKernel<E, BM, BN, WM, WN, RING, OUT, COLS_A, COLS_B>;
    __shared__ __align__(16) char lds[K::kLds];
    K::run(a, lds);
}

}  // namespace bsr
