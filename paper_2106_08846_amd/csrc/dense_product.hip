// The dense products' launches: 8-bit rows with scales, the gated block's projections and its
// gradients, on the tiled matrix-core kernel (dense_tile.h).
#include <type_traits>

#include "dense_plan.h"
#include "dense_ring.h"
#include "dense_rows.h"
#include "dense_split.h"

namespace bsr {

namespace {

constexpr int kThreads = 256;

template <class T> constexpr int64_t kSize = sizeof(T);

// Launch `kernel` over the tiles of K.
template <class K, int BM>
void launch_tiles(void (*kernel)(ProductArgs), ProductArgs a, void *stream, unsigned slices = 1) {
    a.tiles_m = int((a.M + BM - 1) / BM);
    a.tiles_n = int((a.N + K::kTileN - 1) / K::kTileN);
    hipLaunchKernelGGL(kernel, dim3(unsigned(a.tiles_m) * unsigned(a.tiles_n), slices),
                       dim3(K::kThreads), 0, as_stream(stream), a);
}
template <class E, int BM, int BN, int WM, int WN, int RING, Out OUT, bool COLS_A, bool COLS_B>
void launch_ring(const ProductArgs &a, void *stream) {
    launch_tiles<RingKernel<E, BM, BN, WM, WN, RING, OUT, COLS_A, COLS_B>, BM>(
        dense_ring_kernel<E, BM, BN, WM, WN, RING, OUT, COLS_A, COLS_B>, a, stream);
}
template <class E, int BM, int BN, int WM, int WN, int HELD, Out OUT>
void launch_tile(const ProductArgs &a, void *stream) {
    launch_tiles<TileKernel<E, BM, BN, WM, WN, HELD, OUT>, BM>(
        dense_tile_kernel<E, BM, BN, WM, WN, HELD, OUT>, a, stream);
}
template <int BM, int BN, int WM, int WN, Out OUT>
void launch_split(const ProductArgs &a, bool aligned, void *stream) {
    using K = SplitKernel<BM, BN, WM, WN, true, OUT>;
    if constexpr (OUT != Out::kStore)    // the gradients' operands are laid out by the library
        if (!aligned)
            return launch_tiles<K, BM>(dense_split_kernel<BM, BN, WM, WN, false, OUT>, a, stream);
    launch_tiles<K, BM>(dense_split_kernel<BM, BN, WM, WN, true, OUT>, a, stream);
}

template <class E, int NT, Out OUT>
void launch_rows(const ProductArgs &a, bool aligned, void *stream) {
    using K = RowsKernel<E, NT, true, OUT>;
    const auto kernel = aligned ? dense_rows_kernel<E, NT, true, OUT>
                                : dense_rows_kernel<E, NT, false, OUT>;
    const unsigned groups_n = unsigned((a.N + K::kChannels - 1) / K::kChannels);
    const unsigned groups_m = unsigned((a.M + 16 * NT - 1) / (16 * NT));
    hipLaunchKernelGGL(kernel, dim3(groups_n, groups_m), dim3(64 * K::kWaves), 0, as_stream(stream), a);
}

bool rows_aligned(const void *p, int64_t ld) {
    return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(ld)) & 15) == 0;
}

template <class E, Out OUT, bool COLS_A, bool COLS_B>
void launch_ring_tile(const ProductArgs &a, int tile, void *stream) {
    switch (tile) {
        case 0: return launch_ring<E, 256, 256, 2, 4, 4, OUT, COLS_A, COLS_B>(a, stream);
        case 1: return launch_ring<E, 192, 256, 2, 4, 4, OUT, COLS_A, COLS_B>(a, stream);
        case 2: return launch_ring<E, 128, 256, 2, 4, 4, OUT, COLS_A, COLS_B>(a, stream);
        case 3: return launch_ring<E, 128, 128, 2, 4, 4, OUT, COLS_A, COLS_B>(a, stream);
        default: return launch_ring<E, 64, 64, 2, 2, 8, OUT, COLS_A, COLS_B>(a, stream);
    }
}

// The product's channels from n on, as a product of its own.
ProductArgs channels_from(ProductArgs a, int64_t n, bool cols_b) {
    const int64_t out_size = a.out_bf16 ? 2 : 4;
    const auto skip = [&](const char *p, int64_t ld) { return p ? p + (cols_b ? 2 * n : n * ld) : p; };
    const auto vec = [&](const float *p) { return p ? p + n : p; };
    const auto out = [&](void *p) { return p ? static_cast<char *>(p) + n * out_size : nullptr; };
    a.B0 = skip(a.B0, a.ldb0);
    a.B1 = skip(a.B1, a.ldb1);
    a.s0 = vec(a.s0);
    a.s1 = vec(a.s1);
    a.b0 = vec(a.b0);
    a.b1 = vec(a.b1);
    a.out = out(a.out);
    a.out2 = out(a.out2);
    a.G = a.G ? a.G + n : nullptr;
    a.U = a.U ? a.U + n : nullptr;
    a.N -= n;
    return a;
}

// Rows of the weights that a product's channels take in its tiles.
int64_t weight_rows(const ProductArgs &a, bool dual) { return dual ? 2 * a.N : a.N; }

template <class E, Out OUT, bool COLS_A = false, bool COLS_B = false>
void launch_ring_product(const ProductArgs &a, void *stream) {
    constexpr bool dual = OUT == Out::kGated;
    const int64_t cus = device_cu_count(), rows = weight_rows(a, dual);
    if (const int64_t whole = rows_in_whole_rounds(a.M, rows, cus)) {
        ProductArgs first = a;
        first.N = dual ? whole / 2 : whole;
        const ProductArgs rest = channels_from(a, first.N, COLS_B);
        launch_ring_tile<E, OUT, COLS_A, COLS_B>(first, 0, stream);
        const int tile = cheapest_tile(kRingTiles, a.M, weight_rows(rest, dual), cus);
        return launch_ring_tile<E, OUT, COLS_A, COLS_B>(rest, tile, stream);
    }
    launch_ring_tile<E, OUT, COLS_A, COLS_B>(a, cheapest_tile(kRingTiles, a.M, rows, cus), stream);
}

template <class E, Out OUT> void launch_product(const ProductArgs &a, void *stream) {
    constexpr bool dual = OUT == Out::kGated;
    const bool aligned = a.Kb % 16 == 0 && rows_aligned(a.A, a.lda) && rows_aligned(a.B0, a.ldb0) &&
                         (!dual || rows_aligned(a.B1, a.ldb1));
    if constexpr (OUT != Out::kStore) {
        // Beyond one group of 32 only where its workgroups, each with a whole contraction to itself, fit
        // the chip in one round: bf16 64 x 1024 x 4096 takes 12 us here and 19 in tiles, 128 x 1024 x
        // 8192 23 and 34, 64 x 4096 x 4096 (two rounds) 24 and 19.
        if (a.M <= 16) return launch_rows<E, 1, OUT>(a, aligned, stream);
        if (a.M <= 32 || ((a.M + 31) / 32) * ((a.N + 15) / 16) <= device_cu_count())
            return launch_rows<E, 2, OUT>(a, aligned, stream);
    }
    const int64_t cus = device_cu_count(), rows = weight_rows(a, dual);
    if constexpr (sizeof(E) == 4) {
        if (cheapest_tile(kSplitTiles, a.M, rows, cus) == 0)
            launch_split<128, 128, 4, 2, OUT>(a, aligned, stream);
        else
            launch_split<64, 64, 4, 2, OUT>(a, aligned, stream);
    } else if (aligned) {
        launch_ring_product<E, OUT>(a, stream);
    } else {
        switch (cheapest_tile(kRegisterTiles, a.M, rows, cus)) {
            case 0: return launch_tile<E, 256, 256, 2, 4, 1, OUT>(a, stream);
            case 1: return launch_tile<E, 128, 256, 2, 4, 1, OUT>(a, stream);
            case 2: return launch_tile<E, 128, 128, 2, 4, 2, OUT>(a, stream);
            default: return launch_tile<E, 64, 64, 2, 2, 3, OUT>(a, stream);
        }
    }
}

// f(constant activation) for the block's activation.
template <class F> void with_act(int act, F &&f) {
    switch (act) {
        case BSR_ACT_SILU: f(std::integral_constant<int, BSR_ACT_SILU>{}); break;
        case BSR_ACT_GELU: f(std::integral_constant<int, BSR_ACT_GELU>{}); break;
        case BSR_ACT_GELU_TANH: f(std::integral_constant<int, BSR_ACT_GELU_TANH>{}); break;
        default: f(std::integral_constant<int, BSR_ACT_RELU>{}); break;
    }
}

template <class T>
void gated(const void *X, int64_t T_, int64_t ldx, const float *sx, const bsr_gated_t &W, void *H,
           int h_dtype, int64_t ldh, float *G, float *U, int64_t ldp, void *stream) {
    ProductArgs a{};
    a.A = static_cast<const char *>(X);
    a.B0 = static_cast<const char *>(W.Wg);
    a.B1 = static_cast<const char *>(W.Wu);
    a.lda = ldx * kSize<T>;
    a.ldb0 = W.ldg * kSize<T>;
    a.ldb1 = W.ldu * kSize<T>;
    a.M = T_;
    a.N = W.F;
    a.Kb = int(W.K * kSize<T>);
    a.sx = sx;
    a.s0 = W.sg;
    a.s1 = W.su;
    a.b0 = W.bg;
    a.b1 = W.bu;
    a.out = H;
    a.ldo = ldh;
    a.out_bf16 = h_dtype == BSR_BF16;
    a.act = W.act;
    a.G = G;
    a.U = U;
    a.ldp = ldp;
    launch_product<T, Out::kGated>(a, stream);
}

// --- gradients ----------------------------------------------------------------------------------
// The two gradient products sum over the hidden width and over the tokens, along which their
// operands are not contiguous.  bf16: the product kernel takes them as they are (column operands);
// fp32: dG and dU are written in both orders where they are made, X and the weights are transposed.
// Padding keeps every row 16-byte aligned and holds zeros.

constexpr int kT = 64;   // tile of the transposing kernels
template <class T> constexpr int kV = 16 / int(sizeof(T));      // elements of 16 bytes

// A kT x kT tile in LDS, written by rows and read by columns, 16 bytes of the matrices at a time.
// The pitch of 2 elements more puts the rows of a column that consecutive lanes read on different
// banks.
template <class T> struct TransposeTile {
    T cell[kT][kT + 2];
    __device__ __forceinline__ void put(int row, int col, const T (&v)[kV<T>]) {
#pragma unroll
        for (int i = 0; i < kV<T>; ++i) cell[row][col + i] = v[i];
    }
    // out[c][r] for the tile at rows r0 (a multiple of 64), columns c0: `C` columns exist, out's rows
    // have `pad` elements (a multiple of 16 bytes).
    __device__ __forceinline__ void store(T *out, int64_t ldo, int64_t r0, int64_t c0, int64_t C,
                                          int64_t pad) const {
        constexpr int per = kT / kV<T>;
        for (int e = threadIdx.x; e < kT * per; e += kThreads) {
            const int c = e / per, r = e % per * kV<T>;
            if (c0 + c >= C || r0 + r >= pad) continue;
            T v[kV<T>];
#pragma unroll
            for (int i = 0; i < kV<T>; ++i) v[i] = cell[r + i][c];
            __builtin_memcpy(out + (c0 + c) * ldo + r0 + r, v, 16);
        }
    }
};

// kV elements p[0 .. n), the rest zero.
template <class T> __device__ __forceinline__ void load_some(const T *p, int64_t n, T (&v)[kV<T>]) {
    if (n >= kV<T>) {
        __builtin_memcpy(v, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kV<T>; ++i) v[i] = i < n ? p[i] : T{};
    }
}

// out[c][r] = in[r][c] for r < R, c < C; out's rows are padded with zeros to `pad` columns.  The
// gradients' three matrices (both weights and the tokens) go in one launch (6 us for 1000 tokens, 768
// features and 1531 hidden units; 11 in two): tiles from first[i] on are matrix i's.  Beyond 2^16
// tiles a workgroup takes several: 2^24 of them, which the sizes allow, would be more threads than a
// launch can have.
struct Transposes {
    const float *in[3];
    float *out[3];
    int64_t ldi[3], R[3], C[3], ldo[3], pad[3];
    unsigned first[3];
    int matrices;
    unsigned tiles;
    void add(const void *from, int64_t ldi_, int64_t R_, int64_t C_, float *to, int64_t ldo_,
             int64_t pad_) {
        const int i = matrices++;
        in[i] = static_cast<const float *>(from);
        out[i] = to;
        ldi[i] = ldi_;
        R[i] = R_;
        C[i] = C_;
        ldo[i] = ldo_;
        pad[i] = pad_;
        first[i] = tiles;
        tiles += unsigned((pad_ + kT - 1) / kT * ((C_ + kT - 1) / kT));
    }
};
__global__ __launch_bounds__(kThreads) void transpose_kernel(Transposes of) {
    __shared__ TransposeTile<float> tile;
    for (unsigned at = blockIdx.x; at < of.tiles; at += gridDim.x) {
        int i = 0;
#pragma unroll
        for (int j = 1; j < 3; ++j)
            if (j < of.matrices && at >= of.first[j]) i = j;
        const float *in = of.in[i];
        const int64_t ldi = of.ldi[i], R = of.R[i], C = of.C[i], pad = of.pad[i];
        const unsigned id = at - of.first[i], across = unsigned((pad + kT - 1) / kT);
        const int64_t r0 = int64_t(id % across) * kT, c0 = int64_t(id / across) * kT;
        constexpr int V = kV<float>, per = kT / V;
#pragma unroll
        for (int e = threadIdx.x; e < kT * per; e += kThreads) {
            const int r = e / per, c = e % per * V;
            float v[V];
            load_some(in + (r0 + r) * ldi + c0 + c, r0 + r < R ? C - c0 - c : 0, v);
            tile.put(r, c, v);
        }
        __syncthreads();
        tile.store(of.out[i], of.ldo[i], r0, c0, C, pad);
        __syncthreads();
    }
}

// out[r][c] = in[r][c] for c < C, rows of `pad` elements (a multiple of 16 bytes) padded with zeros.
template <class T>
__global__ __launch_bounds__(kThreads) void copy_rows_kernel(const T *__restrict__ in, int64_t ldi,
                                                             int64_t R, int64_t C, T *__restrict__ out,
                                                             int64_t pad) {
    const int64_t per = pad / kV<T>, n = R * per;
    for (int64_t e = int64_t(blockIdx.x) * kThreads + threadIdx.x; e < n;
         e += int64_t(gridDim.x) * kThreads) {
        const int64_t r = e / per, c = e % per * kV<T>;
        T v[kV<T>];
        load_some(in + r * ldi + c, C - c, v);
        __builtin_memcpy(out + r * pad + c, v, 16);
    }
}

// D[t][f] = dH U act'(G), D[t][Fp + f] = dH act(G), zeros up to Fp, and the sums of their columns over
// the tile's tokens.  Into Dt goes, as ALSO says, the transpose Dt[f][t], Dt[F + f][t], or, in D's layout,
// what the rounding of D to bf16 dropped, itself rounded to bf16 (at most 2^-16 of a value is left out
// then; a value that rounds to infinity drops nothing).
//
// bf16: D is rounded because it is an operand of the bf16 instructions, an error of at most 2^-8 a term,
// of the size of a bf16 gradient's own rounding (6144 x 2048 x 8192: gradients 0.235% off, 0.166% with
// D in fp32).  fp32 gradients have no such rounding, so they take the dropped part too: the weights'
// product takes 700 us instead of 343 there, the slopes 180 instead of 160, the whole step 1.28-1.30
// times as long.
//
// Memory bound: 16 bytes of D (4 or 8 hidden units of a token) per thread and pass.  6144 tokens of 8192
// hidden units in bf16 (700 MB) take 160 us on MI355X, 4.4 TB/s; reading G and U past the caches made
// no difference, and tiles of 256 hidden units gained 6 us there and cost 8 on a step of 100 tokens (53
// us).
enum class Also { kNothing, kTransposed, kDropped };
__device__ __forceinline__ bf16 dropped(float v, bf16 kept) {
    const float k = to_float(kept);
    return to_bf16(fabsf(k) < INFINITY ? v - k : 0.0f);
}
template <class T, int ACT, Also ALSO>
__global__ __launch_bounds__(kThreads) void gated_slope_kernel(
    const T *__restrict__ dH, int64_t lddh, const float *__restrict__ G,
    const float *__restrict__ U, int64_t ldp, int64_t T_, int64_t F, T *__restrict__ D, int64_t Fp,
    T *__restrict__ Dt, int64_t Tp, float *__restrict__ partial) {
    constexpr int V = kV<T>, per = kT / V, kRows = kThreads / per;
    constexpr bool kBoth = ALSO == Also::kTransposed;
    __shared__ typename std::conditional<kBoth, TransposeTile<T>, char>::type tg, tu;
    __shared__ float sums[2][kRows][kT + 1];
    const int64_t t0 = int64_t(blockIdx.x) * kT, f0 = int64_t(blockIdx.y) * kT;
    const int y = threadIdx.x / per, x = threadIdx.x % per * V;
    const int64_t f = f0 + x;
    float pg[V] = {}, pu[V] = {};
#pragma unroll
    for (int i = y; i < kT; i += kRows) {
        const int64_t t = t0 + i, n = t < T_ ? F - f : 0;
        T dh[V], dg[V], du[V], lg[V], lu[V];
        float g[V], u[V];
        load_some(dH + t * lddh + f, n, dh);
        if (n >= V) {
            __builtin_memcpy(g, G + t * ldp + f, sizeof g);
            __builtin_memcpy(u, U + t * ldp + f, sizeof u);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                g[j] = j < n ? G[t * ldp + f + j] : 0.0f;
                u[j] = j < n ? U[t * ldp + f + j] : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float a, da;
            activate_slope<ACT>(g[j], a, da);
            const float h = to_float(dh[j]);
            const float vg = j < n ? h * u[j] * da : 0.0f, vu = j < n ? h * a : 0.0f;
            pg[j] += vg;
            pu[j] += vu;
            dg[j] = from_float<T>(vg);
            du[j] = from_float<T>(vu);
            if constexpr (ALSO == Also::kDropped) {
                lg[j] = dropped(vg, dg[j]);
                lu[j] = dropped(vu, du[j]);
            }
        }
        if constexpr (kBoth) {
            tg.put(i, x, dg);
            tu.put(i, x, du);
        }
        if (t < T_ && f < Fp) {
            __builtin_memcpy(D + t * 2 * Fp + f, dg, 16);
            __builtin_memcpy(D + t * 2 * Fp + Fp + f, du, 16);
            if constexpr (ALSO == Also::kDropped) {
                __builtin_memcpy(Dt + t * 2 * Fp + f, lg, 16);
                __builtin_memcpy(Dt + t * 2 * Fp + Fp + f, lu, 16);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        sums[0][y][x + j] = pg[j];
        sums[1][y][x + j] = pu[j];
    }
    __syncthreads();
    if constexpr (kBoth) {
        tg.store(Dt, Tp, t0, f0, F, Tp);
        tu.store(Dt + F * Tp, Tp, t0, f0, F, Tp);
    }
    if (threadIdx.x < 2 * kT) {
        const int which = threadIdx.x / kT, c = threadIdx.x % kT;
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) s += sums[which][r][c];
        if (f0 + c < F) partial[int64_t(blockIdx.x) * 2 * F + which * F + f0 + c] = s;
    }
}

// The sums of `blocks` rows of partial sums, 2 F each: kBiasCols columns to a workgroup, whose groups
// of threads take every kBiasRows-th row and are added, in order, through LDS (a thread that walks all
// rows of its column waits for memory at each: 16384 of them at the most tokens).
constexpr int kBiasCols = 16, kBiasRows = kThreads / kBiasCols;
template <class T>
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(const float *__restrict__ partial,
                                                             int64_t blocks, int64_t F,
                                                             T *__restrict__ dbg,
                                                             T *__restrict__ dbu) {
    __shared__ float sums[kBiasRows][kBiasCols + 1];
    const int c = threadIdx.x % kBiasCols, y = threadIdx.x / kBiasCols;
    const int64_t f = int64_t(blockIdx.x) * kBiasCols + c;
    float s = 0.0f;
    if (f < 2 * F) {
#pragma unroll 8
        for (int64_t b = y; b < blocks; b += kBiasRows) s += partial[b * 2 * F + f];
    }
    sums[y][c] = s;
    __syncthreads();
    if (y > 0 || f >= 2 * F) return;
#pragma unroll
    for (int r = 1; r < kBiasRows; ++r) s += sums[r][c];
    if (f < F) {
        if (dbg) dbg[f] = from_float<T>(s);
    } else if (dbu) {
        dbu[f - F] = from_float<T>(s);
    }
}

// rows x cols elements of zeros.
template <class T>
__global__ __launch_bounds__(kThreads) void zero_rows_kernel(T *__restrict__ p, int64_t rows,
                                                             int64_t cols, int64_t ld) {
    const int64_t n = rows * cols;
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += int64_t(gridDim.x) * kThreads)
        p[i / cols * ld + i % cols] = T{};
}

unsigned cover(int64_t n, int64_t tile) { return unsigned((n + tile - 1) / tile); }

// A matrix as a column operand: itself where its rows are whole 16-byte chunks on 16-byte boundaries,
// else copied to `space` with rows of Kp elements.
struct ColumnOperand {
    const char *p;
    int64_t ld;      // bytes
};
ColumnOperand as_columns(const void *in, int64_t ldi, int64_t R, int64_t C, char *space, int64_t Kp,
                         void *stream) {
    if (C % 8 == 0 && rows_aligned(in, ldi * 2)) return {static_cast<const char *>(in), ldi * 2};
    hipLaunchKernelGGL(copy_rows_kernel<bf16>, dim3(grid_for(R * (Kp / 8), kThreads, 4096)),
                       dim3(kThreads), 0, as_stream(stream), static_cast<const bf16 *>(in), ldi, R, C,
                       reinterpret_cast<bf16 *>(space), Kp);
    return {space, Kp * 2};
}

// The slices' sums, in order, to where the product goes.
template <class TG>
__global__ __launch_bounds__(kThreads) void join_slices_kernel(ProductArgs a,
                                                               const float *__restrict__ sums,
                                                               int slices) {
    const int64_t per = (a.N + 3) / 4, n = a.M * per;
    for (int64_t e = int64_t(blockIdx.x) * kThreads + threadIdx.x; e < n;
         e += int64_t(gridDim.x) * kThreads) {
        const int64_t m = e / per, c = e % per * 4;
        const int cnt = int(a.N - c < 4 ? a.N - c : 4);
        f32x4 v = load4(sums, m * a.N + c, cnt, 0.0f);
        for (int z = 1; z < slices; ++z) v += load4(sums, (z * a.M + m) * a.N + c, cnt, 0.0f);
        const int64_t row = m < a.split ? m : m - a.split;
        if (row < a.limit)
            store4<false>(m < a.split ? a.out : a.out2, row * a.ldo + c, sizeof(TG) == 2, v, cnt);
    }
}

// A gradient product, cut into slices of its contraction where its outputs are too few to fill the
// chip: with them a training step of 100 x 1000 x 4000 (dX: 32 tiles, 250 steps) takes 55 us in bf16,
// 80 without.
template <class T, class TG, bool COLS_A>
void gradient_product(const ProductArgs &a, int slices, float *sums, void *stream) {
    constexpr bool columns = sizeof(T) == 2;
    if (slices == 1) {
        if constexpr (columns)
            launch_ring_product<T, Out::kStore, COLS_A, true>(a, stream);
        else
            launch_product<T, Out::kStore>(a, stream);
        return;
    }
    ProductArgs part = a;
    const int steps = (a.Kb + 32 * int(sizeof(T)) - 1) / (32 * int(sizeof(T)));
    part.slice = (steps + slices - 1) / slices;
    part.out = sums;
    const unsigned used = unsigned((steps + part.slice - 1) / part.slice);
    if constexpr (columns) {
        using K = RingKernel<T, 64, 64, 2, 2, 8, Out::kStore, COLS_A, true>;
        launch_tiles<K, 64>(dense_ring_kernel<T, 64, 64, 2, 2, 8, Out::kStore, COLS_A, true>, part,
                            stream, used);
    } else {
        using K = SplitKernel<64, 64, 4, 2, true, Out::kStore>;
        launch_tiles<K, 64>(dense_split_kernel<64, 64, 4, 2, true, Out::kStore>, part, stream, used);
    }
    hipLaunchKernelGGL(join_slices_kernel<TG>, dim3(grid_for(a.M * ((a.N + 3) / 4), kThreads, 2048)),
                       dim3(kThreads), 0, as_stream(stream), a, sums, int(used));
}

template <class T, class TG>
void backward(const void *dH, int64_t lddh, const void *X, int64_t T_, int64_t ldx,
              const bsr_gated_t &W, const float *G, const float *U, int64_t ldp, void *dX,
              int64_t lddx, void *dWg, void *dWu, int64_t lddw, void *dbg, void *dbu, void *ws,
              void *stream) {
    constexpr bool columns = sizeof(T) == 2;
    const int64_t K = W.K, F = W.F;
    const GatedWorkspace l = gated_workspace_layout(T_, K, F, raw_enum(W.dtype));
    char *base = static_cast<char *>(ws);
    T *D = reinterpret_cast<T *>(base + l.grad_offset);
    T *Dt = reinterpret_cast<T *>(base + l.gradt_offset);
    char *x_space = base + l.x_offset, *w_space = base + l.w_offset;
    float *partial = reinterpret_cast<float *>(base + l.partial_offset);
    float *sums = reinterpret_cast<float *>(base + l.slice_offset);
    constexpr bool dropped = columns && std::is_same<TG, float>::value;     // of the weights' product
    if (T_ > 0)
        with_act(W.act, [&](auto act) {
            constexpr Also plain = columns ? Also::kNothing : Also::kTransposed;
            auto kernel = gated_slope_kernel<T, decltype(act)::value, plain>;
            if constexpr (dropped)
                if (dWg) kernel = gated_slope_kernel<T, decltype(act)::value, Also::kDropped>;
            hipLaunchKernelGGL(kernel, dim3(cover(columns ? T_ : l.Tp, kT), cover(l.Fp, kT)),
                               dim3(kThreads), 0, as_stream(stream), static_cast<const T *>(dH), lddh,
                               G, U, ldp, T_, F, D, l.Fp, Dt, l.Tp, partial);
        });
    if (dbg || dbu)
        hipLaunchKernelGGL(bias_grad_kernel<TG>, dim3(cover(2 * F, kBiasCols)), dim3(kThreads), 0,
                           as_stream(stream), partial, int64_t(cover(T_, kT)), F,
                           static_cast<TG *>(dbg), static_cast<TG *>(dbu));
    if constexpr (!columns) {
        Transposes of{};
        float *Wt = reinterpret_cast<float *>(w_space);
        if (dX) {
            of.add(W.Wg, W.ldg, F, K, Wt, 2 * l.Fp, l.Fp);
            of.add(W.Wu, W.ldu, F, K, Wt + l.Fp, 2 * l.Fp, l.Fp);
        }
        if (dWg) of.add(X, ldx, T_, K, reinterpret_cast<float *>(x_space), l.Tp, l.Tp);
        if (of.matrices && T_ > 0)
            hipLaunchKernelGGL(transpose_kernel, dim3(grid_for(of.tiles, 1, kTransposeGroups)),
                               dim3(kThreads), 0, as_stream(stream), of);
    }
    ProductArgs a{};
    a.A = reinterpret_cast<const char *>(D);
    a.lda = 2 * l.Fp * kSize<T>;
    if (dX && T_ > 0) {           // D (T x 2 Fp) times (Wg; Wu)
        a.Kb = int(2 * l.Fp * kSize<T>);
        a.M = a.split = a.limit = T_;
        a.N = K;
        a.out = dX;
        a.ldo = lddx;
        a.out_bf16 = std::is_same<T, bf16>::value;
        if constexpr (columns) {
            const ColumnOperand g = as_columns(W.Wg, W.ldg, F, K, w_space, l.Kp, stream);
            const ColumnOperand u = as_columns(W.Wu, W.ldu, F, K, w_space + F * l.Kp * 2, l.Kp, stream);
            a.B0 = g.p;
            a.B1 = u.p;
            a.ldb0 = g.ld;
            a.ldb1 = u.ld;
            a.rows_k = int(F);
            a.half = int(l.Fp / 32);
        } else {
            a.B0 = w_space;
            a.ldb0 = a.lda;
        }
        gradient_product<T, T, false>(a, l.x_slices, sums, stream);
    }
    if (dWg && T_ > 0) {          // D^T (2 F x T) times X; with what D's rounding dropped, twice the terms
        a.N = K;
        a.out = dWg;
        a.out2 = dWu;
        a.ldo = lddw;
        a.limit = F;
        a.out_bf16 = std::is_same<TG, bf16>::value;
        if constexpr (columns) {
            const ColumnOperand x = as_columns(X, ldx, T_, K, x_space, l.Kp, stream);
            a.B0 = a.B1 = x.p;
            a.ldb0 = a.ldb1 = x.ld;
            a.rows_k = int(T_);
            a.half = cover(T_, 32);
            a.Kb = (dropped ? 2 : 1) * a.half * 64;
            a.A1 = dropped ? reinterpret_cast<const char *>(Dt) : a.A;
            a.M = 2 * l.Fp;
            a.split = l.Fp;
        } else {
            a.A = reinterpret_cast<const char *>(Dt);
            a.B0 = x_space;
            a.lda = a.ldb0 = l.Tp * kSize<T>;
            a.Kb = int(l.Tp * kSize<T>);
            a.M = 2 * F;
            a.split = F;
        }
        gradient_product<T, TG, columns>(a, l.w_slices, sums, stream);
    } else if (dWg) {
        for (void *p : {dWg, dWu})
            hipLaunchKernelGGL(zero_rows_kernel<TG>, dim3(grid_for(F * K, kThreads, 4096)),
                               dim3(kThreads), 0, as_stream(stream), static_cast<TG *>(p), F, K, lddw);
    }
}

}  // namespace

bsr_status launch_matmul_i8(const int8_t *Xq, int64_t T, int64_t K, int64_t ldx, const float *sx,
                            const int8_t *Wq, int64_t N, int64_t ldw, const float *sw,
                            const float *bias, void *Y, int y_dtype, int64_t ldy, void *stream) {
    ProductArgs a{};
    a.A = reinterpret_cast<const char *>(Xq);
    a.B0 = reinterpret_cast<const char *>(Wq);
    a.lda = ldx;
    a.ldb0 = ldw;
    a.M = T;
    a.N = N;
    a.Kb = int(K);
    a.sx = sx;
    a.s0 = sw;
    a.b0 = bias;
    a.out = Y;
    a.ldo = ldy;
    a.out_bf16 = y_dtype == BSR_BF16;
    launch_product<int8_t, Out::kScale>(a, stream);
    return launch_status();
}

bsr_status launch_gated(const void *X, int64_t T, int64_t ldx, const bsr_gated_t &W, void *H,
                        int64_t ldh, float *G, float *U, int64_t ldp, void *stream) {
    const int dt = raw_enum(W.dtype);
    const auto f = dt == BSR_BF16 ? gated<bf16> : gated<float>;
    f(X, T, ldx, nullptr, W, H, dt, ldh, G, U, ldp, stream);
    return launch_status();
}

bsr_status launch_gated_i8(const int8_t *Xq, int64_t T, int64_t ldx, const float *sx,
                           const bsr_gated_t &W, void *H, int h_dtype, int64_t ldh, void *stream) {
    gated<int8_t>(Xq, T, ldx, sx, W, H, h_dtype, ldh, nullptr, nullptr, 0, stream);
    return launch_status();
}

bsr_status launch_gated_backward(const void *dH, int64_t lddh, const void *X, int64_t T,
                                 int64_t ldx, const bsr_gated_t &W, const float *G,
                                 const float *U, int64_t ldp, void *dX, int64_t lddx, void *dWg,
                                 void *dWu, int64_t lddw, void *dbg, void *dbu, int grad_dtype,
                                 void *workspace, void *stream) {
    const bool b = raw_enum(W.dtype) == BSR_BF16, g = grad_dtype == BSR_BF16;
    const auto f = b ? (g ? backward<bf16, bf16> : backward<bf16, float>)
                     : (g ? backward<float, bf16> : backward<float, float>);
    f(dH, lddh, X, T, ldx, W, G, U, ldp, dX, lddx, dWg, dWu, lddw, dbg, dbu, workspace, stream);
    return launch_status();
}

}  // namespace bsr
