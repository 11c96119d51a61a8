// Layer norm with the residual sum before it, and its gradients.
//
// Memory bound: the forward pass reads X (and R) and writes Y (and S), the backward pass reads dY and S
// (and dS) and writes dX, each once; a row stays in registers between its sums and its outputs.  The mean is
// taken before the deviations: two sums in turn over registers cost nothing beside the loads, and a row far
// from zero keeps its variance.
//
// MI355X, 8192 x 4096 bf16 (268 MB in all) on inputs that no cache holds: forward with R and S 57 us (4.7
// TB/s), backward with dS and the join of the sums 60 (4.5 TB/s); on the same inputs again 40 and 48, partly
// from the memory-side cache.  A large copy moves 5.17 TB/s.  One row of 1024 fp32 takes 1.9 us, a memory
// latency, two sums over a wave and the two ends of a kernel.
#include "row_vec.h"

namespace bsr {

namespace {

struct NormArgs {
    const void *X, *R;
    const float *gamma, *beta;
    void *Y, *S;
    float *mean, *rstd;
    int64_t T, ldx, ldr, ldy, lds;
    int K;
    float eps;
};

// kVec values of a vector that may be missing.
template <int END>
__device__ __forceinline__ void load_or(const float *p, int k, int K, float other, float (&v)[kVec]) {
    if (p) {
        load_vec<float, END>(p, k, K, v);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = other;
    }
}

// The sum of v over a row's waves, in every lane; `at` is the row's own LDS, used once.
template <int WAVES> __device__ __forceinline__ float row_sum(float v, float *at) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += at[w];
    }
    return v;
}

// Whether element i of the vector at k is one of the row's K.  The sums ask: beyond the row's end a value
// reads as 0, which may be far from the row's mean.
template <int END> __device__ __forceinline__ bool in_row(int k, int i, int K) {
    return END == kWholeSteps || (END == kWholeVectors ? k < K : k + i < K);
}

constexpr int kHeld = 8;       // load steps of a row that the forward pass holds in registers

// WAVES waves per row, ROWS rows per workgroup, whose rows end as END says.  Rows
// longer than the registers hold are read again for the deviations and for the outputs.
template <class T, int WAVES, int ROWS, int END>
__global__ __launch_bounds__(64 * WAVES * ROWS) void norm_kernel(NormArgs a) {
    static_assert(WAVES == 1 || ROWS == 1, "one row per barrier");
    constexpr int kSpan = 64 * WAVES * kVec;
    __shared__ float red[2][WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = a.K;
    const int64_t row = int64_t(blockIdx.x) * ROWS + wave / WAVES;
    if (row >= a.T) return;                    // whole waves, and no barrier where ROWS > 1
    const T *x = static_cast<const T *>(a.X) + row * a.ldx;
    const T *r = a.R ? static_cast<const T *>(a.R) + row * a.ldr : nullptr;
    T *y = static_cast<T *>(a.Y) + row * a.ldy;
    T *sum_out = a.S ? static_cast<T *>(a.S) + row * a.lds : nullptr;
    const int k0 = (wave % WAVES * 64 + lane) * kVec;
    // S[k ..], rounded to the type.
    const auto load = [&](int k, float (&v)[kVec]) {
        load_vec<T, END>(x, k, K, v);
        if (r) {
            float w[kVec];
            load_vec<T, END>(r, k, K, w);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = to_float(from_float<T>(v[i] + w[i]));
        }
    };
    const auto squares = [&](int k, const float (&v)[kVec], float mean) {
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float d = in_row<END>(k, i, K) ? v[i] - mean : 0.0f;
            q = fmaf(d, d, q);
        }
        return q;
    };
    float v[kHeld][kVec];
#pragma unroll
    for (int s = 0; s < kHeld; ++s) {
        if (s * kSpan >= K) break;
        load(k0 + s * kSpan, v[s]);
    }
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < kHeld; ++s) {
        if (s * kSpan >= K) break;
        if (sum_out) write_vec<T, END, true>(sum_out, k0 + s * kSpan, K, v[s]);
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum += v[s][i];
    }
    for (int k = k0 + kHeld * kSpan; k < K; k += kSpan) {
        float w[kVec];
        load(k, w);
        if (sum_out) write_vec<T, END, true>(sum_out, k, K, w);
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum += w[i];
    }
    const float mean = row_sum<WAVES>(sum, red[0]) / float(K);
    float square = 0.0f;
#pragma unroll
    for (int s = 0; s < kHeld; ++s) {
        if (s * kSpan >= K) break;
        square += squares(k0 + s * kSpan, v[s], mean);
    }
    for (int k = k0 + kHeld * kSpan; k < K; k += kSpan) {
        float w[kVec];
        load(k, w);
        square += squares(k, w, mean);
    }
    const float rstd = 1.0f / sqrtf(row_sum<WAVES>(square, red[1]) / float(K) + a.eps);
    if (lane == 0 && wave % WAVES == 0 && a.mean) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
    const auto store = [&](int k, const float (&v)[kVec]) {
        float g[kVec], b[kVec], out[kVec];
        load_or<END>(a.gamma, k, K, 1.0f, g);
        load_or<END>(a.beta, k, K, 0.0f, b);
#pragma unroll
        for (int i = 0; i < kVec; ++i) out[i] = fmaf((v[i] - mean) * rstd, g[i], b[i]);
        write_vec<T, END, true>(y, k, K, out);
    };
#pragma unroll
    for (int s = 0; s < kHeld; ++s) {
        if (s * kSpan >= K) break;
        store(k0 + s * kSpan, v[s]);
    }
    for (int k = k0 + kHeld * kSpan; k < K; k += kSpan) {
        float w[kVec];
        load(k, w);
        store(k, w);
    }
}

constexpr int64_t kRowsPerLaunch = int64_t(1) << 21;     // a grid has under 2^32 threads

template <class T, int WAVES, int ROWS> void launch_norm(const NormArgs &args, void *stream) {
    const int end = row_end(args.K, 64 * WAVES * kVec);
    const auto kernel = end == kWholeSteps     ? norm_kernel<T, WAVES, ROWS, kWholeSteps>
                        : end == kWholeVectors ? norm_kernel<T, WAVES, ROWS, kWholeVectors>
                                               : norm_kernel<T, WAVES, ROWS, kAnyEnd>;
    for (int64_t t = 0; t < args.T; t += kRowsPerLaunch) {
        NormArgs a = args;
        a.T = args.T - t < kRowsPerLaunch ? args.T - t : kRowsPerLaunch;
        a.X = static_cast<const T *>(a.X) + t * a.ldx;
        if (a.R) a.R = static_cast<const T *>(a.R) + t * a.ldr;
        a.Y = static_cast<T *>(a.Y) + t * a.ldy;
        if (a.S) a.S = static_cast<T *>(a.S) + t * a.lds;
        if (a.mean) a.mean += t, a.rstd += t;
        hipLaunchKernelGGL(kernel, dim3(unsigned((a.T + ROWS - 1) / ROWS)), dim3(64 * WAVES * ROWS), 0,
                           as_stream(stream), a);
    }
}

template <class T> void norm(const NormArgs &a, void *stream) {
    constexpr int64_t held = 64 * kVec * kHeld;   // elements of a row that a wave holds
    // Few long rows on a wave each leave CUs idle: 777 x 1531 fp32 takes 5.8 us so and 5.2 on four.
    if (a.K <= 1024 || (a.K <= held && a.T >= 2048))
        launch_norm<T, 1, 4>(a, stream);
    else if (a.K <= 4 * held)
        launch_norm<T, 4, 1>(a, stream);
    else
        launch_norm<T, 16, 1>(a, stream);
}

// --- gradients ----------------------------------------------------------------------------------

struct NormGradArgs {
    const void *dY, *S, *dS;
    const float *gamma, *mean, *rstd;
    void *dX;
    float *partial;          // [groups][2][K], or NULL: neither dgamma nor dbeta
    int64_t T, lddy, lds, ldds, lddx;
    int K;
};

// Rows of up to 1024 WAVES columns: a workgroup takes ROWS rows side by side, WAVES waves each, kBatch times
// at once, and walks on over the rows with its columns' gamma, dgamma and dbeta in registers.
template <class T, int WAVES, int ROWS, int END>
__global__ __launch_bounds__(64 * WAVES * ROWS) void norm_backward_kernel(NormGradArgs a) {
    constexpr int kSteps = 2, kSpan = 64 * WAVES * kVec, kWidth = kSteps * kSpan;
    // Two rows of bf16 in flight; fp32 and sixteen waves have registers for one.  (fp32 rows on sixteen waves
    // that end off a load step keep two to five registers of a lane in memory all the same: 2000 x 5000 with dS
    // takes 42 us, 3.8 TB/s.)
    constexpr int kBatch = WAVES > 4 || sizeof(T) > 2 ? 1 : 2;
    __shared__ float red[2][2 * kBatch][ROWS][WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, K = a.K;
    const int place = wave / WAVES, part = wave % WAVES, k0 = (part * 64 + lane) * kVec;
    float gamma[kSteps][kVec], dgamma[kSteps][kVec] = {}, dbeta[kSteps][kVec] = {};
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
        if (s * kSpan < K) load_or<END>(a.gamma, k0 + s * kSpan, K, 1.0f, gamma[s]);
    int parity = 0;
    const int64_t stride = int64_t(gridDim.x) * ROWS;
    struct Batch {
        T d[kBatch][kSteps][kVec], x[kBatch][kSteps][kVec], more[kBatch][kSteps][kVec];
        float mean[kBatch], rstd[kBatch];
        bool in[kBatch];
    };
    const auto fetch = [&](int64_t base, Batch &to) {
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int64_t row = base + place + b * stride;
            to.in[b] = row < a.T;
            if (!to.in[b]) continue;
            to.mean[b] = a.mean[row];
            to.rstd[b] = a.rstd[row];
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if (s * kSpan >= K) break;
                const int k = k0 + s * kSpan;
                take_vec<T, END>(static_cast<const T *>(a.dY) + row * a.lddy, k, K, to.d[b][s]);
                take_vec<T, END>(static_cast<const T *>(a.S) + row * a.lds, k, K, to.x[b][s]);
                if (a.dS)
                    take_vec<T, END>(static_cast<const T *>(a.dS) + row * a.ldds, k, K, to.more[b][s]);
            }
        }
    };
    // The next rows are loaded before this round's sums are joined, where the registers hold them and no lane
    // asks for the end of its row: 8192 x 4096 bf16 with dS takes this kernel 49 us so and 55 without
    // (2048 x 8192 on sixteen waves 34 and 33).  Rows that end within a vector cost more than that: 777 x 1531
    // fp32 takes 11.4 us and 777 x 1528 8.4, on inputs that no cache holds.
    constexpr bool kAhead = END != kAnyEnd && WAVES <= 4;
    Batch next = {};
    if (kAhead) fetch(int64_t(blockIdx.x) * ROWS, next);
    // Every wave makes the same rounds, for their barriers.
    for (int64_t base = int64_t(blockIdx.x) * ROWS; base < a.T; base += kBatch * stride) {
        if (!kAhead) fetch(base, next);
        const Batch now = next;
        float c[2 * kBatch];
        if (kAhead) fetch(base + kBatch * stride, next);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            float c1 = 0.0f, c2 = 0.0f;
            if (now.in[b]) {
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    if (s * kSpan >= K) break;
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        const float dy = to_float(now.d[b][s][i]);
                        // beyond the row's end mean * rstd may be infinite, and 0 times it NaN
                        const float h = in_row<END>(k0 + s * kSpan, i, K)
                                            ? (to_float(now.x[b][s][i]) - now.mean[b]) * now.rstd[b]
                                            : 0.0f;
                        dgamma[s][i] = fmaf(dy, h, dgamma[s][i]);
                        dbeta[s][i] += dy;
                        const float g = dy * gamma[s][i];
                        c1 += g;
                        c2 = fmaf(g, h, c2);
                    }
                }
            }
            c[2 * b] = c1;
            c[2 * b + 1] = c2;
        }
        if (!a.dX) continue;
#pragma unroll
        for (int i = 0; i < 2 * kBatch; ++i) c[i] = wave_sum(c[i]);
        if constexpr (WAVES > 1) {
            // The other half is written for the next round, and this one again only after its barrier.
            if (lane == 0)
#pragma unroll
                for (int i = 0; i < 2 * kBatch; ++i) red[parity][i][place][part] = c[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2 * kBatch; ++i) {
                c[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) c[i] += red[parity][i][place][w];
            }
            parity ^= 1;
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (!now.in[b]) break;
            const float c1 = c[2 * b] / float(K), c2 = c[2 * b + 1] / float(K);
            T *dx = static_cast<T *>(a.dX) + (base + place + b * stride) * a.lddx;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if (s * kSpan >= K) break;
                float out[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float h = (to_float(now.x[b][s][i]) - now.mean[b]) * now.rstd[b];
                    out[i] = fmaf(to_float(now.d[b][s][i]) * gamma[s][i] - c1 - h * c2, now.rstd[b],
                                  to_float(now.more[b][s][i]));
                }
                write_vec<T, END>(dx, k0 + s * kSpan, K, out);
            }
        }
    }
    if (!a.partial) return;
    if constexpr (ROWS > 1) {                  // the upper half of the places to the lower, until one is left
        __shared__ __align__(16) float half[ROWS / 2][2][kWidth];
#pragma unroll
        for (int n = ROWS / 2; n > 0; n /= 2) {
            if (place >= n && place < 2 * n)
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    write_vec<float, kWholeSteps>(half[place - n][0], k0 + s * kSpan, kWidth, dgamma[s]);
                    write_vec<float, kWholeSteps>(half[place - n][1], k0 + s * kSpan, kWidth, dbeta[s]);
                }
            __syncthreads();
            if (place < n)
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    float g[kVec], e[kVec];
                    load_vec<float, kWholeSteps>(half[place][0], k0 + s * kSpan, kWidth, g);
                    load_vec<float, kWholeSteps>(half[place][1], k0 + s * kSpan, kWidth, e);
#pragma unroll
                    for (int i = 0; i < kVec; ++i) dgamma[s][i] += g[i], dbeta[s][i] += e[i];
                }
            __syncthreads();
        }
        if (place > 0) return;
    }
    float *to = a.partial + int64_t(blockIdx.x) * 2 * K;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        if (s * kSpan >= K) break;
        write_vec<float, END>(to, k0 + s * kSpan, K, dgamma[s]);
        write_vec<float, END>(to + K, k0 + s * kSpan, K, dbeta[s]);
    }
}

// Longer rows: dX by a workgroup per row, which reads its row twice, and the sums over the rows apart.
template <class T> __global__ __launch_bounds__(1024) void norm_dx_kernel(NormGradArgs a) {
    constexpr int kSpan = 1024 * kVec;
    __shared__ float red[2][2][16];
    const int K = a.K, k0 = threadIdx.x * kVec;
    int parity = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        const T *dy = static_cast<const T *>(a.dY) + row * a.lddy;
        const T *sum = static_cast<const T *>(a.S) + row * a.lds;
        const float mean = a.mean[row], rstd = a.rstd[row];
        const auto load = [&](int k, float (&g)[kVec], float (&h)[kVec]) {
            float w[kVec];
            load_vec<T, kAnyEnd>(dy, k, K, g);
            load_vec<T, kAnyEnd>(sum, k, K, h);
            load_or<kAnyEnd>(a.gamma, k, K, 1.0f, w);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                g[i] *= w[i];
                h[i] = (h[i] - mean) * rstd;
            }
        };
        float c1 = 0.0f, c2 = 0.0f, g[kVec], h[kVec];
        for (int k = k0; k < K; k += kSpan) {
            load(k, g, h);
#pragma unroll
            for (int i = 0; i < kVec; ++i) c1 += g[i], c2 = fmaf(g[i], in_row<kAnyEnd>(k, i, K) ? h[i] : 0.0f, c2);
        }
        c1 = row_sum<16>(c1, red[parity][0]) / float(K);
        c2 = row_sum<16>(c2, red[parity][1]) / float(K);
        parity ^= 1;
        T *dx = static_cast<T *>(a.dX) + row * a.lddx;
        for (int k = k0; k < K; k += kSpan) {
            float out[kVec], more[kVec] = {};
            load(k, g, h);
            if (a.dS) load_vec<T, kAnyEnd>(static_cast<const T *>(a.dS) + row * a.ldds, k, K, more);
#pragma unroll
            for (int i = 0; i < kVec; ++i) out[i] = fmaf(g[i] - c1 - h[i] * c2, rstd, more[i]);
            write_vec<T, kAnyEnd>(dx, k, K, out);
        }
    }
}
constexpr int kColumnThreads = 256, kColumns = kColumnThreads * kVec;
template <class T> __global__ __launch_bounds__(kColumnThreads) void norm_columns_kernel(NormGradArgs a) {
    const int K = a.K, k = int(blockIdx.x) * kColumns + threadIdx.x * kVec;
    if (k >= K) return;
    float dgamma[kVec] = {}, dbeta[kVec] = {};
    for (int64_t row = blockIdx.y; row < a.T; row += gridDim.y) {
        float d[kVec], h[kVec];
        load_vec<T, kAnyEnd>(static_cast<const T *>(a.dY) + row * a.lddy, k, K, d);
        load_vec<T, kAnyEnd>(static_cast<const T *>(a.S) + row * a.lds, k, K, h);
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            dgamma[i] = fmaf(d[i], (h[i] - mean) * rstd, dgamma[i]);
            dbeta[i] += d[i];
        }
    }
    float *to = a.partial + int64_t(blockIdx.y) * 2 * K;
    write_vec<float, kAnyEnd>(to, k, K, dgamma);
    write_vec<float, kAnyEnd>(to + K, k, K, dbeta);
}

// The groups' sums joined, in an order fixed by their number: 32 columns to a workgroup, whose half-waves
// take every 32nd group each, eight loads at a time.
constexpr int kJoinWaves = 16, kJoinColumns = 32, kJoinParts = 64 / kJoinColumns * kJoinWaves;
template <class G>
__global__ __launch_bounds__(64 * kJoinWaves) void norm_join_kernel(const float *partial, int groups, int K,
                                                                    G *dgamma, G *dbeta) {
    __shared__ float parts[kJoinParts][kJoinColumns];
    const int column = threadIdx.x % kJoinColumns, part = threadIdx.x / kJoinColumns;
    const int64_t at = int64_t(blockIdx.x) * kJoinColumns + column, width = 2 * int64_t(K);
    float sum = 0.0f;
    if (at < width) {
        int g = part;
        for (; g + 7 * kJoinParts < groups; g += 8 * kJoinParts) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = partial[(g + i * kJoinParts) * width + at];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
        for (; g < groups; g += kJoinParts) sum += partial[g * width + at];
    }
    parts[part][column] = sum;
    __syncthreads();
    if (part > 0 || at >= width) return;
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinParts; ++w) sum += parts[w][column];
    G *to = at < K ? dgamma : dbeta;
    if (to) to[at < K ? at : at - K] = from_float<G>(sum);
}

template <class T, int WAVES, int ROWS> void launch_backward(const NormGradArgs &a, int groups, void *stream) {
    const int end = row_end(a.K, 64 * WAVES * kVec);
    const auto kernel = end == kWholeSteps     ? norm_backward_kernel<T, WAVES, ROWS, kWholeSteps>
                        : end == kWholeVectors ? norm_backward_kernel<T, WAVES, ROWS, kWholeVectors>
                                               : norm_backward_kernel<T, WAVES, ROWS, kAnyEnd>;
    hipLaunchKernelGGL(kernel, dim3(unsigned(groups)), dim3(64 * WAVES * ROWS), 0, as_stream(stream), a);
}

template <class T> void norm_backward(const NormGradArgs &a, int groups, void *stream) {
    if (a.K <= kNormFusedWidth) {
        switch (norm_row_waves(a.K)) {
            case 1: return launch_backward<T, 1, kNormPlaces[0]>(a, groups, stream);
            case 4: return launch_backward<T, 4, kNormPlaces[1]>(a, groups, stream);
            default: return launch_backward<T, 16, kNormPlaces[2]>(a, groups, stream);
        }
    }
    if (a.dX)
        hipLaunchKernelGGL(norm_dx_kernel<T>, dim3(grid_for(a.T, 1, 1 << 16)), dim3(1024), 0,
                           as_stream(stream), a);
    if (a.partial)
        hipLaunchKernelGGL(norm_columns_kernel<T>,
                           dim3(unsigned((a.K + kColumns - 1) / kColumns), unsigned(groups)),
                           dim3(kColumnThreads), 0, as_stream(stream), a);
}

template <class G>
void join(const float *partial, int groups, int64_t K, void *dgamma, void *dbeta, void *stream) {
    hipLaunchKernelGGL(norm_join_kernel<G>, dim3(unsigned((2 * K + kJoinColumns - 1) / kJoinColumns)),
                       dim3(64 * kJoinWaves), 0,
                       as_stream(stream), partial, groups, int(K), static_cast<G *>(dgamma),
                       static_cast<G *>(dbeta));
}

}  // namespace

bsr_status launch_layer_norm(const void *X, int64_t ldx, const void *R, int64_t ldr, int64_t T, int64_t K,
                             int dtype, const float *gamma, const float *beta, float eps, void *Y,
                             int64_t ldy, void *S, int64_t lds, float *mean, float *rstd, void *stream) {
    const NormArgs a{X, R, gamma, beta, Y, S, mean, rstd, T, ldx, ldr, ldy, lds, int(K), eps};
    dtype == BSR_BF16 ? norm<bf16>(a, stream) : norm<float>(a, stream);
    return launch_status();
}

bsr_status launch_layer_norm_backward(const void *dY, int64_t lddy, const void *S, int64_t lds, int64_t T,
                                      int64_t K, int dtype, const float *gamma, const float *mean,
                                      const float *rstd, const void *dS, int64_t ldds, void *dX,
                                      int64_t lddx, void *dgamma, void *dbeta, int grad_dtype,
                                      void *workspace, void *stream) {
    const bool vectors = dgamma || dbeta;
    const int groups = layer_norm_workspace(T, K).groups;
    const NormGradArgs a{dY, S, dS, gamma, mean, rstd, dX, vectors ? static_cast<float *>(workspace) : nullptr,
                         T, lddy, lds, ldds, lddx, int(K)};
    if (T > 0) (dtype == BSR_BF16 ? norm_backward<bf16> : norm_backward<float>)(a, groups, stream);
    if (vectors)
        (grad_dtype == BSR_BF16 ? join<bf16> : join<float>)(a.partial, groups, K, dgamma, dbeta, stream);
    return launch_status();
}

}  // namespace bsr
