// Rows of a matrix in 8 bits: q = rint(x * (127 / max|x|)), scale = max|x| / 127.
//
// Memory bound: every element is read once and one byte is written for it.  A row belongs to 1, 4 or
// 16 waves, whichever is the first to hold it in registers (4096 elements a wave), so that the
// maximum and the quotients come from one read; longer rows are read again for the quotients (from
// the L2, mostly).  The maximum is taken over the bit patterns of |x| (order of the values, with NaN
// above infinity), so a NaN or an infinity anywhere in the row reaches its scale.
// 8192 rows of 4096 bf16 take 16.5 us (MI355X), 6.1 TB/s over both directions; a single row of 1024
// takes 1.8 us, a memory latency and the two ends of a kernel.
#include "dense_math.h"

namespace bsr {

namespace {

constexpr int kVec = 8;        // elements per lane and load step
constexpr int kHeld = 8;       // load steps held in registers

__device__ __forceinline__ unsigned abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// kVec elements from x[k] on, as fp32; those from K on are 0.  WHOLE: there are none from K on.
template <class T, bool WHOLE>
__device__ __forceinline__ void load_vec(const T *x, int k, int K, float (&v)[kVec]) {
    if (WHOLE || k + kVec <= K) {
        T raw[kVec];
        __builtin_memcpy(raw, x + k, sizeof raw);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = to_float(raw[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = k + i < K ? to_float(x[k + i]) : 0.0f;
    }
}

template <bool WHOLE>
__device__ __forceinline__ void store_vec(int8_t *q, int k, int K, const float (&v)[kVec],
                                          float lift, float r) {
    int8_t b[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) b[i] = int8_t(int(rintf((v[i] * lift) * r)));
    if (WHOLE || k + kVec <= K) {
        __builtin_memcpy(q + k, b, kVec);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (k + i < K) q[k + i] = b[i];
    }
}

// WAVES waves per row, ROWS rows per workgroup.  WHOLE: K is a multiple of a load step's 64 * WAVES *
// kVec elements, so that no lane checks for the end of the row.
template <class T, int WAVES, int ROWS, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES * ROWS) void quantize_rows_kernel(
    const T *__restrict__ X, int64_t T_, int K, int64_t ldx, int8_t *__restrict__ Q, int64_t ldq,
    float *__restrict__ scale) {
    static_assert(WAVES == 1 || ROWS == 1, "one row per barrier");
    constexpr int kSpan = 64 * WAVES * kVec;   // elements per load step of a row
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = int64_t(blockIdx.x) * ROWS + wave / WAVES;
    if (row >= T_) return;                     // whole waves, and no barrier where ROWS > 1
    const T *x = X + row * ldx;
    int8_t *q = Q + row * ldq;
    const int k0 = (wave % WAVES * 64 + lane) * kVec;
    float v[kHeld][kVec];
    unsigned top = 0;
#pragma unroll
    for (int s = 0; s < kHeld; ++s) {
        if (s * kSpan >= K) break;
        load_vec<T, WHOLE>(x, k0 + s * kSpan, K, v[s]);
    }
#pragma unroll
    for (int s = 0; s < kHeld; ++s) {
        if (s * kSpan >= K) break;
#pragma unroll
        for (int i = 0; i < kVec; ++i) top = max(top, abs_bits(v[s][i]));
    }
    for (int k = kHeld * kSpan; k < K; k += kSpan) {
        float w[kVec];
        load_vec<T, WHOLE>(x, k0 + k, K, w);
#pragma unroll
        for (int i = 0; i < kVec; ++i) top = max(top, abs_bits(w[i]));
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = max(top, unsigned(__shfl_xor(int(top), d)));
    if constexpr (WAVES > 1) {
        __shared__ unsigned smax[WAVES];
        if (lane == 0) smax[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = max(top, smax[w]);
    }
    const float a = __uint_as_float(top);
    if (lane == 0 && wave % WAVES == 0) scale[row] = a / 127.0f;
    // Rows of zeros, or with an infinity or a NaN: every q is 0 (as rint(NaN) -> 0 and rint(0) give).
    const bool plain = top > 0 && top < 0x7f800000u;
    const float lift = a < 0x1p-64f ? 0x1p64f : 1.0f;
    const float r = plain ? 127.0f / (a * lift) : 0.0f;
    if (!plain) {
        for (int k = k0; k < K; k += kSpan)
            for (int i = 0; i < kVec; ++i)
                if (k + i < K) q[k + i] = 0;
        return;
    }
#pragma unroll
    for (int s = 0; s < kHeld; ++s) {
        if (s * kSpan >= K) break;
        store_vec<WHOLE>(q, k0 + s * kSpan, K, v[s], lift, r);
    }
    for (int k = kHeld * kSpan; k < K; k += kSpan) {
        float w[kVec];
        load_vec<T, WHOLE>(x, k0 + k, K, w);
        store_vec<WHOLE>(q, k0 + k, K, w, lift, r);
    }
}

template <class T, int WAVES, int ROWS>
void launch(const T *X, int64_t T_, int64_t K, int64_t ldx, int8_t *Q, int64_t ldq, float *scale,
            void *stream) {
    const auto kernel = K % (64 * WAVES * kVec) == 0 ? quantize_rows_kernel<T, WAVES, ROWS, true>
                                                     : quantize_rows_kernel<T, WAVES, ROWS, false>;
    constexpr int64_t most = int64_t(1) << 21;     // rows of a launch: a grid has under 2^32 threads
    for (int64_t t = 0; t < T_; t += most) {
        const int64_t n = T_ - t < most ? T_ - t : most;
        hipLaunchKernelGGL(kernel, dim3(unsigned((n + ROWS - 1) / ROWS)), dim3(64 * WAVES * ROWS), 0,
                           as_stream(stream), X + t * ldx, n, int(K), ldx, Q + t * ldq, ldq, scale + t);
    }
}

template <class T>
void quantize(const void *X, int64_t T_, int64_t K, int64_t ldx, int8_t *Q, int64_t ldq,
              float *scale, void *stream) {
    const T *x = static_cast<const T *>(X);
    constexpr int64_t held = 64 * kVec * kHeld;   // elements of a row that a wave holds
    if (K <= held)
        launch<T, 1, 4>(x, T_, K, ldx, Q, ldq, scale, stream);
    else if (K <= 4 * held)
        launch<T, 4, 1>(x, T_, K, ldx, Q, ldq, scale, stream);
    else
        launch<T, 16, 1>(x, T_, K, ldx, Q, ldq, scale, stream);
}

}  // namespace

bsr_status launch_quantize_rows(const void *X, int x_dtype, int64_t T, int64_t K, int64_t ldx,
                                int8_t *Q, int64_t ldq, float *scale, void *stream) {
    const auto f = x_dtype == BSR_BF16 ? quantize<bf16> : quantize<float>;
    f(X, T, K, ldx, Q, ldq, scale, stream);
    return launch_status();
}

}  // namespace bsr
