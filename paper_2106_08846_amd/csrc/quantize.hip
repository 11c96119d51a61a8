// Rows of a matrix in 8 bits: q = rint(x * (127 / max|x|)), scale = max|x| / 127, one row to a
// workgroup.  The maximum is taken over the bit patterns of |x| (order of the values, with NaN above
// infinity), so a NaN or an infinity anywhere in the row reaches its scale.
#include "dense_math.h"

namespace bsr {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ unsigned abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

template <class T>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(
    const T *__restrict__ X, int64_t K, int64_t ldx, int8_t *__restrict__ Q, int64_t ldq,
    float *__restrict__ scale) {
    const T *x = X + int64_t(blockIdx.x) * ldx;
    int8_t *q = Q + int64_t(blockIdx.x) * ldq;
    __shared__ unsigned smax[kThreads];
    unsigned top = 0;
    for (int64_t k = threadIdx.x; k < K; k += kThreads) top = max(top, abs_bits(to_float(x[k])));
    smax[threadIdx.x] = top;
    __syncthreads();
    for (int s = kThreads / 2; s > 0; s >>= 1) {
        if (int(threadIdx.x) < s) smax[threadIdx.x] = max(smax[threadIdx.x], smax[threadIdx.x + s]);
        __syncthreads();
    }
    const float a = __uint_as_float(smax[0]);
    const float lift = a < 0x1p-64f ? 0x1p64f : 1.0f;
    const float r = 127.0f / (a * lift);
    for (int64_t k = threadIdx.x; k < K; k += kThreads) {
        const float v = rintf((to_float(x[k]) * lift) * r);
        q[k] = v == v ? int8_t(v) : int8_t(0);
    }
    if (threadIdx.x == 0) scale[blockIdx.x] = a / 127.0f;
}

}  // namespace

bsr_status launch_quantize_rows(const void *X, int x_dtype, int64_t T, int64_t K, int64_t ldx,
                                int8_t *Q, int64_t ldq, float *scale, void *stream) {
    const dim3 grid(static_cast<unsigned>(T)), block(kThreads);
    if (x_dtype == BSR_BF16)
        hipLaunchKernelGGL(quantize_rows_kernel<bf16>, grid, block, 0, as_stream(stream),
                           static_cast<const bf16 *>(X), K, ldx, Q, ldq, scale);
    else
        hipLaunchKernelGGL(quantize_rows_kernel<float>, grid, block, 0, as_stream(stream),
                           static_cast<const float *>(X), K, ldx, Q, ldq, scale);
    return launch_status();
}

}  // namespace bsr
