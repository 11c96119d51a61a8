// Rows of a matrix, eight elements at a time per lane, and sums over a wave.
#pragma once

#include "dense_math.h"

namespace bsr {

constexpr int kVec = 8;        // elements per lane and load step

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

// The same elements written, rounded to the type.
template <class T, bool WHOLE>
__device__ __forceinline__ void write_vec(T *y, int k, int K, const float (&v)[kVec]) {
    T raw[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) raw[i] = from_float<T>(v[i]);
    if (WHOLE || k + kVec <= K) {
        __builtin_memcpy(y + k, raw, sizeof raw);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (k + i < K) y[k + i] = raw[i];
    }
}

// v of the lane that DPP control CTRL names, which stays within a row of 16 lanes.
template <int CTRL> __device__ __forceinline__ unsigned dpp(unsigned v) {
    return unsigned(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140;

// The sum over a wave, in every lane: pairs, quads, halves and rows of 16 lanes by DPP, then the four
// rows (a wave's sum by six LDS permutes takes four times as long).
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp<kSwap1>(v);
    v += dpp<kSwap2>(v);
    v += dpp<kMirror8>(v);
    v += dpp<kMirror16>(v);
    const int bits = __builtin_bit_cast(int, v);
    const auto row = [&](int lane) {
        return __builtin_bit_cast(float, __builtin_amdgcn_readlane(bits, lane));
    };
    return (row(0) + row(16)) + (row(32) + row(48));
}

// The largest of each row of 16 lanes, in every one of them.
__device__ __forceinline__ unsigned row_max(unsigned v) {
    v = max(v, dpp<kSwap1>(v));
    v = max(v, dpp<kSwap2>(v));
    v = max(v, dpp<kMirror8>(v));
    return max(v, dpp<kMirror16>(v));
}

}  // namespace bsr
