// Rows of a matrix, eight elements at a time per lane, and sums over a wave.
#pragma once

#include "dense_math.h"

namespace bsr {

constexpr int kVec = 8;        // elements per lane and load step

__device__ __forceinline__ unsigned abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// How a row of K elements ends within a wave's load steps: at any element, at the end of a load step (no
// lane checks for the end), or at the end of a lane's kVec elements.
constexpr int kAnyEnd = 0, kWholeSteps = 1, kWholeVectors = 2;

// kVec elements from x[k] on; those from K on are 0.
template <class T, int END> __device__ __forceinline__ void take_vec(const T *x, int k, int K, T (&v)[kVec]) {
    if (END == kWholeSteps || (END == kWholeVectors ? k < K : k + kVec <= K)) {
        __builtin_memcpy(v, x + k, sizeof v);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = T{};
        if (END == kAnyEnd && k < K)           // lanes past the row's end skip this together
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (k + i < K) v[i] = x[k + i];
    }
}
// The same as fp32.
template <class T, int END> __device__ __forceinline__ void load_vec(const T *x, int k, int K, float (&v)[kVec]) {
    T raw[kVec];
    take_vec<T, END>(x, k, K, raw);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = to_float(raw[i]);
}
// The bytes of v at p (any alignment), past the caches: a stream of outputs otherwise drives the inputs that
// are still to be read out of them (8-bit codes of 8192 x 4096 bf16 take 23.4 us through them, 19.7 past).
template <class V> __device__ __forceinline__ void stream_out(void *p, const V &v) {
    constexpr int kWords = sizeof(V) / 4 < 4 ? sizeof(V) / 4 : 4;
    typedef unsigned Words __attribute__((ext_vector_type(kWords), aligned(1)));
#pragma unroll
    for (unsigned i = 0; i < sizeof(V) / sizeof(Words); ++i) {
        Words w;
        __builtin_memcpy(&w, reinterpret_cast<const char *>(&v) + i * sizeof w, sizeof w);
        __builtin_nontemporal_store(w, static_cast<Words *>(p) + i);
    }
}

// Written, rounded to the type; PAST: past the caches, 16 bytes a lane, where that is all the lane writes (two
// such halves of an fp32 vector leave partial lines: norm of 4096 x 1024 fp32 15.7 us, 17.8 past them).
template <class T, int END, bool PAST = false>
__device__ __forceinline__ void write_vec(T *y, int k, int K, const float (&v)[kVec]) {
    T raw[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) raw[i] = from_float<T>(v[i]);
    if (END == kWholeSteps || k + kVec <= K) {
        if constexpr (PAST && sizeof raw == 16)
            stream_out(y + k, raw);
        else
            __builtin_memcpy(y + k, raw, sizeof raw);
    } else if (END == kAnyEnd && k < K) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (k + i < K) y[k + i] = raw[i];
    }
}
// How rows of K elements end in load steps of `span`.
inline int row_end(int64_t K, int64_t span) {
    return K % span == 0 ? kWholeSteps : K % kVec == 0 ? kWholeVectors : kAnyEnd;
}

// v of the lane that DPP control CTRL names, which stays within a row of 16 lanes.
template <int CTRL> __device__ __forceinline__ unsigned dpp(unsigned v) {
    return unsigned(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
// Lane I of each quad, or of each row of 16.
template <int I, class T> __device__ __forceinline__ T quad_lane(T v) { return dpp<I * 0x55>(v); }
template <int I, class T> __device__ __forceinline__ T row_lane(T v) { return dpp<0x150 + I>(v); }
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

// The largest of the four lanes that are a multiple of 16 apart, in every one of them.
__device__ __forceinline__ unsigned column_max(unsigned v) {
    const auto half = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(unsigned(half[0]), unsigned(half[1]));
    const auto row = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return max(unsigned(row[0]), unsigned(row[1]));
}

}  // namespace bsr
