// What the kernels of a policy's memory share: the functions of one value that they apply, and parts of rows.
#pragma once
#include "policy_device.h"

namespace bps {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// 1 / (1 + e^-x): 0 and 1 at the ends, where e^-x is infinite or nothing
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-x)); }
// d/dx of x sigmoid(x)
__device__ __forceinline__ float silu_slope(float x, float s) { return s * __builtin_fmaf(x, 1.0f - s, 1.0f); }

// ln(1 + e^v) = max(v, 0) + ln(1 + e) with e = e^-|v| <= 1, and ln(1 + e) = 2 artanh(s) with s = e / (2 + e) <= 1/3; artanh(s) / s is
// a polynomial in s^2 <= 1/9 whose coefficients were fitted for the least relative error there, 0.08 of half a step.  Small
// results keep their relative precision, which 1 + e would not: steps of a thousandth are usual.
__device__ __forceinline__ float softplus(float v) {
    const float e = exp_of(-__builtin_fabsf(v));
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
    float p = 0x1.1ed7c2p-3f;
    p = __builtin_fmaf(p, q, 0x1.1ebd0cp-3f);
    p = __builtin_fmaf(p, q, 0x1.99d208p-3f);
    p = __builtin_fmaf(p, q, 0x1.555502p-2f);
    p = __builtin_fmaf(p, q, 1.0f);
    return __builtin_fmaf(2.0f * s, p, fmaxf(v, 0.0f));
}

// Steps of sequence b
__device__ __forceinline__ int64_t steps_of(const int32_t* lengths, uint32_t b, uint32_t steps) {
    if (!lengths) return steps;
    const int32_t n = lengths[b];
    return n < 0 ? 0 : (uint32_t)n < steps ? n : steps;
}

// The first n of N elements (n = N: all of them, at once); the others read as zero and are not written.
template <class T, int N>
__device__ __forceinline__ void load_part(const typename T::raw* p, uint32_t n, float (&x)[N]) {
    if (n >= N) {
        load<T, N>(p, x);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = k < (int)n ? to_float(p[k]) : 0.0f;
    }
}
template <class T, int N>
__device__ __forceinline__ void store_part(typename T::raw* p, uint32_t n, const float (&x)[N]) {
    if (n >= N) {
        store<T, N>(p, x);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < (int)n) p[k] = rounded<T>(x[k]);
    }
}
// The same of a type known when the kernel runs: F32 where `wide`.
template <class T, int N>
__device__ __forceinline__ void load_weights(const void* p, uint64_t at, bool wide, uint32_t n, float (&x)[N]) {
    if (wide)
        load_part<F32, N>(static_cast<const float*>(p) + at, n, x);
    else
        load_part<T, N>(static_cast<const typename T::raw*>(p) + at, n, x);
}

// Where a lane's vector of N elements of a row lies: the last one begins earlier where the row ends inside it, so that it is loaded at
// once too, and only its elements from .. to are the lane's own.
struct Place {
    uint32_t at, from, to;
    template <int N>
    __device__ __forceinline__ static Place of(uint32_t c, uint32_t width) {
        constexpr uint32_t kAll = N;
        if (width < kAll) return {0, 0, c ? 0 : width};
        const uint32_t at = min(c, width - kAll);
        return {at, c < width ? c - at : 0, c < width ? kAll : 0};
    }
    // The same where c < width; `to` is the same for all lanes.
    template <int N>
    __device__ __forceinline__ static Place inside(uint32_t c, uint32_t width) {
        const uint32_t all = min(width, (uint32_t)N), at = min(c, width - all);
        return {at, c - at, all};
    }
    // The elements of others read as zero.
    template <int N>
    __device__ __forceinline__ void own(float (&x)[N]) const {
        if (from)
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = k < (int)from ? 0.0f : x[k];
    }
    // Only its own, for memory that is written in place; the others read as zero.
    template <class T, int N>
    __device__ __forceinline__ void load(const typename T::raw* row, float (&x)[N]) const {
        const typename T::raw* p = row + at;
        if (from == 0 && to == N) {
            bps::load<T, N>(p, x);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = k >= (int)from && k < (int)to ? to_float(p[k]) : 0.0f;
        }
    }
    template <class T, int N>
    __device__ __forceinline__ void store(typename T::raw* row, const float (&x)[N]) const { store_at<T, N>(row + at, x); }
    template <class T, int N>
    __device__ __forceinline__ void store_at(typename T::raw* p, const float (&x)[N]) const {
        if (from == 0 && to == N) {
            bps::store<T, N>(p, x);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k >= (int)from && k < (int)to) p[k] = rounded<T>(x[k]);
        }
    }
};
// Such a vector as it is in memory: several are loaded before the first is waited for, which conversions in the branches that load
// them would do.
template <class T, int N>
struct Part {
    static constexpr int kWords = N * sizeof(typename T::raw) / sizeof(Words);
    Words w[kWords] = {};
    __device__ __forceinline__ void load(const typename T::raw* row, const Place& place) {
        constexpr int kEach = N / kWords;
        const typename T::raw* p = row + place.at;
        if (place.to == N) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = load_words<T>(p + i * kEach);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = Words{};
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k < (int)place.to) {
                    if constexpr (sizeof(*p) == 4)
                        w[k / kEach][k % kEach] = __float_as_uint(to_float(p[k]));
                    else
                        w[k / kEach][k % kEach / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[k]) << (16 * (k % 2));
                }
        }
    }
    // Holds conversions back behind the loads before it.
    __device__ __forceinline__ void arrive() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) __asm__("" : "+v"(w[i]));
    }
    __device__ __forceinline__ void get(const Place& place, float (&x)[N]) const {
        constexpr int kEach = N / kWords;
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = word_float<T>(w[k / kEach], k % kEach);
        place.own(x);
    }
};

}  // namespace bps
