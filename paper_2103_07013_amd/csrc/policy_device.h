// What the kernels of a policy's operators share: element types, loads of 16 bytes, sums over a wavefront.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bps {

struct F32 {
    using raw = float;
    static constexpr int kPer16 = 4;
};
struct Bf16 {
    using raw = uint16_t;
    static constexpr int kPer16 = 8;
};
struct F16 {
    using raw = _Float16;
    static constexpr int kPer16 = 8;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(_Float16 x) { return (float)x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

template <class T>
__device__ __forceinline__ typename T::raw rounded(float x);
template <>
__device__ __forceinline__ float rounded<F32>(float x) { return x; }
template <>
__device__ __forceinline__ _Float16 rounded<F16>(float x) { return (_Float16)x; }
// to nearest, ties to even; NaN stays NaN
template <>
__device__ __forceinline__ uint16_t rounded<Bf16>(float x) {
    __bf16 b = (__bf16)x;
    return __builtin_bit_cast(uint16_t, b);
}

// N elements that lie anywhere: rows of odd widths start at any element.  Global loads and stores of gfx950 take any
// alignment, so these are single instructions of up to 16 bytes.
template <class Raw, int N>
struct __attribute__((packed, aligned(sizeof(Raw)))) Pack {
    Raw v[N];
};

template <class T, int N>
__device__ __forceinline__ void load(const typename T::raw* p, float (&x)[N]) {
    const Pack<typename T::raw, N> q = *reinterpret_cast<const Pack<typename T::raw, N>*>(p);
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = to_float(q.v[k]);
}
template <class T, int N>
__device__ __forceinline__ void store(typename T::raw* p, const float (&x)[N]) {
    Pack<typename T::raw, N> q;
#pragma unroll
    for (int k = 0; k < N; ++k) q.v[k] = rounded<T>(x[k]);
    *reinterpret_cast<Pack<typename T::raw, N>*>(p) = q;
}

__device__ __forceinline__ int64_t token_at(const void* tokens, int tokens64, uint64_t i) {
    return tokens64 ? static_cast<const int64_t*>(tokens)[i] : (int64_t) static_cast<const int32_t*>(tokens)[i];
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}

}  // namespace bps
