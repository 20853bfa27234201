// What the kernels of a policy's operators share: element types, loads of 16 bytes, what lanes of a wavefront
// exchange.
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
// The same as they lie in memory, for loads that are to be on their way before the first value is converted.
typedef uint32_t Words __attribute__((ext_vector_type(4)));
typedef Words WordsAnywhere __attribute__((aligned(2)));
template <class T>
__device__ __forceinline__ Words load_words(const typename T::raw* p) { return *reinterpret_cast<const WordsAnywhere*>(p); }
template <class T>
__device__ __forceinline__ float word_float(const Words& w, int k) {
    if constexpr (sizeof(typename T::raw) == 4)
        return __uint_as_float(w[k]);
    else
        return to_float(__builtin_bit_cast(typename T::raw, (uint16_t)(w[k / 2] >> (16 * (k % 2)))));
}
template <class T, int N>
__device__ __forceinline__ void store(typename T::raw* p, const float (&x)[N]) {
    Pack<typename T::raw, N> q;
#pragma unroll
    for (int k = 0; k < N; ++k) q.v[k] = rounded<T>(x[k]);
    *reinterpret_cast<Pack<typename T::raw, N>*>(p) = q;
}

// The same past the caches, for results that are larger than the last one of them (see past_caches).
template <class T, int N>
__device__ __forceinline__ void store_past(typename T::raw* p, const float (&x)[N]) {
    constexpr int kWords = N * (int)sizeof(typename T::raw) / 4;
    if constexpr (kWords == 4 || kWords == 2) {
        typedef uint32_t words __attribute__((ext_vector_type(kWords)));
        typedef words placed __attribute__((aligned(sizeof(typename T::raw))));
        Pack<typename T::raw, N> q;
#pragma unroll
        for (int k = 0; k < N; ++k) q.v[k] = rounded<T>(x[k]);
        __builtin_nontemporal_store(__builtin_bit_cast(words, q), reinterpret_cast<placed*>(p));
    } else {
        store<T, N>(p, x);
    }
}

template <class T, int N>
__device__ __forceinline__ void store(typename T::raw* p, const float (&x)[N], bool past) {
    if (past)
        store_past<T, N>(p, x);
    else
        store<T, N>(p, x);
}

// Whether results of `rows` rows are better written past the caches: where they do not fit the Infinity Cache
// (256 MiB), so that inputs may stay there, and all rows begin at whole cache lines, since parts of lines are
// not joined on the way.  Measured, through / past the caches: gradient of 8192 x 131072 bf16 logits 826 / 780
// us, and the pass before it, which then finds some of the logits, 405 / 371; 262144 rows of 2048 bf16 332 /
// 312; 50257 rows of 769 float32 (not whole lines) 31 / 45; state of 1.2e8 parameters as float32 251 / 270
// (there it stays as it was).
inline bool past_caches(const void* p, int64_t stride, size_t size, uint64_t rows, uint64_t width) {
    return rows * width * size > 256u << 20 && (reinterpret_cast<uintptr_t>(p) % 128) == 0 && stride * (int64_t)size % 128 == 0;
}

__device__ __forceinline__ int64_t token_at(const void* tokens, int tokens64, uint64_t i) {
    return tokens64 ? static_cast<const int64_t*>(tokens)[i] : (int64_t) static_cast<const int32_t*>(tokens)[i];
}

// The value of lane (lane ^ X): a permutation within 16 lanes where there is one, through the LDS crossbar otherwise.
template <int X>
__device__ __forceinline__ uint32_t from_lane_xor(uint32_t v) {
    static_assert(X > 0 && X < 64, "within the wavefront");
    if constexpr (X == 1) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);          // quad_perm 1 0 3 2
    else if constexpr (X == 2) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);     // quad_perm 2 3 0 1
    else if constexpr (X == 3) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x1B, 0xF, 0xF, true);     // quad_perm 3 2 1 0
    else if constexpr (X == 7) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true);    // mirrored within 8
    else if constexpr (X == 8) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true);    // rotated by 8 within 16
    else if constexpr (X == 15) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true);   // mirrored within 16
    else if constexpr (X == 4) return from_lane_xor<7>(from_lane_xor<3>(v));
    else if constexpr (X < 32) return (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, (X << 10) | 0x1F);
    else return (uint32_t)__shfl_xor((int)v, X, 64);
}
template <int X>
__device__ __forceinline__ float from_lane_xor(float v) { return __uint_as_float(from_lane_xor<X>(__float_as_uint(v))); }
template <int X>
__device__ __forceinline__ uint64_t from_lane_xor(uint64_t v) {
    return (uint64_t)from_lane_xor<X>((uint32_t)(v >> 32)) << 32 | from_lane_xor<X>((uint32_t)v);
}

__device__ __forceinline__ uint32_t lanes_before(uint64_t lanes) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0u));
}

// f(x, value of x in the other lane) over all G lanes of a group
template <int G, class X, class F>
__device__ __forceinline__ X group_reduce(X x, F f) {
    if constexpr (G > 1) x = f(x, from_lane_xor<1>(x));
    if constexpr (G > 2) x = f(x, from_lane_xor<2>(x));
    if constexpr (G > 4) x = f(x, from_lane_xor<4>(x));
    if constexpr (G > 8) x = f(x, from_lane_xor<8>(x));
    if constexpr (G > 16) x = f(x, from_lane_xor<16>(x));
    if constexpr (G > 32) x = f(x, from_lane_xor<32>(x));
    return x;
}

}  // namespace bps
