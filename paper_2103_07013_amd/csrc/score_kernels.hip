// Log probabilities of given tokens, with entropy and best alternatives, and their gradient.
//
//   y = scale x over the entries that take part (allowed by the mask, x > -inf);  m = max x
//   z = sum e^(scale (x - m)),  s = sum e^(scale (x - m)) scale (x - m)
//   lse = scale m + ln z,  logp = scale (x_t - m) - ln z,  entropy = ln z - s / z
//   d logp / dx_j = scale (d_jt - p_j),  d entropy / dx_j = -scale p_j (ln p_j + entropy)
//
// All sums are held in float32.  Exponents are taken to the base 2.
#include "policy_device.h"
#include "policy_kernels.h"

namespace bps {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;
// stands for differences below it where they are multiplied by a probability that is zero
constexpr float kFar = -1e30f;
constexpr float kInf = __builtin_inff();

// A part of a row: the largest entry, the sum of 2^d and of d 2^d, d = (x - m) scale log2 e.  m starts at the lowest
// finite value, so that entries of -inf are told from entries of that value.
struct Part {
    float m, z, s;
};
__device__ __forceinline__ Part nothing() { return {kLowest, 0.0f, 0.0f}; }

__device__ __forceinline__ Part joined(const Part& a, const Part& b, float c) {
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf((a.m - m) * c, kFar), db = fmaxf((b.m - m) * c, kFar);
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    return {m, fmaf(fa, a.z, fb * b.z), fa * fmaf(da, a.z, a.s) + fb * fmaf(db, b.z, b.s)};
}

template <int N>
__device__ __forceinline__ void add(Part& p, const float (&x)[N], float c) {
    float m = p.m;
#pragma unroll
    for (int k = 0; k < N; ++k) m = fmaxf(m, x[k]);
    if (m > p.m) {
        const float d = fmaxf((p.m - m) * c, kFar), f = __builtin_amdgcn_exp2f(d);
        p.s = f * fmaf(d, p.z, p.s);
        p.z *= f;
        p.m = m;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float d = (x[k] - m) * c, e = __builtin_amdgcn_exp2f(d);
        p.z += e;
        p.s = fmaf(e, fmaxf(d, kFar), p.s);
    }
}

// N entries of a row from `at` on; what is masked or behind the row's end is -inf.
template <class T, int N, bool MASK>
__device__ __forceinline__ void row_entries(const typename T::raw* row, const uint8_t* mask, uint32_t at, uint32_t end, float (&x)[N]) {
    if (at + N <= end) {
        load<T, N>(row + at, x);
        if (MASK) {
            const Pack<uint8_t, N> q = *reinterpret_cast<const Pack<uint8_t, N>*>(mask + at);
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = q.v[k] ? x[k] : -kInf;
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = at + k < end && (!MASK || mask[at + k]) ? to_float(row[at + k]) : -kInf;
    }
}

// What decides the order of alternatives: the entry as a number that grows with it (NaN above all, -0 as 0), then
// the lower index.  No entry that takes part has the number 0.
__device__ __forceinline__ uint64_t order_of(float x, uint32_t at) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t up = x != x ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return (uint64_t)up << 32 | (uint32_t)~at;
}

template <class T, bool MASK>
__global__ __launch_bounds__(256) void k_score(ScoreArgs a) {
    constexpr int N = T::kPer16;
    __shared__ Part parts[4];
    __shared__ uint64_t best[4];
    const uint32_t tid = threadIdx.x, wave = tid >> 6, lane = tid & 63u;
    const float c = a.scale * kLog2e;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const typename T::raw* row = static_cast<const typename T::raw*>(a.logits) + (int64_t)r * a.row_stride;
        const uint8_t* mask = MASK ? a.mask + (int64_t)r * a.mask_stride : nullptr;
        Part p = nothing();
        for (uint32_t at = tid * N; at < a.entries; at += 256 * N) {
            float x[N];
            row_entries<T, N, MASK>(row, mask, at, a.entries, x);
            add(p, x, c);
        }
        for (int d = 32; d; d >>= 1) p = joined(p, {__shfl_xor(p.m, d, 64), __shfl_xor(p.z, d, 64), __shfl_xor(p.s, d, 64)}, c);
        __syncthreads();
        if (lane == 0) parts[wave] = p;
        __syncthreads();
        p = joined(joined(parts[0], parts[1], c), joined(parts[2], parts[3], c), c);
        const float ln_z = logf(p.z);
        if (tid == 0) {
            const bool empty = p.z == 0.0f;
            a.norm[2 * r] = p.m;
            a.norm[2 * r + 1] = ln_z;
            a.lse[r] = empty ? -kInf : fmaf(a.scale, p.m, ln_z);
            a.entropy[r] = empty ? 0.0f : ln_z - kLn2 * (p.s / p.z);
            const int64_t t = token_at(a.tokens, a.tokens64, r);
            float lp = 0.0f;
            if (t < -1 || t >= (int64_t)a.entries) {
                lp = __builtin_nanf("");
            } else if (t >= 0) {
                const float x = !MASK || mask[t] ? to_float(row[t]) : -kInf;
                lp = empty ? -kInf : fmaf(x - p.m, a.scale, -ln_z);
            }
            a.logp[r] = lp;
        }
        uint64_t below = ~0ull;
        for (uint32_t k = 0; k < a.top_k; ++k) {
            uint64_t b = 0;
            for (uint32_t at = tid; at < a.entries; at += 256) {
                const float x = !MASK || mask[at] ? to_float(row[at]) : -kInf;
                const uint64_t o = order_of(x, at);
                if (x != -kInf && o < below && o > b) b = o;
            }
            for (int d = 32; d; d >>= 1) {
                const uint64_t o = __shfl_xor((unsigned long long)b, d, 64);
                b = o > b ? o : b;
            }
            __syncthreads();
            if (lane == 0) best[wave] = b;
            __syncthreads();
            for (int w = 0; w < 4; ++w) b = best[w] > b ? best[w] : b;
            if (tid == 0) {
                const uint64_t to = r * a.top_k + k;
                const uint32_t at = ~(uint32_t)b;
                a.top_ids[to] = b ? (int32_t)at : -1;
                a.top_logp[to] = b ? fmaf(to_float(row[at]) - p.m, a.scale, -ln_z) : -kInf;
            }
            below = b;
        }
    }
}

template <class T, bool MASK>
__global__ __launch_bounds__(256) void k_score_grad(ScoreGradArgs a) {
    constexpr int N = T::kPer16;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const typename T::raw* row = static_cast<const typename T::raw*>(a.logits) + (int64_t)r * a.row_stride;
        const uint8_t* mask = MASK ? a.mask + (int64_t)r * a.mask_stride : nullptr;
        typename T::raw* out = static_cast<typename T::raw*>(a.out) + (int64_t)r * a.out_stride;
        const float m = a.norm[2 * r], ln_z = a.norm[2 * r + 1], entropy = a.entropy[r], logp = a.logp[r];
        const int64_t t = token_at(a.tokens, a.tokens64, r);
        const float gh = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
        const float gl = !a.grad_logp || t == -1 || logp == -kInf ? 0.0f : t < -1 || t >= (int64_t)a.entries ? __builtin_nanf("") : a.grad_logp[r];
        const float base = fmaf(gh, entropy, gl);
        for (uint32_t at = threadIdx.x * N; at < a.entries; at += 256 * N) {
            float x[N], g[N];
            row_entries<T, N, MASK>(row, mask, at, a.entries, x);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float lp = fmaf(x[k] - m, a.scale, -ln_z);
                const float p = __builtin_amdgcn_exp2f(lp * kLog2e);
                g[k] = -p * fmaf(gh, lp, base);
                if (at + k == (uint64_t)t) g[k] += gl;
                g[k] = x[k] == -kInf ? 0.0f : g[k] * a.scale;
            }
            if (at + N <= a.entries) {
                store<T, N>(out + at, g);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (at + k < a.entries) out[at + k] = rounded<T>(g[k]);
            }
        }
    }
}

uint32_t groups(uint64_t n) { return (uint32_t)(n < 65536 ? n : 65536); }

template <class T>
hipError_t score(const ScoreArgs& a, hipStream_t stream) {
    if (a.mask)
        hipLaunchKernelGGL((k_score<T, true>), dim3(groups(a.rows)), dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((k_score<T, false>), dim3(groups(a.rows)), dim3(256), 0, stream, a);
    return hipGetLastError();
}
template <class T>
hipError_t score_grad(const ScoreGradArgs& a, hipStream_t stream) {
    if (a.mask)
        hipLaunchKernelGGL((k_score_grad<T, true>), dim3(groups(a.rows)), dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((k_score_grad<T, false>), dim3(groups(a.rows)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

size_t score_workspace(int32_t, uint64_t, uint32_t, uint32_t) { return 0; }

hipError_t launch_score(int32_t dtype, const ScoreArgs& a, hipStream_t stream) {
    return dtype == BPS_F32 ? score<F32>(a, stream) : dtype == BPS_BF16 ? score<Bf16>(a, stream) : score<F16>(a, stream);
}
hipError_t launch_score_grad(int32_t dtype, const ScoreGradArgs& a, hipStream_t stream) {
    return dtype == BPS_F32 ? score_grad<F32>(a, stream) : dtype == BPS_BF16 ? score_grad<Bf16>(a, stream) : score_grad<F16>(a, stream);
}

}  // namespace bps
