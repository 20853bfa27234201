// AdamW over many tensors at once; states in 32 or in 8 bits.  The rule is in include/bps.h: every operation is
// rounded by itself (the library is built without contraction), so that what 8-bit states are rounded to can be
// reproduced bit for bit.
//
// A work-group takes a chunk of kAdamChunk elements of one tensor; a table made with the handle says which, so
// that tensors of any size keep all compute units busy and a launch takes up to kAdamGrads of them.  A lane
// takes four elements at a time, a wavefront the 256 of a state block, whose largest magnitudes are found
// across its lanes (both at once, as the halves of one word).
//
// What bounds it, on one MI355X (median kernel times): the memory.  4e8 float32 parameters 2.03 ms (5.5 TB/s of
// the 28 bytes each has to move; a copy reaches 4.9); 1.2e8 bf16 ones with float32 masters and 8-bit states 333
// us (5.8 TB/s of 16 bytes each), with the vector units near their limit too: the exact root and quotient,
// three products of the hash and the codes take about 90 instructions an element; read back 210 us (5.7 TB/s).
// 5.3e6 parameters in 38 tensors with a bound on the norm 7 and 26 us.
#include "policy_device.h"
#include "policy_kernels.h"

namespace bps {

namespace {

constexpr uint32_t kPerLane = 4;
static_assert(kStateBlock == 64 * kPerLane, "a wavefront's elements share an exponent");
static_assert(kAdamChunk == kAdamGroup * kPerLane, "a chunk is what a work-group takes at once");

// 8-bit codes are the upper bits of a float32 with a bias of their own: shifted to where those are, subnormal
// ones included, a code is a float that is a power of two away from what it stands for.  e: the block's
// exponent byte.
template <int TOP>
__device__ __forceinline__ float decoded(uint32_t code, uint32_t e) {
    return __builtin_amdgcn_ldexpf(__uint_as_float(code << 20), (int)e - TOP);
}

// the exponent byte for a magnitude's bits: the least that holds it
template <uint32_t LEAST>
__device__ __forceinline__ uint32_t exponent_for(uint32_t magnitude) {
    const uint32_t e = (magnitude + 0x0FFFFFu) >> 23;
    return e < LEAST ? LEAST : e > 255u ? 255u : e;
}

// The other way: the code's place is above 20 bits, to which 20 bits of dither (a 16-bit number, times 16) are
// added before they are cut off.
template <int TOP>
__device__ __forceinline__ uint32_t encoded(float magnitude, uint32_t e, uint32_t dither) {
    return (__float_as_uint(__builtin_amdgcn_ldexpf(magnitude, TOP - (int)e)) + (dither << 4)) >> 20;
}

// The larger of both halves over the wavefront, in all lanes.
__device__ __forceinline__ uint32_t wave_max_of_halves(uint32_t x) {
    typedef uint16_t halves __attribute__((ext_vector_type(2)));
    return group_reduce<64>(x, [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(halves, a), __builtin_bit_cast(halves, b)));
    });
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}

// Sums of squares: each work-group those of every gridDim.x-th four chunks, so that four loads are on their way
// at once.  In 64 bits, since the square of a float32 from 1.8e19 on is none, nor is that of one below 1e-23;
// the memory bounds it either way.
template <class G>
__global__ __launch_bounds__(kAdamGroup) void k_adamw_norm(AdamPlan plan, AdamGrads grads, uint32_t first_tensor, uint32_t first_chunk, uint32_t chunks, uint32_t first_sum,
                                                           AdamScalars s) {
    __shared__ double sums[kAdamGroup / 64];
    constexpr uint32_t kTogether = 4;
    const uint32_t tid = threadIdx.x, i = tid * kPerLane;
    double sum = 0.0;
    for (uint32_t c = blockIdx.x * kTogether; c < chunks; c += gridDim.x * kTogether) {
        const typename G::raw* g[kTogether];
        uint32_t n[kTogether];
#pragma unroll
        for (uint32_t u = 0; u < kTogether; ++u) {
            const AdamChunk chunk = plan.chunks[first_chunk + (c + u < chunks ? c + u : c)];
            const uint64_t from = (uint64_t)chunk.index * kAdamChunk, left = plan.tensors[chunk.tensor].count - from;
            const typename G::raw* grad = static_cast<const typename G::raw*>(grads.at[chunk.tensor - first_tensor]);
            n[u] = !grad || c + u >= chunks ? 0u : left < kAdamChunk ? (uint32_t)left : kAdamChunk;
            g[u] = grad ? grad + from : nullptr;
        }
        float x[kTogether][kPerLane];
#pragma unroll
        for (uint32_t u = 0; u < kTogether; ++u) {
            if (i + kPerLane <= n[u]) {
                load<G, kPerLane>(g[u] + i, x[u]);
            } else {
#pragma unroll
                for (uint32_t k = 0; k < kPerLane; ++k) x[u][k] = i + k < n[u] ? to_float(g[u][i + k]) : 0.0f;
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < kTogether; ++u)
#pragma unroll
            for (uint32_t k = 0; k < kPerLane; ++k) {
                const double y = x[u][k] * s.grad_scale;
                sum = fma(y, y, sum);
            }
    }
    sum = wave_sum(sum);
    if ((tid & 63u) == 0) sums[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) plan.partial[first_sum + blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// The 2-norm from the sums of squares, by every work-group of the step for itself, in an order that all share.
__device__ __forceinline__ float norm_of(const double* partial, uint32_t n, double* total) {
    const uint32_t tid = threadIdx.x;
    double all = 0.0;
    for (uint32_t i = 0; i < n; i += 4 * kAdamGroup) {
        double x[4];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) x[u] = i + u * kAdamGroup + tid < n ? partial[i + u * kAdamGroup + tid] : 0.0;
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) all += x[u];
    }
    all = wave_sum(all);
    if ((tid & 63u) == 0) total[tid >> 6] = all;
    __syncthreads();
    return (float)sqrt((total[0] + total[1]) + (total[2] + total[3]));
}

template <class P, class G, int BITS, bool CLIP>
__global__ __launch_bounds__(kAdamGroup) void k_adamw(AdamPlan plan, AdamGrads grads, uint32_t first_tensor, uint32_t first_chunk, AdamScalars s,
                                                      float* norm_out) {
    constexpr bool kMaster = sizeof(typename P::raw) == 2;
    float clip = 1.0f;
    if (CLIP) {
        __shared__ double total[kAdamGroup / 64];
        const float norm = norm_of(plan.partial, s.partials, total);
        if (norm_out && first_chunk + blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
        if (!(norm < __builtin_inff())) return;
        clip = norm > s.max_norm ? s.max_norm / norm : 1.0f;
    }
    const AdamChunk chunk = plan.chunks[first_chunk + blockIdx.x];
    const typename G::raw* g = static_cast<const typename G::raw*>(grads.at[chunk.tensor - first_tensor]);
    if (!g) return;
    const AdamTensor t = plan.tensors[chunk.tensor];
    const float keep = (float)(1.0 - s.lr * t.lr_scale * t.weight_decay), step_size = (float)(s.step_size * t.lr_scale);
    const uint64_t from = (uint64_t)chunk.index * kAdamChunk, left = t.count - from;
    const uint32_t n = left < kAdamChunk ? (uint32_t)left : kAdamChunk, i = threadIdx.x * kPerLane;
    if (i / kStateBlock * kStateBlock >= n) return;      // whole wavefronts: a state block belongs to one tensor
    const uint64_t at = from + i, state = t.start + at;
    const uint32_t live = i >= n ? 0u : n - i < kPerLane ? n - i : kPerLane;
    float x[kPerLane], w[kPerLane], m[kPerLane], v[kPerLane];
    typename P::raw* param = static_cast<typename P::raw*>(t.param) + at;
    float* weight = kMaster ? t.master + at : reinterpret_cast<float*>(t.param) + at;
    if (live == kPerLane) {
        load<G, kPerLane>(g + at, x);
        load<F32, kPerLane>(weight, w);
    } else {
#pragma unroll
        for (uint32_t k = 0; k < kPerLane; ++k) {
            x[k] = k < live ? to_float(g[at + k]) : 0.0f;
            w[k] = k < live ? weight[k] : 0.0f;
        }
    }
    uint32_t code_m = 0, code_v = 0;
    if (BITS == 32) {
        // a state block belongs to one tensor, so that all four are this lane's
        load<F32, kPerLane>(static_cast<float*>(plan.exp_avg) + state, m);
        load<F32, kPerLane>(static_cast<float*>(plan.exp_avg_sq) + state, v);
    } else {
        code_m = *reinterpret_cast<const uint32_t*>(static_cast<uint8_t*>(plan.exp_avg) + state);
        code_v = *reinterpret_cast<const uint32_t*>(static_cast<uint8_t*>(plan.exp_avg_sq) + state);
        // one block for the whole wavefront
        const uint32_t em = __builtin_amdgcn_readfirstlane(plan.exp_avg_exponent[state / kStateBlock]);
        const uint32_t ev = __builtin_amdgcn_readfirstlane(plan.exp_avg_sq_exponent[state / kStateBlock]);
#pragma unroll
        for (uint32_t k = 0; k < kPerLane; ++k) {
            const uint32_t cm = code_m >> (8 * k) & 255u, cv = code_v >> (8 * k) & 255u;
            m[k] = __uint_as_float(__float_as_uint(decoded<15>(cm & 127u, em)) | (cm & 128u) << 24);
            v[k] = decoded<31>(cv, ev);
        }
        if (em == 255u || ev == 255u) {
#pragma unroll
            for (uint32_t k = 0; k < kPerLane; ++k) {
                if (em == 255u) m[k] = __builtin_nanf("");
                if (ev == 255u) v[k] = __builtin_nanf("");
            }
        }
        if (live != kPerLane) {      // behind the tensor's end: no part of the block's largest
#pragma unroll
            for (uint32_t k = 0; k < kPerLane; ++k)
                if (k >= live) m[k] = v[k] = 0.0f;
        }
    }
#pragma unroll
    for (uint32_t k = 0; k < kPerLane; ++k) {
        x[k] = x[k] * s.grad_scale;
        if (CLIP) x[k] = x[k] * clip;
        m[k] = m[k] * s.beta1 + x[k] * s.one_minus_beta1;
        v[k] = v[k] * s.beta2 + x[k] * s.one_minus_beta2 * x[k];
        w[k] = w[k] * keep - m[k] / (sqrtf(v[k]) * s.root_c2 + s.eps) * step_size;
    }
    if (live == kPerLane) {
        store<F32, kPerLane>(weight, w);
        if (kMaster) store<P, kPerLane>(param, w);
    } else {
#pragma unroll
        for (uint32_t k = 0; k < kPerLane; ++k)
            if (k < live) {
                weight[k] = w[k];
                if (kMaster) param[k] = rounded<P>(w[k]);
            }
    }
    if (BITS == 32) {
        if (live) {
            store<F32, kPerLane>(static_cast<float*>(plan.exp_avg) + state, m);
            store<F32, kPerLane>(static_cast<float*>(plan.exp_avg_sq) + state, v);
        }
    } else {
        uint32_t largest_m = 0, largest_v = 0;
#pragma unroll
        for (uint32_t k = 0; k < kPerLane; ++k) {
            const uint32_t bm = __float_as_uint(m[k]) & 0x7FFFFFFFu, bv = __float_as_uint(v[k]) & 0x7FFFFFFFu;
            largest_m = bm > largest_m ? bm : largest_m;
            largest_v = bv > largest_v ? bv : largest_v;
        }
        const uint32_t both = __builtin_amdgcn_readfirstlane(wave_max_of_halves(exponent_for<20>(largest_m) | exponent_for<36>(largest_v) << 16));
        const uint32_t em = both & 0xFFFFu, ev = both >> 16;
        code_m = code_v = 0;
#pragma unroll
        for (uint32_t k = 0; k < kPerLane; ++k) {
            const uint32_t h = mixed(((uint32_t)(state + k) * kGolden) ^ s.key);
            code_m |= (encoded<15>(fabsf(m[k]), em, h & 0xFFFFu) | (m[k] < 0.0f ? 128u : 0u)) << (8 * k);
            code_v |= encoded<31>(v[k], ev, h >> 16) << (8 * k);
        }
        if (em == 255u) code_m = 0;
        if (ev == 255u) code_v = 0;
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(plan.exp_avg) + state) = code_m;
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(plan.exp_avg_sq) + state) = code_v;
        if ((threadIdx.x & 63u) == 0) {
            plan.exp_avg_exponent[state / kStateBlock] = (uint8_t)em;
            plan.exp_avg_sq_exponent[state / kStateBlock] = (uint8_t)ev;
        }
    }
}

// 8-bit states as float32: 16 consecutive blocks to a work-group, four to a wavefront.
constexpr uint32_t kReadBlocks = 16;
__global__ __launch_bounds__(256) void k_adamw_read(AdamPlan plan, uint64_t blocks, float* exp_avg, float* exp_avg_sq) {
    constexpr uint32_t kEach = kReadBlocks / 4;
    const uint64_t first = (uint64_t)blockIdx.x * kReadBlocks + threadIdx.x / 64 * kEach;
    uint32_t code_m[kEach], code_v[kEach], em[kEach], ev[kEach];
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) {
        const uint64_t b = first + j < blocks ? first + j : blocks - 1, at = b * kStateBlock + (threadIdx.x & 63u) * kPerLane;
        code_m[j] = *reinterpret_cast<const uint32_t*>(static_cast<uint8_t*>(plan.exp_avg) + at);
        code_v[j] = *reinterpret_cast<const uint32_t*>(static_cast<uint8_t*>(plan.exp_avg_sq) + at);
        em[j] = plan.exp_avg_exponent[b];
        ev[j] = plan.exp_avg_sq_exponent[b];
    }
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) {
        if (first + j >= blocks) return;
        const uint64_t at = (first + j) * kStateBlock + (threadIdx.x & 63u) * kPerLane;
        float m[kPerLane], v[kPerLane];
#pragma unroll
        for (uint32_t k = 0; k < kPerLane; ++k) {
            const uint32_t cm = code_m[j] >> (8 * k) & 255u;
            const float x = decoded<15>(cm & 127u, em[j]), y = decoded<31>(code_v[j] >> (8 * k) & 255u, ev[j]);
            m[k] = em[j] == 255u ? __builtin_nanf("") : cm & 128u ? -x : x;
            v[k] = ev[j] == 255u ? __builtin_nanf("") : y;
        }
        store<F32, kPerLane>(exp_avg + at, m);
        store<F32, kPerLane>(exp_avg_sq + at, v);
    }
}

template <class G>
void norm(const AdamPlan& p, const AdamGrads& g, uint32_t first_tensor, uint32_t first_chunk, uint32_t chunks, uint32_t first_sum, uint32_t groups, const AdamScalars& s,
          hipStream_t stream) {
    hipLaunchKernelGGL((k_adamw_norm<G>), dim3(groups), dim3(kAdamGroup), 0, stream, p, g, first_tensor, first_chunk, chunks, first_sum, s);
}

template <class P, class G, int BITS>
void step(const AdamPlan& p, const AdamGrads& g, uint32_t first_tensor, uint32_t first_chunk, uint32_t chunks, bool clipped, const AdamScalars& s, float* norm_out,
          hipStream_t stream) {
    if (clipped)
        hipLaunchKernelGGL((k_adamw<P, G, BITS, true>), dim3(chunks), dim3(kAdamGroup), 0, stream, p, g, first_tensor, first_chunk, s, norm_out);
    else
        hipLaunchKernelGGL((k_adamw<P, G, BITS, false>), dim3(chunks), dim3(kAdamGroup), 0, stream, p, g, first_tensor, first_chunk, s, norm_out);
}
template <class P, class G>
void step(int32_t bits, const AdamPlan& p, const AdamGrads& g, uint32_t first_tensor, uint32_t first_chunk, uint32_t chunks, bool clipped, const AdamScalars& s, float* norm_out,
          hipStream_t stream) {
    if (bits == 32)
        step<P, G, 32>(p, g, first_tensor, first_chunk, chunks, clipped, s, norm_out, stream);
    else
        step<P, G, 8>(p, g, first_tensor, first_chunk, chunks, clipped, s, norm_out, stream);
}

}  // namespace

hipError_t launch_adamw_norm(int32_t grad_dtype, const AdamPlan& p, const AdamGrads& g, uint32_t first_tensor, uint32_t first_chunk, uint32_t chunks,
                             uint32_t first_sum, uint32_t groups, const AdamScalars& s, hipStream_t stream) {
    if (grad_dtype == BPS_F32)
        norm<F32>(p, g, first_tensor, first_chunk, chunks, first_sum, groups, s, stream);
    else if (grad_dtype == BPS_BF16)
        norm<Bf16>(p, g, first_tensor, first_chunk, chunks, first_sum, groups, s, stream);
    else
        norm<F16>(p, g, first_tensor, first_chunk, chunks, first_sum, groups, s, stream);
    return hipGetLastError();
}

hipError_t launch_adamw_step(int32_t param_dtype, int32_t grad_dtype, int32_t state_bits, const AdamPlan& p, const AdamGrads& g, uint32_t first_tensor,
                             uint32_t first_chunk, uint32_t chunks, bool clipped, const AdamScalars& s, float* norm_out,
          hipStream_t stream) {
    if (param_dtype == BPS_F32)
        step<F32, F32>(state_bits, p, g, first_tensor, first_chunk, chunks, clipped, s, norm_out, stream);
    else if (param_dtype == BPS_BF16 && grad_dtype == BPS_BF16)
        step<Bf16, Bf16>(state_bits, p, g, first_tensor, first_chunk, chunks, clipped, s, norm_out, stream);
    else if (param_dtype == BPS_BF16)
        step<Bf16, F32>(state_bits, p, g, first_tensor, first_chunk, chunks, clipped, s, norm_out, stream);
    else if (grad_dtype == BPS_F16)
        step<F16, F16>(state_bits, p, g, first_tensor, first_chunk, chunks, clipped, s, norm_out, stream);
    else
        step<F16, F32>(state_bits, p, g, first_tensor, first_chunk, chunks, clipped, s, norm_out, stream);
    return hipGetLastError();
}

hipError_t launch_adamw_read(const AdamPlan& p, uint64_t blocks, float* exp_avg, float* exp_avg_sq, hipStream_t stream) {
    hipLaunchKernelGGL(k_adamw_read, dim3((uint32_t)((blocks + kReadBlocks - 1) / kReadBlocks)), dim3(256), 0, stream, p, blocks, exp_avg, exp_avg_sq);
    return hipGetLastError();
}

}  // namespace bps
