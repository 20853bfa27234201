// The norms around a block with its gate, its scale and the residual sum, and their gradient (include/bps_memory.h states the rule).
//
// R lanes hold a row in registers, P vectors of 16 bytes of the block's type to a lane: each input is read once and each
// result written once.  Work-groups, of 256 / R rows at a time where a wavefront holds a row or more, go on to further rows, with the weights
// kept.  A lane's vectors are all loaded before the first is converted; waited for one by one, in the branches that load them, 8192 x 8192 bf16
// took 208 us for 140 and 5003 x 769 f16 with its gradient 42 for 33.  Bound by memory: 32768 x 4096, bf16 blocks on a float32 stream, 400 us (4.7 TB/s) and 538
// (5.5) for the gradient; 300000 x 256 float32 300 (5.1) and 470 (5.2); 8192 x 8192 bf16 140 (4.8) and 412 (2.6), a row to all of a compute
// unit, whose wavefronts then wait together and whose sums leave no registers for loads ahead.  Odd widths: 20012 x 769 f16 39 us, x 768 33.
// Lanes of 16 wavefronts have 128 registers, which are too few for the gradient of over 4096 columns: 100 to 136 bytes of a lane go to memory for every row,
// 660 to 680 from 8193 columns on (4096 x 16384 bf16 1360 us, 0.8 TB/s), and 20 in the forward pass of such float32 rows (318 us, 4.2 TB/s; bf16, none, 181, 3.7).
#include <type_traits>

#include "memory_device.h"
#include "memory_kernels.h"

namespace bps {

namespace {

template <int R>
constexpr int kSlots = R <= 64 ? 256 / R : 1;      // rows that a work-group has at a time

// The sum over the R lanes of a row; `shared` is not used again before the next barrier.
template <int R>
__device__ __forceinline__ float row_sum(float x, float* shared) {
    x = group_reduce<(R < 64 ? R : 64)>(x, [](float p, float q) { return p + q; });
    if constexpr (R > 64) {
        __syncthreads();
        if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = x;
        __syncthreads();
        x = shared[0];
#pragma unroll
        for (int k = 1; k < R / 64; ++k) x += shared[k];
    }
    return x;
}

template <class T, int R>
__device__ __forceinline__ Place place_of(int j, uint32_t width) {
    return Place::of<T::kPer16>((j * R + threadIdx.x % R) * T::kPer16, width);
}

template <class T>
__device__ __forceinline__ void load_vector(const void* p, bool wide, const Place& place, float (&x)[T::kPer16]) {
    constexpr int V = T::kPer16;
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = 1.0f;
    if (p && place.to) load_weights<T, V>(p, place.at, wide, place.to, x);
    place.own(x);
}

template <class T, class S, int R, int P>
__global__ __launch_bounds__(R * kSlots<R>, R == 512 ? 4 : 1) void k_norm(const bps_norm a) {
    constexpr int V = T::kPer16;
    using raw = typename T::raw;
    using stream_raw = typename S::raw;
    __shared__ float shared[R < 64 ? 1 : R / 64];
    const bool wide = a.weight_dtype == BPS_F32;
    const float share = 1.0f / (float)a.width;
    float post[P][V], scale[P][V], pre[P][V];
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const Place place = place_of<T, R>(j, a.width);
        load_vector<T>(a.post_weight, wide, place, post[j]);
        load_vector<T>(a.scale, wide, place, scale[j]);
        load_vector<T>(a.pre_weight, wide, place, pre[j]);
    }
    for (uint64_t row = (uint64_t)blockIdx.x * kSlots<R> + threadIdx.x / R; row < a.rows; row += (uint64_t)gridDim.x * kSlots<R>) {
        float b[P][V], r[P][V], g[P][V];
        const raw* block = static_cast<const raw*>(a.block) + (int64_t)row * a.block_stride;
        const raw* gate = static_cast<const raw*>(a.gate) + (int64_t)row * a.gate_stride;
        const stream_raw* residual = static_cast<const stream_raw*>(a.residual) + (int64_t)row * a.residual_stride;
        Part<T, V> blocks[P], gates[P];
        Part<S, V> residuals[P];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const Place place = place_of<T, R>(j, a.width);
            if (place.to) {
                blocks[j].load(block, place);
                residuals[j].load(residual, place);
                if (a.gate) gates[j].load(gate, place);
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const Place place = place_of<T, R>(j, a.width);
            blocks[j].arrive();
            residuals[j].arrive();
            gates[j].arrive();
            blocks[j].get(place, b[j]);
            residuals[j].get(place, r[j]);
            gates[j].get(place, g[j]);
#pragma unroll
            for (int v = 0; v < V; ++v) sum = __builtin_fmaf(b[j][v], b[j][v], sum);
        }
        float root = 1.0f;
        if (a.post_weight) root = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<R>(sum, shared), share, a.eps));
        float square = 0.0f;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const Place place = place_of<T, R>(j, a.width);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float m = b[j][v] * root * post[j][v];
                if (a.gate) {
                    const float s = sigmoid(g[j][v]);
                    m *= a.activation ? g[j][v] * s : s;
                }
                r[j][v] = __builtin_fmaf(m, scale[j][v], r[j][v]);
                square = __builtin_fmaf(r[j][v], r[j][v], square);
            }
            if (a.residual_out && place.to) place.store<S, V>(static_cast<stream_raw*>(a.residual_out) + (int64_t)row * a.residual_out_stride, r[j]);
        }
        float last = 1.0f;
        if (a.pre_weight) {
            last = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<R>(square, shared), share, a.eps));
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const Place place = place_of<T, R>(j, a.width);
#pragma unroll
                for (int v = 0; v < V; ++v) r[j][v] = r[j][v] * last * pre[j][v];
                if (place.to) place.store<T, V>(static_cast<raw*>(a.out) + (int64_t)row * a.out_stride, r[j]);
            }
        }
        if (a.roots && threadIdx.x % R == 0) {
            a.roots[row] = root;
            a.roots[a.rows + row] = last;
        }
    }
}

// With h = (residual + m) / root, w = grad_out pre_weight:  d = grad_residual_out + (w - h mean(w h)) / root is the gradient of the
// sum, and so of the residual; that of m's factors follows, and through the block's norm in the same way.  What the forward pass computed is
// computed again from its inputs.  Sums over rows are left for each work-group: those of post_weight, scale and pre_weight, as far as
// there are such.
template <class T, class S, int R, int P>
__global__ __launch_bounds__(R * kSlots<R>) void k_norm_grad(const bps_norm a, float* sums) {
    constexpr int V = T::kPer16;
    using raw = typename T::raw;
    using stream_raw = typename S::raw;
    __shared__ float shared[R < 64 ? 1 : R / 64];
    const bool wide = a.weight_dtype == BPS_F32;
    const float share = 1.0f / (float)a.width;
    float post[P][V], scale[P][V], pre[P][V], d_post[P][V] = {}, d_scale[P][V] = {}, d_pre[P][V] = {};
    auto load_weights = [&](int j) {
        const Place place = place_of<T, R>(j, a.width);
        load_vector<T>(a.post_weight, wide, place, post[j]);
        load_vector<T>(a.scale, wide, place, scale[j]);
        load_vector<T>(a.pre_weight, wide, place, pre[j]);
    };
    // Weights stay in registers, and the next row is on its way while this one is worked on: 32768 x 4096 538 us, 5003 x 769 f16 19 (600 and
    // 22 without the loads ahead).  The 128 registers of a lane of 16 wavefronts have no room for either beside the sums, of which some go to
    // memory even so.
    constexpr bool kKeep = R < 1024;
    if constexpr (kKeep) load_weights(0);
    const bool through = a.pre_weight && a.grad_out;
    struct Row {
        Part<T, V> block[P], gate[P], out[P];
        Part<S, V> residual[P], stream[P];
        float root = 1.0f, last = 1.0f;
    };
    auto fetch = [&](Row& x, uint64_t row) {
        if (a.post_weight) x.root = a.roots[row];
        if (a.pre_weight) x.last = a.roots[a.rows + row];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const Place place = place_of<T, R>(j, a.width);
            if (!place.to) continue;
            x.block[j].load(static_cast<const raw*>(a.block) + (int64_t)row * a.block_stride, place);
            if (a.gate) x.gate[j].load(static_cast<const raw*>(a.gate) + (int64_t)row * a.gate_stride, place);
            if (through) {
                x.residual[j].load(static_cast<const stream_raw*>(a.residual) + (int64_t)row * a.residual_stride, place);
                x.out[j].load(static_cast<const raw*>(a.grad_out) + (int64_t)row * a.grad_out_stride, place);
            }
            if (a.grad_residual_out) x.stream[j].load(static_cast<const stream_raw*>(a.grad_residual_out) + (int64_t)row * a.grad_residual_out_stride, place);
        }
    };
    const uint64_t step = (uint64_t)gridDim.x * kSlots<R>;
    uint64_t row = (uint64_t)blockIdx.x * kSlots<R> + threadIdx.x / R;
    Row next;
    if (kKeep && row < a.rows) fetch(next, row);
    for (; row < a.rows; row += step) {
        float b[P][V], r[P][V], g[P][V], f[P][V], d[P][V], go[P][V], sum = 0.0f;
        Row now = next;
        if constexpr (!kKeep) fetch(now, row);
        auto open = [&](int j) {
            const Place place = place_of<T, R>(j, a.width);
            if constexpr (!kKeep) {
                __asm__ volatile("" ::: "memory");
                load_weights(j);
            }
            now.block[j].arrive();
            now.gate[j].arrive();
            now.residual[j].arrive();
            now.out[j].arrive();
            now.stream[j].arrive();
            now.block[j].get(place, b[j]);
            now.gate[j].get(place, g[j]);
            now.residual[j].get(place, r[j]);
            now.out[j].get(place, go[j]);
            now.stream[j].get(place, d[j]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                b[j][v] *= now.root;
                f[j][v] = 1.0f;
                if (a.gate) {
                    const float s = sigmoid(g[j][v]);
                    f[j][v] = a.activation ? g[j][v] * s : s;
                    g[j][v] = a.activation ? silu_slope(g[j][v], s) : s * (1.0f - s);
                }
                // the sum over its root, and what reaches it
                r[j][v] = __builtin_fmaf(b[j][v] * post[j][v] * f[j][v], scale[j][v], r[j][v]) * now.last;
                d_pre[j][v] = __builtin_fmaf(go[j][v], r[j][v], d_pre[j][v]);
                go[j][v] *= pre[j][v];
                sum = __builtin_fmaf(go[j][v], r[j][v], sum);
            }
        };
#pragma unroll
        for (int j = 0; j < P; ++j) open(j);
        if (kKeep && a.rows - row > step) fetch(next, row + step);
        if (through) sum = row_sum<R>(sum, shared) * share;
        float inner = 0.0f;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const Place place = place_of<T, R>(j, a.width);
            if (through) {
#pragma unroll
                for (int v = 0; v < V; ++v) d[j][v] = __builtin_fmaf(__builtin_fmaf(-r[j][v], sum, go[j][v]), now.last, d[j][v]);
            }
            if (place.to) place.store<S, V>(static_cast<stream_raw*>(a.grad_residual) + (int64_t)row * a.grad_residual_stride, d[j]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float n = b[j][v] * post[j][v];
                d_scale[j][v] = __builtin_fmaf(d[j][v], f[j][v] * n, d_scale[j][v]);
                d[j][v] *= scale[j][v];
                g[j][v] *= d[j][v] * n;
                d[j][v] *= f[j][v];
                d_post[j][v] = __builtin_fmaf(d[j][v], b[j][v], d_post[j][v]);
                d[j][v] *= post[j][v];
                inner = __builtin_fmaf(d[j][v], b[j][v], inner);
            }
            if (a.gate && place.to) place.store<T, V>(static_cast<raw*>(a.grad_gate) + (int64_t)row * a.grad_gate_stride, g[j]);
        }
        if (a.post_weight) inner = row_sum<R>(inner, shared) * share;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const Place place = place_of<T, R>(j, a.width);
            if (a.post_weight) {
#pragma unroll
                for (int v = 0; v < V; ++v) d[j][v] = __builtin_fmaf(-b[j][v], inner, d[j][v]) * now.root;
            }
            if (place.to) place.store<T, V>(static_cast<raw*>(a.grad_block) + (int64_t)row * a.grad_block_stride, d[j]);
        }
    }
    const uint32_t vectors = (a.post_weight ? 1 : 0) + (a.scale ? 1 : 0) + (a.pre_weight ? 1 : 0);
    float* s = sums + (uint64_t)blockIdx.x * vectors * a.width;
    auto leave = [&](float (&d)[P][V]) {
        if constexpr (kSlots<R> > 1) {
            // the rows' sums meet in LDS, in the rows' order
            __shared__ float other[kSlots<R>][P * V][R];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < P; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) other[threadIdx.x / R][j * V + v][threadIdx.x % R] = d[j][v];
            __syncthreads();
            if (threadIdx.x < R)
#pragma unroll
            for (int j = 0; j < P; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int k = 1; k < kSlots<R>; ++k) d[j][v] += other[k][j * V + v][threadIdx.x];
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const Place place = place_of<T, R>(j, a.width);
            if (place.to && (kSlots<R> == 1 || threadIdx.x < R)) place.store<F32, V>(s, d[j]);
        }
        s += a.width;
    };
    if (a.post_weight) leave(d_post);
    if (a.scale) leave(d_scale);
    if (a.pre_weight) leave(d_pre);
}

uint32_t vectors_of(const bps_norm& a) { return (a.width + (a.dtype == BPS_F32 ? 3 : 7)) / (a.dtype == BPS_F32 ? 4 : 8); }
// Lanes of a row, one vector to a lane as far as 16 wavefronts go: 32768 x 4096 376 us forward and 534 for the gradient, 5003 x 769 f16 14 and 26.  With
// two to a lane in half the wavefronts they took 475 and 1110, 16 and 46, as long as a lane's vectors were waited for one by one; as they are loaded
// now, together and a row ahead, it is 360 and 440, 14 and 23, which this choice does not make use of.
uint32_t lanes_of(const bps_norm& a) {
    const uint32_t vectors = vectors_of(a);
    return vectors <= 16 ? 16 : vectors <= 64 ? 64 : vectors <= 128 ? 128 : vectors <= 256 ? 256 : vectors <= 512 ? 512 : 1024;
}
uint32_t slots_of(uint32_t lanes) { return lanes <= 64 ? 256 / lanes : 1; }
// Work-groups of the gradient: 2048 wavefronts at most, but one for each compute unit.  2048 / 4096 / 6144, with the joining of the sums: 5003 x 769
// f16 26 / 36 / 42 us, 32768 x 4096 534 / 553 / 556.
// Of rows to 64 lanes or fewer as many times that as leave a lane about 256: sums of thousands of rows one after another are further from 64 bits than what they
// are made of (2^24 x 32 float32, 2048 rows each, 11 x 2^-24 off instead of 6), and more work-groups than are on the card at a time are no slower there:
// 6250000 x 16 float32 853 us for 1050, 1470000 x 68 933 for 1030; 300000 x 2048 bf16, which is left as it is, would take 2010 for 1800.
uint32_t groups_of(const bps_norm& a) {
    const uint32_t lanes = lanes_of(a), slots = slots_of(lanes), least = lanes <= 512 ? 2048 * 64 / (lanes * slots) : 256, limit = lanes <= 64 ? (1 << 20) / least : 1;
    const uint64_t all = (a.rows + slots - 1) / slots, times = (all / 256 + least - 1) / least;
    return (uint32_t)(all < least ? all : least * (times < 1 ? 1 : times < limit ? times : limit));
}
uint32_t sums_of(const bps_norm& a) { return (a.post_weight ? 1 : 0) + (a.scale ? 1 : 0) + (a.pre_weight ? 1 : 0); }

template <class T, class S>
hipError_t norm(const bps_norm& a, float* sums, hipStream_t stream) {
    const uint32_t vectors = vectors_of(a), lanes = lanes_of(a), slots = slots_of(lanes);
    const uint64_t all = (a.rows + slots - 1) / slots;
    const dim3 grid(sums ? groups_of(a) : (uint32_t)(all < 16384 ? all : 16384));
    auto go = [&](auto r, auto p) {
        constexpr int R = decltype(r)::value, P = decltype(p)::value;
        if (sums)
            k_norm_grad<T, S, R, P><<<grid, R * kSlots<R>, 0, stream>>>(a, sums);
        else
            k_norm<T, S, R, P><<<grid, R * kSlots<R>, 0, stream>>>(a);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    if (lanes == 16)
        go(std::integral_constant<int, 16>(), one);
    else if (lanes == 64)
        go(std::integral_constant<int, 64>(), one);
    else if (lanes == 128)
        go(std::integral_constant<int, 128>(), one);
    else if (lanes == 256)
        go(std::integral_constant<int, 256>(), one);
    else if (lanes == 512)
        go(std::integral_constant<int, 512>(), one);
    // With two vectors to each of 512 lanes 8192 x 8192 bf16 took 460 us for 412 before rows were loaded ahead, which only those have the registers
    // for; with that it is 166, which this choice does not make use of.
    else if (vectors <= 1024 && sums)
        k_norm_grad<T, S, 1024, 1><<<grid, 1024, 0, stream>>>(a, sums);
    else if (vectors <= 1024)             // two work-groups of 8 wavefronts on a compute unit: 8192 x 8192 bf16 142 us, one of 16 203
        k_norm<T, S, 512, 2><<<grid, 512, 0, stream>>>(a);
    else if (T::kPer16 == 8 || vectors <= 2048)
        go(std::integral_constant<int, 1024>(), two);
    else if constexpr (T::kPer16 == 4)
        go(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>());
    return hipGetLastError();
}

hipError_t any_norm(const bps_norm& a, float* sums, hipStream_t stream) {
    if (a.dtype == BPS_F32) return norm<F32, F32>(a, sums, stream);
    if (a.dtype == BPS_BF16) return a.residual_dtype == BPS_F32 ? norm<Bf16, F32>(a, sums, stream) : norm<Bf16, Bf16>(a, sums, stream);
    return a.residual_dtype == BPS_F32 ? norm<F16, F32>(a, sums, stream) : norm<F16, F16>(a, sums, stream);
}

}  // namespace

hipError_t launch_norm(const bps_norm& a, hipStream_t stream) { return any_norm(a, nullptr, stream); }

// Not 0 where there are rows, so that the sums' address tells the gradient.
size_t norm_grad_workspace(const bps_norm& a) { return (size_t)groups_of(a) * (sums_of(a) ? sums_of(a) : 1) * a.width * sizeof(float); }

hipError_t launch_norm_grad(const bps_norm& a, void* workspace, hipStream_t stream) {
    float* sums = static_cast<float*>(workspace);
    if (a.rows)
        if (hipError_t e = any_norm(a, sums, stream)) return e;
    const uint32_t groups = groups_of(a);
    const size_t stride = (size_t)sums_of(a) * a.width;
    const void* weight[3] = {a.post_weight, a.scale, a.pre_weight};
    void* out[3] = {a.grad_post_weight, a.grad_scale, a.grad_pre_weight};
    JoinJobs jobs;
    for (int k = 0; k < 3; ++k) {
        if (!weight[k]) continue;
        jobs.add(sums, a.width, 1, a.weight_dtype, out[k]);
        sums += a.width;
    }
    return launch_join_parts(jobs, groups, stride, stream);
}

}  // namespace bps
