// Causal convolution over time, each channel by itself, and its gradient (include/bps_memory.h states the rule).
//
// A thread holds 16 bytes of channels (the last one's begin earlier where the channels end inside them, and the others' are left out
// of what it stores) and walks over a run of steps with the last inputs in registers, so that every input is
// read once, and once more by the next run's thread for its first taps - 1 windows.  Bound by memory, as long as runs are long enough:
// 8 x 4096 x 2048 bf16 with 4 taps 50 us, 5.4 TB/s; 1024 x 32 x 512 float32 26 us, 5.0 TB/s.  Rows of odd widths, whose
// vectors begin anywhere: 12 x 5003 x 1111 f16 with 4 taps 70 us, 3.8 TB/s, 1104 channels 58 us, 4.6.
#include <type_traits>

#include "memory_device.h"
#include "memory_kernels.h"

namespace bps {

namespace {

constexpr uint32_t kGroup = 256;
constexpr uint32_t kManyTaps = 6;
constexpr int kAhead = 4;                 // steps whose inputs are loaded together
// 131072 / 262144 / 524288: 8 x 4096 x 2048 bf16 with 4 taps 52 / 52 / 50 us, gradient 111 / 122 / 160
constexpr uint32_t kThreads = 131072;     // that a launch has at least, where there is work for as many

template <class T, int K, int V>
struct Window {
    static constexpr int kBefore = K > 1 ? K - 1 : 1;
    float before[kBefore][V];             // inputs of the steps before the present one, the oldest first

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < kBefore; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) before[k][v] = 0.0f;
    }
    __device__ __forceinline__ void push(const float (&x)[V]) {
        if constexpr (K > 1) {
#pragma unroll
            for (int k = 0; k + 1 < kBefore; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) before[k][v] = before[k + 1][v];
#pragma unroll
            for (int v = 0; v < V; ++v) before[kBefore - 1][v] = x[v];
        }
    }
};

// The window before step `first` of sequence b.
template <class T, int K, int V>
__device__ __forceinline__ void open_window(const bps_conv& a, uint32_t b, int64_t first, const Place& place, Window<T, K, V>& w) {
    using raw = typename T::raw;
    w.clear();
#pragma unroll
    for (int i = K - 1; i >= 1; --i) {
        const int64_t t = first - i;
        float x[V];
        if (t < 0) {
            if (!a.state) continue;
            place.load<T, V>(static_cast<const raw*>(a.state) + b * a.state_stride + (K - 1 + t) * (int64_t)a.channels, x);
        } else {
            if (a.starts.at && a.starts.at[b * a.starts.batch_stride + t * a.starts.step_stride]) w.clear();
            load_part<T, V>(static_cast<const raw*>(a.x.at) + b * a.x.batch_stride + t * a.x.step_stride + place.at, place.to, x);
        }
        w.push(x);
    }
}

template <class T, int K, int V>
__device__ __forceinline__ void load_taps(const bps_conv& a, uint32_t c, uint32_t n, float (&w)[K][V], float (&bias)[V]) {
    const bool wide = a.weight_dtype == BPS_F32;
    // a channel's taps lie together, and so do those of the thread's channels
#pragma unroll
    for (int i = 0; i < K; ++i) {
        float x[V];
        load_weights<T, V>(a.weight, (uint64_t)c * K + i * V, wide, n * K > (uint32_t)(i * V) ? n * K - i * V : 0, x);
#pragma unroll
        for (int v = 0; v < V; ++v) w[(i * V + v) % K][(i * V + v) / K] = x[v];
    }
#pragma unroll
    for (int v = 0; v < V; ++v) bias[v] = 0.0f;
    if (a.bias) load_weights<T, V>(a.bias, c, wide, n, bias);
}

// Inputs of kAhead steps as they lie in memory, on their way together; those from `left` on are the last one before them.
template <class T, int V>
struct Steps {
    Pack<typename T::raw, V> q[kAhead];
    __device__ __forceinline__ void load(const typename T::raw* p, int64_t stride, int left, uint32_t n) {
        if (n >= V) {
#pragma unroll
            for (int s = 0; s < kAhead; ++s) q[s] = *reinterpret_cast<const Pack<typename T::raw, V>*>(p + min(s, left - 1) * stride);
        } else {
#pragma unroll
            for (int s = 0; s < kAhead; ++s)
#pragma unroll
                for (int v = 0; v < V; ++v) q[s].v[v] = v < (int)n ? p[min(s, left - 1) * stride + v] : typename T::raw(0);
        }
    }
    __device__ __forceinline__ void get(int s, float (&x)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = to_float(q[s].v[v]);
    }
};
// Which of them begin an episode, a bit each.
__device__ __forceinline__ uint32_t load_starts(const bps_starts& s, uint32_t b, int64_t t, int left) {
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) bits |= (uint32_t)(k < left && s.at[b * s.batch_stride + (t + min(k, left - 1)) * s.step_stride]) << k;
    return bits;
}

template <class T, int K, int V>
__global__ __launch_bounds__(kGroup) void k_conv(const bps_conv a, const uint32_t run, const uint32_t runs) {
    using raw = typename T::raw;
    const uint32_t vectors = (a.channels + V - 1) / V;
    const uint64_t id = (uint64_t)blockIdx.x * kGroup + threadIdx.x, item = id / vectors;
    if (item >= (uint64_t)a.batch * runs) return;
    const uint32_t b = (uint32_t)(item / runs);
    const Place place = Place::inside<V>((uint32_t)(id % vectors) * V, a.channels);
    const uint32_t c = place.at, n = place.to;
    const int64_t first = (int64_t)(item % runs) * run, last = min(first + run, (int64_t)a.steps), end = steps_of(a.lengths, b, a.steps);
    float w[K][V], bias[V];
    load_taps<T, K, V>(a, c, n, w, bias);
    Window<T, K, V> window;
    open_window<T, K, V>(a, b, first, place, window);
    const raw* x_at = static_cast<const raw*>(a.x.at) + b * a.x.batch_stride + first * a.x.step_stride + c;
    raw* out_at = static_cast<raw*>(a.out.at) + b * a.out.batch_stride + first * a.out.step_stride + c;
    const int64_t stop = min(last, end);
    Steps<T, V> next;
    if (first < stop) next.load(x_at, a.x.step_stride, (int)min(stop - first, (int64_t)kAhead), n);
    for (int64_t t = first; t < stop; t += kAhead) {
        const int left = (int)min(stop - t, (int64_t)kAhead);
        const Steps<T, V> now = next;
        x_at += kAhead * a.x.step_stride;
        if (t + kAhead < stop) next.load(x_at, a.x.step_stride, (int)min(stop - t - kAhead, (int64_t)kAhead), n);
        const uint32_t starts = a.starts.at ? load_starts(a.starts, b, t, left) : 0;
        auto walk = [&](auto plain) {
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
                if (!plain && s >= left) break;
                if (!plain && (starts >> s & 1)) window.clear();
                float x[V], u[V];
                now.get(s, x);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    u[v] = __builtin_fmaf(w[K - 1][v], x[v], bias[v]);
#pragma unroll
                    for (int k = 0; k + 1 < K; ++k) u[v] = __builtin_fmaf(w[k][v], window.before[k][v], u[v]);
                    if (a.silu) u[v] *= sigmoid(u[v]);
                }
                place.store_at<T, V>(out_at, u);
                out_at += a.out.step_stride;
                window.push(x);
            }
        };
        if (left == kAhead && !starts)
            walk(std::true_type());
        else
            walk(std::false_type());
    }
    if (a.state_out && ((first < end && end <= last) || (end == 0 && first == 0))) {
        if constexpr (K > 1) {
            raw* s = static_cast<raw*>(a.state_out) + b * a.state_out_stride;
#pragma unroll
            for (int k = 0; k < K - 1; ++k) place.store<T, V>(s + k * (uint64_t)a.channels, window.before[k]);
        }
    }
    float zero[V] = {};
    for (int64_t t = max(first, end); t < last; ++t, out_at += a.out.step_stride) place.store_at<T, V>(out_at, zero);
}

// With du = grad_out * slope(u):  grad_x[t] = sum over i < K of weight[K - 1 - i] du[t + i], as far as step t + i is of step t's episode;
// grad_weight[k] = sum of du[t] x[t - K + 1 + k].  A run's thread goes on over K - 1 steps of the next run for its last
// steps' sums.  The sums of weight and bias are left for each part of the runs.  Bound by the registers that windows and sums take, 256 with
// 4 taps of 8 channels: two wavefronts a SIMD, 8 x 4096 x 2048 bf16 110 us, 3.7 TB/s (four channels a thread 144; loads ahead of their use, which
// take it to one wavefront, 203).  float32, four channels a thread: 8 x 4096 x 1024 91 us with 4 taps, 4.4 TB/s, 101 with 8.
// Four taps are held to 256 registers, which costs 8 bytes of memory a thread; five have 302 and one wavefront (8 x 4096 x 1024 90 us, held to
// 256 152).
template <class T, int K, int V>
__global__ __launch_bounds__(kGroup, K == 5 ? 1 : 2) void k_conv_grad(const bps_conv a, const uint32_t run, const uint32_t runs, const uint32_t parts, const uint32_t slots, float* sums) {
    using raw = typename T::raw;
    const uint32_t vectors = (a.channels + V - 1) / V;
    // slots > 1: a work-group has that many parts, and threads that belong to none of them
    const uint64_t id = (uint64_t)blockIdx.x * kGroup + threadIdx.x;
    const uint32_t slot = slots > 1 ? threadIdx.x / vectors : 0, at = slots > 1 ? threadIdx.x % vectors : (uint32_t)(id % vectors);
    const uint64_t part = slots > 1 ? (uint64_t)blockIdx.x * slots + slot : id / vectors;
    const bool on = slot < slots && part < parts;
    if (slots == 1 && !on) return;
    const Place place = Place::inside<V>(at * V, a.channels);
    const uint32_t c = place.at, n = place.to;
    float w[K][V], bias[V], dw[K][V], db[V];
    load_taps<T, K, V>(a, c, n, w, bias);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        db[v] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) dw[k][v] = 0.0f;
    }
    for (uint64_t item = on ? part : (uint64_t)a.batch * runs; item < (uint64_t)a.batch * runs; item += parts) {
        const uint32_t b = (uint32_t)(item / runs);
        const int64_t first = (int64_t)(item % runs) * run, last = min(first + run, (int64_t)a.steps), end = steps_of(a.lengths, b, a.steps);
        Window<T, K, V> window;
        open_window<T, K, V>(a, b, first, place, window);
        float sum[K][V];                  // of grad_x, of the step that is i steps back
#pragma unroll
        for (int i = 0; i < K; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) sum[i][v] = 0.0f;
        const raw* x_at = static_cast<const raw*>(a.x.at) + b * a.x.batch_stride + first * a.x.step_stride + c;
        const raw* g_at = static_cast<const raw*>(a.grad_out.at) + b * a.grad_out.batch_stride + first * a.grad_out.step_stride + c;
        raw* dx_at = static_cast<raw*>(a.grad_x.at) + b * a.grad_x.batch_stride + (first - (K - 1)) * a.grad_x.step_stride + c;
        int age = K;                      // steps since the episode began, as far as they matter
        // the run's steps, and K - 1 behind it: beyond the sequence's end nothing is left to add
        const int64_t stop = last + K - 1;
        for (int64_t t = first; t < stop; t += kAhead) {
            const int left = (int)min(stop - t, (int64_t)kAhead), inside = (int)min(end - t, (int64_t)kAhead);
            float x_now[kAhead][V] = {}, g_now[kAhead][V] = {};
            if (inside > 0) {
                Steps<T, V> x, g;
                x.load(x_at, a.x.step_stride, inside, n);
                g.load(g_at, a.grad_out.step_stride, inside, n);
#pragma unroll
                for (int s = 0; s < kAhead; ++s) {
                    x.get(s, x_now[s]);
                    g.get(s, g_now[s]);
                }
            }
            x_at += kAhead * a.x.step_stride;
            g_at += kAhead * a.grad_out.step_stride;
            const uint32_t starts = a.starts.at && inside > 0 ? load_starts(a.starts, b, t, inside) : 0;
            auto walk = [&](auto plain) {
#pragma unroll
                for (int s = 0; s < kAhead; ++s) {
                    if (!plain && s >= left) break;
                    float(&x)[V] = x_now[s], (&g)[V] = g_now[s];
                    if (plain || s < inside) {
                        if (!plain) {
                            age = min(age + 1, K);
                            if (starts >> s & 1) {
                                window.clear();
                                age = 0;
                            }
                        }
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            float u = __builtin_fmaf(w[K - 1][v], x[v], bias[v]);
#pragma unroll
                            for (int k = 0; k + 1 < K; ++k) u = __builtin_fmaf(w[k][v], window.before[k][v], u);
                            if (a.silu) g[v] *= silu_slope(u, sigmoid(u));
                        }
                        if (plain || t + s < last) {
#pragma unroll
                            for (int v = 0; v < V; ++v) {
                                db[v] += g[v];
                                dw[K - 1][v] = __builtin_fmaf(g[v], x[v], dw[K - 1][v]);
#pragma unroll
                                for (int k = 0; k + 1 < K; ++k) dw[k][v] = __builtin_fmaf(g[v], window.before[k][v], dw[k][v]);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < K; ++i)
                            if (plain || i <= age)
#pragma unroll
                                for (int v = 0; v < V; ++v) sum[i][v] = __builtin_fmaf(w[K - 1 - i][v], g[v], sum[i][v]);
                    }
                    if (plain || t + s - (K - 1) >= first) place.store_at<T, V>(dx_at, sum[K - 1]);
                    dx_at += a.grad_x.step_stride;
#pragma unroll
                    for (int i = K - 1; i >= 1; --i)
#pragma unroll
                        for (int v = 0; v < V; ++v) sum[i][v] = sum[i - 1][v];
#pragma unroll
                    for (int v = 0; v < V; ++v) sum[0][v] = 0.0f;
                    window.push(x);
                }
            };
            // most steps: inside the run and its sequence, with no episode that begins in or just before them
            if (inside == kAhead && !starts && age >= K && t - first >= K - 1 && t + kAhead <= last)
                walk(std::true_type());
            else
                walk(std::false_type());
        }
    }
    float* s = sums + (slots > 1 ? blockIdx.x : part) * (K + 1) * (uint64_t)a.channels;
    if (slots == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) place.store<F32, V>(s + k * (uint64_t)a.channels, dw[k]);
        place.store<F32, V>(s + K * (uint64_t)a.channels, db);
        return;
    }
    // the slots' sums meet in LDS, in their order, a channel to a thread
    __shared__ float all[V][kGroup + 1];
    auto leave = [&](const float (&x)[V], int k) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) all[v][threadIdx.x] = x[v];
        __syncthreads();
        for (uint32_t channel = threadIdx.x; channel < a.channels; channel += kGroup) {
            float sum = 0.0f;
            const uint32_t first = Place::inside<V>(channel / V * V, a.channels).at;
            for (uint32_t other = 0; other < slots; ++other) sum += all[channel - first][other * vectors + channel / V];
            s[k * (uint64_t)a.channels + channel] = sum;
        }
    };
#pragma unroll
    for (int k = 0; k < K; ++k) leave(dw[k], k);
    leave(db, K);
}

constexpr uint32_t kJoinColumns = 64, kJoinSlices = 16, kJoinAhead = 8;

// A column of sums for each of 64 lanes, the parts dealt out to 16 wavefronts, which have 8 of them on their way at a time.
__global__ __launch_bounds__(kJoinColumns* kJoinSlices) void k_join_parts(const JoinJobs jobs, uint32_t count, size_t stride) {
    __shared__ float all[kJoinSlices][kJoinColumns];
    const JoinJob& job = jobs.job[blockIdx.y];
    const uint32_t lane = threadIdx.x % kJoinColumns, slice = threadIdx.x / kJoinColumns;
    const uint64_t columns = (uint64_t)job.width * job.inner;
    for (uint64_t first = (uint64_t)blockIdx.x * kJoinColumns; first < columns; first += (uint64_t)gridDim.x * kJoinColumns) {
        const uint64_t column = first + lane;
        float sum = 0.0f;
        if (column < columns) {
            const float* p = job.parts + column;
            uint32_t k = slice;
            for (; k + (kJoinAhead - 1) * kJoinSlices < count; k += kJoinAhead * kJoinSlices) {
                float x[kJoinAhead];
#pragma unroll
                for (uint32_t i = 0; i < kJoinAhead; ++i) x[i] = p[(k + i * kJoinSlices) * stride];
                // in pairs, whose roundings are those of three additions and not of eight
#pragma unroll
                for (uint32_t n = kJoinAhead / 2; n; n /= 2)
#pragma unroll
                    for (uint32_t i = 0; i < n; ++i) x[i] += x[i + n];
                sum += x[0];
            }
            for (; k < count; k += kJoinSlices) sum += p[k * stride];
        }
        __syncthreads();
        all[slice][lane] = sum;
        __syncthreads();
        if (slice || column >= columns) continue;
#pragma unroll
        for (uint32_t p = 1; p < kJoinSlices; ++p) sum += all[p][lane];
        const uint64_t at = column % job.width * job.inner + column / job.width;
        if (job.dtype == BPS_F32)
            static_cast<float*>(job.out)[at] = sum;
        else if (job.dtype == BPS_BF16)
            static_cast<uint16_t*>(job.out)[at] = rounded<Bf16>(sum);
        else
            static_cast<_Float16*>(job.out)[at] = rounded<F16>(sum);
    }
}

// Steps of a run: as many as leave the launch kThreads threads, at most 64, at least 8.
uint32_t run_of(const bps_conv& a, uint32_t vectors) {
    uint32_t run = 64;
    while (run > 8 && (uint64_t)a.batch * ((a.steps + run - 1) / run) * vectors < kThreads) run /= 2;
    return run;
}
// Channels of a thread: 16 bytes of them, but four of the gradient's from 6 taps on, whose sums take too many registers otherwise: 8 x 4096 x
// 1024 bf16 with four and eight 67 and 106 us with 6 taps, 73 and 127 with 8.  With 5 taps, which have eight, it is 56 and 90 as well; with 4, of 2048
// channels, 144 and 110.
uint32_t width_of(const bps_conv& a, bool grad) { return a.dtype == BPS_F32 || (grad && a.taps >= kManyTaps) ? 4 : 8; }
uint32_t vectors_of(const bps_conv& a, bool grad) { return (a.channels + width_of(a, grad) - 1) / width_of(a, grad); }
uint32_t runs_of(const bps_conv& a, uint32_t run) { return a.steps ? (a.steps - 1) / run + 1 : 1; }
uint32_t parts_of(const bps_conv& a) {
    const uint32_t vectors = vectors_of(a, true);
    const uint64_t items = a.steps ? (uint64_t)a.batch * runs_of(a, run_of(a, vectors)) : 0, most = kThreads / vectors;
    return (uint32_t)(items < most ? items : most ? most : 1);
}

// Parts that a work-group of the gradient has, whose sums it joins: 228 x 3234 x 14 bf16 with 3 taps 54 us instead of 242, float32 44 instead of 134.
uint32_t slots_of(uint32_t vectors) { return vectors <= kGroup / 4 ? kGroup / vectors : 1; }

template <class T>
hipError_t conv(const bps_conv& a, hipStream_t stream) {
    constexpr int V = T::kPer16;
    const uint32_t vectors = vectors_of(a, false), run = run_of(a, vectors), runs = runs_of(a, run);
    const uint64_t threads = (uint64_t)a.batch * runs * vectors;
    const dim3 grid((uint32_t)((threads + kGroup - 1) / kGroup));
    switch (a.taps) {
        case 1: k_conv<T, 1, V><<<grid, kGroup, 0, stream>>>(a, run, runs); break;
        case 2: k_conv<T, 2, V><<<grid, kGroup, 0, stream>>>(a, run, runs); break;
        case 3: k_conv<T, 3, V><<<grid, kGroup, 0, stream>>>(a, run, runs); break;
        case 4: k_conv<T, 4, V><<<grid, kGroup, 0, stream>>>(a, run, runs); break;
        case 5: k_conv<T, 5, V><<<grid, kGroup, 0, stream>>>(a, run, runs); break;
        case 6: k_conv<T, 6, V><<<grid, kGroup, 0, stream>>>(a, run, runs); break;
        case 7: k_conv<T, 7, V><<<grid, kGroup, 0, stream>>>(a, run, runs); break;
        default: k_conv<T, 8, V><<<grid, kGroup, 0, stream>>>(a, run, runs); break;
    }
    return hipGetLastError();
}

template <class T>
hipError_t conv_grad(const bps_conv& a, float* sums, hipStream_t stream) {
    constexpr int V = T::kPer16;
    const uint32_t vectors = vectors_of(a, true), run = run_of(a, vectors), runs = runs_of(a, run), parts = parts_of(a);
    const uint32_t slots = slots_of(vectors);
    const dim3 grid(slots > 1 ? (parts + slots - 1) / slots : (uint32_t)(((uint64_t)parts * vectors + kGroup - 1) / kGroup));
    if (parts) switch (a.taps) {
        case 1: k_conv_grad<T, 1, V><<<grid, kGroup, 0, stream>>>(a, run, runs, parts, slots, sums); break;
        case 2: k_conv_grad<T, 2, V><<<grid, kGroup, 0, stream>>>(a, run, runs, parts, slots, sums); break;
        case 3: k_conv_grad<T, 3, V><<<grid, kGroup, 0, stream>>>(a, run, runs, parts, slots, sums); break;
        case 4: k_conv_grad<T, 4, V><<<grid, kGroup, 0, stream>>>(a, run, runs, parts, slots, sums); break;
        case 5: k_conv_grad<T, 5, V><<<grid, kGroup, 0, stream>>>(a, run, runs, parts, slots, sums); break;
        case 6: k_conv_grad<T, 6, 4><<<grid, kGroup, 0, stream>>>(a, run, runs, parts, slots, sums); break;
        case 7: k_conv_grad<T, 7, 4><<<grid, kGroup, 0, stream>>>(a, run, runs, parts, slots, sums); break;
        default: k_conv_grad<T, 8, 4><<<grid, kGroup, 0, stream>>>(a, run, runs, parts, slots, sums); break;
    }
    // sums of no parts are zero
    if (hipError_t e = hipGetLastError()) return e;
    JoinJobs jobs;
    jobs.add(sums, a.channels, a.taps, a.weight_dtype, a.grad_weight);
    if (a.grad_bias) jobs.add(sums + (size_t)a.taps * a.channels, a.channels, 1, a.weight_dtype, a.grad_bias);
    return launch_join_parts(jobs, (parts + slots - 1) / slots, (size_t)(a.taps + 1) * a.channels, stream);
}

}  // namespace

hipError_t launch_join_parts(const JoinJobs& jobs, uint32_t count, size_t stride, hipStream_t stream) {
    uint64_t columns = 0;
    for (uint32_t k = 0; k < jobs.count; ++k) {
        const uint64_t mine = (uint64_t)jobs.job[k].width * jobs.job[k].inner;
        if (mine > columns) columns = mine;
    }
    if (!columns) return hipSuccess;
    const uint64_t groups = (columns + kJoinColumns - 1) / kJoinColumns, most = 1 << 20;      // work-groups go on to further columns
    k_join_parts<<<dim3((uint32_t)(groups < most ? groups : most), jobs.count), kJoinColumns * kJoinSlices, 0, stream>>>(jobs, count, stride);
    return hipGetLastError();
}

hipError_t launch_conv(const bps_conv& a, hipStream_t stream) {
    return a.dtype == BPS_F32 ? conv<F32>(a, stream) : a.dtype == BPS_BF16 ? conv<Bf16>(a, stream) : conv<F16>(a, stream);
}

size_t conv_grad_workspace(const bps_conv& a) { return (size_t)parts_of(a) * (a.taps + 1) * a.channels * sizeof(float); }

hipError_t launch_conv_grad(const bps_conv& a, void* workspace, hipStream_t stream) {
    float* sums = static_cast<float*>(workspace);
    return a.dtype == BPS_F32 ? conv_grad<F32>(a, sums, stream) : a.dtype == BPS_BF16 ? conv_grad<Bf16>(a, sums, stream) : conv_grad<F16>(a, sums, stream);
}

}  // namespace bps
