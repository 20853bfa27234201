// Selective scan over time and its gradient (include/bps.h states the rule).
//
// A lane holds one channel with all of its states in registers and walks over time, so that no step needs another lane: sums over
// the states are sums within a lane.  B and C are the same for all lanes of a wavefront.  Where channels and sequences are too few to
// fill the card, the time is cut into chunks: a first pass finds what each chunk makes of states of zero and the
// sum of its steps, from which a second one finds the states at each chunk's beginning (the decays of a whole chunk are e^(A sum of d)), and the
// last one goes over all chunks at once.  The gradient does the same from the end to the beginning.
#include "memory_device.h"
#include "memory_kernels.h"

namespace bps {

namespace {

constexpr int kTile = (int)kHeldSteps;    // steps whose inputs are loaded together

struct ScanPlan {
    uint32_t tiles;                       // of 64 channels of a group
    uint32_t chunks, chunk_steps;
    uint32_t parts;                       // the gradient's work-groups that share the pieces of a tile among them
    float *ends, *spans;                  // [chunks][batch][states][channels], [chunks][batch][2][channels]: with more than one chunk
    float *sums, *shared;                 // the gradient's: [parts][states + 2][channels], [tiles][batch][steps][groups][2 states]
};

// Where a wavefront is: its channel, and whether that is one of its own.
struct Place {
    uint32_t group, channel;
    bool on;
};
__device__ __forceinline__ Place place_of(const bps_scan& a, const ScanPlan& p, uint32_t tile) {
    const uint32_t each = a.channels / a.groups, group = tile / p.tiles, c = tile % p.tiles * 64 + threadIdx.x;
    return {group, group * each + min(c, each - 1), c < each};
}

__device__ __forceinline__ int64_t steps_of(const int32_t* lengths, uint32_t b, uint32_t steps) {
    if (!lengths) return steps;
    const int32_t n = lengths[b];
    return n < 0 ? 0 : (uint32_t)n < steps ? n : steps;
}

template <class T>
struct Inputs {
    typename T::raw v[kTile];
    // steps t .. t + kTile - 1 of a sequence, those before `first` and from `end` on as the nearest one between
    __device__ __forceinline__ void load(const bps_sequence& s, uint32_t b, int64_t t, int64_t end, uint32_t c) {
        const typename T::raw* p = static_cast<const typename T::raw*>(s.at) + b * s.batch_stride + c;
#pragma unroll
        for (int k = 0; k < kTile; ++k) v[k] = p[min(t + k, end - 1) * s.step_stride];
    }
    __device__ __forceinline__ float operator[](int k) const { return to_float(v[k]); }
};

// B and C of kTile steps as float32, [step][B 0 .. N - 1, C 0 .. N - 1]; those of states that there are not are 0.
template <class T, int N>
__device__ __forceinline__ void load_shared(const bps_scan& a, uint32_t b, int64_t t, int64_t end, uint32_t group, float (&to)[kTile][2 * N]) {
    using raw = typename T::raw;
#pragma unroll
    for (int e = 0; e < (2 * N * kTile + 63) / 64; ++e) {
        const uint32_t i = e * 64 + threadIdx.x, k = i / (2 * N), n = i % N;
        if (i >= 2 * N * kTile) break;
        const bps_sequence& s = i % (2 * N) < N ? a.B : a.C;
        float x = 0.0f;
        if (n < a.states) x = to_float((static_cast<const raw*>(s.at) + b * s.batch_stride + min(t + k, end - 1) * s.step_stride)[group * a.states + n]);
        to[k][i % (2 * N)] = x;
    }
}

// Which of kTile steps begin an episode, a bit each.
__device__ __forceinline__ uint32_t load_starts(const bps_starts& s, uint32_t b, int64_t t, int64_t end) {
    if (!s.at) return 0;
    const int64_t k = t + threadIdx.x;
    return (uint32_t)__ballot(threadIdx.x < kTile && k < end && s.at[b * s.batch_stride + min(k, end - 1) * s.step_stride]);
}

__device__ __forceinline__ float step_size(float delta, float bias, bool soft) {
    const float v = delta + bias;
    return soft ? softplus(v) : v;
}

template <int N>
__device__ __forceinline__ void load_rates(const bps_scan& a, uint32_t c, float (&rate)[N], float factor) {
#pragma unroll
    for (int n = 0; n < N; ++n) rate[n] = n < (int)a.states ? a.A[n * (uint64_t)a.channels + c] * factor : 0.0f;
}

template <int N>
__device__ __forceinline__ void load_states(const float* s, const bps_scan& a, uint32_t c, float (&h)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) h[n] = s && n < (int)a.states ? s[n * (uint64_t)a.channels + c] : 0.0f;
}
template <int N>
__device__ __forceinline__ void store_states(float* s, const bps_scan& a, const Place& at, const float (&h)[N]) {
    if (!s || !at.on) return;
#pragma unroll
    for (int n = 0; n < N; ++n)
        if (n < (int)a.states) s[n * (uint64_t)a.channels + at.channel] = h[n];
}

// FIRST: what each chunk makes of states of zero, and its steps' sum.  Otherwise the outputs.
template <class T, int N, bool FIRST>
__global__ __launch_bounds__(64) void k_scan(const bps_scan a, const ScanPlan p) {
    using raw = typename T::raw;
    __shared__ float shared[kTile][2 * N];
    const uint32_t all_tiles = p.tiles * a.groups, tile = blockIdx.x % all_tiles;
    const uint64_t item = blockIdx.x / all_tiles;
    const uint32_t chunk = (uint32_t)(item % p.chunks), b = (uint32_t)(item / p.chunks);
    const Place at = place_of(a, p, tile);
    const uint32_t c = at.channel;
    const int64_t length = steps_of(a.lengths, b, a.steps), first = (int64_t)chunk * p.chunk_steps, last = min(first + p.chunk_steps, (int64_t)a.steps),
                  end = min(last, length);
    const uint64_t cell = ((uint64_t)chunk * a.batch + b);
    float h[N], rate[N];
    load_rates<N>(a, c, rate, kLog2e);
    const float bias = a.delta_bias ? a.delta_bias[c] : 0.0f, skip = !FIRST && a.D ? a.D[c] : 0.0f;
    if constexpr (FIRST)
        load_states<N>(nullptr, a, c, h);
    else
        load_states<N>(p.chunks > 1 ? p.ends + cell * a.states * a.channels : a.state ? a.state + b * a.state_stride : nullptr, a, c, h);
    float span = 0.0f, keeps = 1.0f;
    raw* out = FIRST ? nullptr : static_cast<raw*>(a.out.at) + b * a.out.batch_stride + c;
    for (int64_t t = first; t < end; t += kTile) {
        Inputs<T> x, delta, gate;
        x.load(a.x, b, t, end, c);
        delta.load(a.delta, b, t, end, c);
        if (!FIRST && a.gate.at) gate.load(a.gate, b, t, end, c);
        const uint32_t starts = load_starts(a.starts, b, t, end);
        __syncthreads();
        load_shared<T, N>(a, b, t, end, at.group, shared);
        __syncthreads();
        if constexpr (!FIRST)
            if (a.held) store_states<N>(a.held + ((uint64_t)b * ((a.steps + kTile - 1) / kTile) + t / kTile) * a.states * a.channels, a, at, h);
#pragma unroll
        for (int k = 0; k < kTile; ++k) {
            if (t + k >= end) break;
            if (starts >> k & 1) {
                keeps = 0.0f;
#pragma unroll
                for (int n = 0; n < N; ++n) h[n] = 0.0f;
            }
            const float d = step_size(delta[k], bias, a.softplus), in = d * x[k];
            span += d;
            float y = skip * x[k];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                h[n] = __builtin_fmaf(h[n], __builtin_amdgcn_exp2f(d * rate[n]), in * shared[k][n]);
                if constexpr (!FIRST) y = __builtin_fmaf(h[n], shared[k][N + n], y);
            }
            if constexpr (!FIRST) {
                if (a.gate.at) y *= gate[k] * sigmoid(gate[k]);
                if (at.on) out[(t + k) * a.out.step_stride] = rounded<T>(y);
            }
        }
    }
    if constexpr (FIRST) {
        store_states<N>(p.ends + cell * a.states * a.channels, a, at, h);
        if (at.on) {
            p.spans[cell * 2 * a.channels + c] = span;
            p.spans[(cell * 2 + 1) * a.channels + c] = keeps;
        }
    } else {
        if (p.chunks == 1 && a.state_out) store_states<N>(a.state_out + b * a.state_out_stride, a, at, h);
        if (at.on)
            for (int64_t t = max(first, length); t < last; ++t) out[t * a.out.step_stride] = rounded<T>(0.0f);
    }
}

// What the first pass left of each chunk becomes what the chunk begins with: REVERSE from the last chunk to the first, with nothing
// behind the last.
template <bool REVERSE>
__global__ __launch_bounds__(256) void k_scan_join(const bps_scan a, const ScanPlan p) {
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x, per = (uint64_t)a.states * a.channels;
    if (id >= a.batch * per) return;
    const uint32_t b = (uint32_t)(id / per), c = (uint32_t)(id % a.channels);
    const float rate = a.A[id % per] * kLog2e;
    float h = !REVERSE && a.state ? a.state[b * a.state_stride + id % per] : 0.0f;
    for (uint32_t i = 0; i < p.chunks; ++i) {
        const uint64_t cell = (uint64_t)(REVERSE ? p.chunks - 1 - i : i) * a.batch + b;
        float* end = p.ends + cell * per + id % per;
        const float mine = *end, span = p.spans[cell * 2 * a.channels + c], keeps = p.spans[(cell * 2 + 1) * a.channels + c];
        *end = h;
        h = keeps != 0.0f ? __builtin_fmaf(h, __builtin_amdgcn_exp2f(span * rate), mine) : mine;
    }
    if (!REVERSE && a.state_out) a.state_out[b * a.state_out_stride + id % per] = h;
}

// Pairs of sums over the upper and lower half of 2 S lanes each: afterwards lanes with bit S hold the second of each pair.
template <int S>
__device__ __forceinline__ float pair_sum(float x, float y) {
    if constexpr (S == 32 || S == 16) {
        typedef uint32_t Two __attribute__((ext_vector_type(2)));
        const auto r = [&] {
            if constexpr (S == 32)
                return __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
            else
                return __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
        }();
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        // a permutation within 16 lanes that turns over bit S, and no higher one
        constexpr int X = 2 * S - 1;
        const bool upper = threadIdx.x & S;
        const float mine = upper ? y : x, other = upper ? x : y;
        return mine + from_lane_xor<X == 7 ? 7 : X>(other);
    }
}

// The sums over 64 lanes of each of K values: lane i gets that of value i K / 64.
template <int K, int S = 32>
__device__ __forceinline__ float lane_sums(float (&v)[K]) {
    if constexpr (K > 1) {
        float half[K / 2];
#pragma unroll
        for (int k = 0; k < K / 2; ++k) half[k] = pair_sum<S>(v[k], v[k + K / 2]);
        return lane_sums<K / 2, S / 2>(half);
    } else {
        float x = v[0];
        if constexpr (S >= 8) x += from_lane_xor<15>(x);
        if constexpr (S >= 4) x += from_lane_xor<7>(x);
        if constexpr (S >= 2) x += from_lane_xor<3>(x);
        if constexpr (S >= 1) x += from_lane_xor<1>(x);
        return x;
    }
}

// What reaches the states in front of each chunk of what is behind its last step: zero there.
template <class T, int N>
__global__ __launch_bounds__(64) void k_scan_grad_first(const bps_scan a, const ScanPlan p) {
    __shared__ float shared[kTile][2 * N];
    const uint32_t all_tiles = p.tiles * a.groups, tile = blockIdx.x % all_tiles;
    const uint64_t item = blockIdx.x / all_tiles;
    const uint32_t chunk = (uint32_t)(item % p.chunks), b = (uint32_t)(item / p.chunks);
    const Place at = place_of(a, p, tile);
    const uint32_t c = at.channel;
    const int64_t length = steps_of(a.lengths, b, a.steps), first = (int64_t)chunk * p.chunk_steps, end = min(min(first + p.chunk_steps, (int64_t)a.steps), length);
    const uint64_t cell = ((uint64_t)chunk * a.batch + b);
    float g[N], rate[N];
    load_rates<N>(a, c, rate, kLog2e);
    const float bias = a.delta_bias ? a.delta_bias[c] : 0.0f;
    float span = 0.0f, keeps = 1.0f;
#pragma unroll
    for (int n = 0; n < N; ++n) g[n] = 0.0f;
    for (int64_t t = first + (end - first - 1) / kTile * kTile; t >= first && first < end; t -= kTile) {
        Inputs<T> delta, gate, grad;
        delta.load(a.delta, b, t, end, c);
        grad.load(a.grad_out, b, t, end, c);
        if (a.gate.at) gate.load(a.gate, b, t, end, c);
        const uint32_t starts = load_starts(a.starts, b, t, end);
        __syncthreads();
        load_shared<T, N>(a, b, t, end, at.group, shared);
        __syncthreads();
#pragma unroll
        for (int k = kTile - 1; k >= 0; --k) {
            if (t + k >= end) continue;
            const float d = step_size(delta[k], bias, a.softplus);
            span += d;
            float dy = grad[k];
            if (a.gate.at) dy *= gate[k] * sigmoid(gate[k]);
            const bool begins = starts >> k & 1;
            if (begins) keeps = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                g[n] = __builtin_fmaf(shared[k][N + n], dy, g[n]);
                g[n] = begins ? 0.0f : g[n] * __builtin_amdgcn_exp2f(d * rate[n]);
            }
        }
    }
    store_states<N>(p.ends + cell * a.states * a.channels, a, at, g);
    if (at.on) {
        p.spans[cell * 2 * a.channels + c] = span;
        p.spans[(cell * 2 + 1) * a.channels + c] = keeps;
    }
}

// The gradient.  With dy = grad_out silu(gate) and g the gradient of the states behind a step,
//   g = C dy + (decay of the step behind) (g behind);   grad_C = sum over channels of dy h;   grad_B = sum over channels of g d x
//   grad_x = d sum of g B + D dy;   grad_d = x sum of g B + sum of A g a h before;   grad_A = sum over time of d g a h before
// kTile steps at a time from the last to the first: forward from the states held before them, with all of their states kept in
// registers, then backward.  Sums over channels are sums over the lanes of a wavefront, left for each tile of 64 channels.
template <class T, int N>
__global__ __launch_bounds__(64) void k_scan_grad(const bps_scan a, const ScanPlan p) {
    using raw = typename T::raw;
    __shared__ float shared[kTile][2 * N];
    const uint32_t all_tiles = p.tiles * a.groups, tile = blockIdx.x % all_tiles, part = blockIdx.x / all_tiles;
    const Place at = place_of(a, p, tile);
    const uint32_t c = at.channel;
    float rate[N], d_rate[N];
    load_rates<N>(a, c, rate, 1.0f);
    const float bias = a.delta_bias ? a.delta_bias[c] : 0.0f, skip = a.D ? a.D[c] : 0.0f;
    float d_skip = 0.0f, d_bias = 0.0f;
#pragma unroll
    for (int n = 0; n < N; ++n) d_rate[n] = 0.0f;
    for (uint64_t item = part; item < (uint64_t)a.batch * p.chunks; item += p.parts) {
        const uint32_t chunk = (uint32_t)(item % p.chunks), b = (uint32_t)(item / p.chunks);
        const int64_t length = steps_of(a.lengths, b, a.steps), first = (int64_t)chunk * p.chunk_steps, last = min(first + p.chunk_steps, (int64_t)a.steps),
                      end = min(last, length);
        raw* dx_at = static_cast<raw*>(a.grad_x.at) + b * a.grad_x.batch_stride + c;
        raw* dd_at = static_cast<raw*>(a.grad_delta.at) + b * a.grad_delta.batch_stride + c;
        raw* dz_at = static_cast<raw*>(a.grad_gate.at) + b * a.grad_gate.batch_stride + c;
        float g[N];                       // of the states before the step behind
        // nothing for the lanes behind the last channel, which have no part in the sums over channels
        load_states<N>(p.chunks > 1 && at.on ? p.ends + ((uint64_t)chunk * a.batch + b) * a.states * a.channels : nullptr, a, c, g);
        for (int64_t t = first + (end - first - 1) / kTile * kTile; t >= first && first < end; t -= kTile) {
            Inputs<T> x, delta, gate, grad;
            x.load(a.x, b, t, end, c);
            delta.load(a.delta, b, t, end, c);
            grad.load(a.grad_out, b, t, end, c);
            if (a.gate.at) gate.load(a.gate, b, t, end, c);
            const uint32_t starts = load_starts(a.starts, b, t, end);
            __syncthreads();
            load_shared<T, N>(a, b, t, end, at.group, shared);
            __syncthreads();
            float h[kTile + 1][N], y[kTile];
            load_states<N>(a.held + ((uint64_t)b * ((a.steps + kTile - 1) / kTile) + t / kTile) * a.states * a.channels, a, c, h[0]);
#pragma unroll
            for (int k = 0; k < kTile; ++k) {
                // a step behind the end has no part in what follows
                const float d = step_size(delta[k], bias, a.softplus), in = d * x[k];
                const bool begins = starts >> k & 1;
                y[k] = skip * x[k];
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const float kept = begins ? 0.0f : h[k][n] * __builtin_amdgcn_exp2f(d * rate[n] * kLog2e);
                    h[k + 1][n] = __builtin_fmaf(in, shared[k][n], kept);
                    y[k] = __builtin_fmaf(h[k + 1][n], shared[k][N + n], y[k]);
                }
            }
#pragma unroll
            for (int k = kTile - 1; k >= 0; --k) {
                if (t + k >= end) continue;
                const float v = delta[k] + bias, d = a.softplus ? softplus(v) : v, in = d * x[k];
                const bool begins = starts >> k & 1;
                float dy = at.on ? grad[k] : 0.0f;
                if (a.gate.at) {
                    const float s = sigmoid(gate[k]);
                    const float dz = dy * y[k] * silu_slope(gate[k], s);
                    dy *= gate[k] * s;
                    if (at.on) dz_at[(t + k) * a.grad_gate.step_stride] = rounded<T>(dz);
                }
                float gb = 0.0f, dd = 0.0f, both[2 * N];
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    g[n] = __builtin_fmaf(shared[k][N + n], dy, g[n]);
                    both[n] = g[n] * in;
                    both[N + n] = dy * h[k + 1][n];
                    gb = __builtin_fmaf(g[n], shared[k][n], gb);
                    g[n] = begins ? 0.0f : g[n] * __builtin_amdgcn_exp2f(d * rate[n] * kLog2e);
                    const float q = begins ? 0.0f : g[n] * h[k][n];
                    d_rate[n] = __builtin_fmaf(q, d, d_rate[n]);
                    dd = __builtin_fmaf(q, rate[n], dd);
                }
                dd = __builtin_fmaf(gb, x[k], dd);
                if (a.softplus) dd *= sigmoid(v);
                d_skip = __builtin_fmaf(dy, x[k], d_skip);
                d_bias += dd;
                if (at.on) {
                    dx_at[(t + k) * a.grad_x.step_stride] = rounded<T>(__builtin_fmaf(d, gb, skip * dy));
                    dd_at[(t + k) * a.grad_delta.step_stride] = rounded<T>(dd);
                }
                const float sum = lane_sums<2 * N>(both);
                constexpr uint32_t kLanes = 64 / (2 * N);
                if (threadIdx.x % kLanes == 0)
                    p.shared[((((uint64_t)(tile % p.tiles) * a.batch + b) * a.steps + t + k) * a.groups + at.group) * 2 * N + threadIdx.x / kLanes] = sum;
            }
        }
        if (at.on)
            for (int64_t t = max(first, length); t < last; ++t) {
                dx_at[t * a.grad_x.step_stride] = dd_at[t * a.grad_delta.step_stride] = rounded<T>(0.0f);
                if (a.gate.at) dz_at[t * a.grad_gate.step_stride] = rounded<T>(0.0f);
            }
    }
    float* s = p.sums + (uint64_t)part * (a.states + 2) * a.channels;
    store_states<N>(s, a, at, d_rate);
    if (at.on) {
        s[a.states * (uint64_t)a.channels + c] = d_skip;
        s[(a.states + 1) * (uint64_t)a.channels + c] = d_bias;
    }
}

// grad_B and grad_C: the sums of all tiles of a group, zero behind a sequence's end.
template <class T, int N>
__global__ __launch_bounds__(256) void k_scan_grad_shared(const bps_scan a, const ScanPlan p) {
    using raw = typename T::raw;
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x, row = id / (2 * N), size = (uint64_t)a.batch * a.steps * a.groups;
    const uint32_t i = id % (2 * N), n = i % N;
    if (row >= size || n >= a.states) return;
    const uint32_t group = (uint32_t)(row % a.groups), b = (uint32_t)(row / a.groups / a.steps);
    const int64_t t = (int64_t)(row / a.groups % a.steps);
    float sum = 0.0f;
    if (t < steps_of(a.lengths, b, a.steps))
        for (uint32_t k = 0; k < p.tiles; ++k) sum += p.shared[(k * size + row) * 2 * N + i];
    const bps_sequence& s = i < N ? a.grad_B : a.grad_C;
    (static_cast<raw*>(s.at) + b * s.batch_stride + t * s.step_stride)[group * a.states + n] = rounded<T>(sum);
}

constexpr uint32_t kWaves = 4096;         // that a launch has at least, where there is work for as many
constexpr uint32_t kLeast = 32;           // steps of a chunk

ScanPlan plan_of(const bps_scan& a) {
    ScanPlan p{};
    p.tiles = (a.channels / a.groups + 63) / 64;
    const uint64_t waves = (uint64_t)a.batch * p.tiles * a.groups;
    const uint64_t want = waves ? kWaves / waves : 1, most = a.steps / kLeast;
    const uint32_t chunks = (uint32_t)(want < most ? want : most);
    p.chunk_steps = chunks > 1 ? ((a.steps + chunks - 1) / chunks + kTile - 1) / kTile * kTile : a.steps ? a.steps : 1;
    p.chunks = a.steps ? (a.steps + p.chunk_steps - 1) / p.chunk_steps : 1;
    const uint64_t items = (uint64_t)a.batch * p.chunks, share = kWaves / (p.tiles * a.groups);
    p.parts = (uint32_t)(items < share ? items : share ? share : 1);
    return p;
}
uint32_t padded(uint32_t states) { return states <= 4 ? 4 : states <= 8 ? 8 : states <= 16 ? 16 : 32; }
size_t chunk_floats(const bps_scan& a, const ScanPlan& p) { return p.chunks > 1 ? (size_t)p.chunks * a.batch * (a.states + 2) * a.channels : 0; }
// the parts of a workspace, each in whole vectors
size_t whole(size_t floats) { return (floats + 3) / 4 * 4; }

void place_chunks(const bps_scan& a, ScanPlan& p, float* space) {
    p.ends = space;
    p.spans = space + (size_t)p.chunks * a.batch * a.states * a.channels;
}

template <class T, int N>
hipError_t scan(const bps_scan& a, const ScanPlan& p, hipStream_t stream) {
    const uint32_t grid = (uint32_t)((uint64_t)a.batch * p.chunks * p.tiles * a.groups);
    if (p.chunks > 1) {
        k_scan<T, N, true><<<grid, 64, 0, stream>>>(a, p);
        if (hipError_t e = hipGetLastError()) return e;
        k_scan_join<false><<<(uint32_t)(((uint64_t)a.batch * a.states * a.channels + 255) / 256), 256, 0, stream>>>(a, p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    k_scan<T, N, false><<<grid, 64, 0, stream>>>(a, p);
    return hipGetLastError();
}

template <class T, int N>
hipError_t scan_grad(const bps_scan& a, const ScanPlan& p, hipStream_t stream) {
    if (p.chunks > 1) {
        k_scan_grad_first<T, N><<<(uint32_t)((uint64_t)a.batch * p.chunks * p.tiles * a.groups), 64, 0, stream>>>(a, p);
        if (hipError_t e = hipGetLastError()) return e;
        k_scan_join<true><<<(uint32_t)(((uint64_t)a.batch * a.states * a.channels + 255) / 256), 256, 0, stream>>>(a, p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (a.batch && a.steps) {
        k_scan_grad<T, N><<<p.parts * p.tiles * a.groups, 64, 0, stream>>>(a, p);
        if (hipError_t e = hipGetLastError()) return e;
        k_scan_grad_shared<T, N><<<(uint32_t)(((uint64_t)a.batch * a.steps * a.groups * 2 * N + 255) / 256), 256, 0, stream>>>(a, p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    const size_t stride = (size_t)(a.states + 2) * a.channels;
    const uint32_t count = a.batch && a.steps ? p.parts : 0;      // sums of nothing are zero
    if (hipError_t e = launch_join_parts(p.sums, count, stride, a.channels * a.states, 1, BPS_F32, a.grad_A, stream)) return e;
    if (a.D)
        if (hipError_t e = launch_join_parts(p.sums + (size_t)a.states * a.channels, count, stride, a.channels, 1, BPS_F32, a.grad_D, stream)) return e;
    if (a.delta_bias)
        if (hipError_t e = launch_join_parts(p.sums + (size_t)(a.states + 1) * a.channels, count, stride, a.channels, 1, BPS_F32, a.grad_delta_bias, stream)) return e;
    return hipSuccess;
}

template <class T>
hipError_t scan_of(const bps_scan& a, const ScanPlan& p, bool grad, hipStream_t stream) {
    switch (padded(a.states)) {
        case 4: return grad ? scan_grad<T, 4>(a, p, stream) : scan<T, 4>(a, p, stream);
        case 8: return grad ? scan_grad<T, 8>(a, p, stream) : scan<T, 8>(a, p, stream);
        case 16: return grad ? scan_grad<T, 16>(a, p, stream) : scan<T, 16>(a, p, stream);
        default: return grad ? scan_grad<T, 32>(a, p, stream) : scan<T, 32>(a, p, stream);
    }
}
hipError_t any_scan(const bps_scan& a, const ScanPlan& p, bool grad, hipStream_t stream) {
    return a.dtype == BPS_F32 ? scan_of<F32>(a, p, grad, stream) : a.dtype == BPS_BF16 ? scan_of<Bf16>(a, p, grad, stream) : scan_of<F16>(a, p, grad, stream);
}

}  // namespace

size_t scan_workspace(const bps_scan& a) { return chunk_floats(a, plan_of(a)) * sizeof(float); }

hipError_t launch_scan(const bps_scan& a, void* workspace, hipStream_t stream) {
    ScanPlan p = plan_of(a);
    place_chunks(a, p, static_cast<float*>(workspace));
    return any_scan(a, p, false, stream);
}

size_t scan_grad_workspace(const bps_scan& a) {
    const ScanPlan p = plan_of(a);
    return (whole(chunk_floats(a, p)) + whole((size_t)p.parts * (a.states + 2) * a.channels) +
            (size_t)p.tiles * a.batch * a.steps * a.groups * 2 * padded(a.states)) * sizeof(float);
}

hipError_t launch_scan_grad(const bps_scan& a, void* workspace, hipStream_t stream) {
    ScanPlan p = plan_of(a);
    float* space = static_cast<float*>(workspace);
    place_chunks(a, p, space);
    p.sums = space + whole(chunk_floats(a, p));
    p.shared = p.sums + whole((size_t)p.parts * (a.states + 2) * a.channels);
    return any_scan(a, p, true, stream);
}

}  // namespace bps
