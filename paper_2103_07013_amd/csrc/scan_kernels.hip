// Selective scan over time and its gradient (include/bps_memory.h states the rule).
//
// L lanes of a wavefront, 64 / L apart, hold a channel, a share of M of its states each in registers, and walk over time.  What is
// computed once for a step and a channel (the step's size, the gate) each of the L does for one of L steps, and hands it to the others;
// sums over the states of L steps are handed back the same way, so that no lane does another's work.  B and C are the same for
// the lanes of a share and come from LDS.  Where channels and sequences are too few to fill the card, the time is cut into chunks:
// a first pass finds what each chunk makes of states of zero and the sum of its steps, from which a second one finds the states
// at each chunk's beginning (the decays of a whole chunk are e^(A sum of d)), and the last one goes over all chunks at once.  The
// gradient does the same from the end to the beginning.
//
// What bounds it is the issue of vector instructions: a state's step is a product, a power of two, a product and two fused ones, five
// instructions of which the power takes two turns, against 8 bytes of a channel's step for all of its 16 states.  With four lanes to a channel
// 37 instructions are issued for 16 channels' step forward, 20 of them those five, and 106 for the gradient, where the least is 52;
// the units issue in 99 % of the cycles forward and 84 % in the gradient.  8 x 4096 x 2048 bf16, 16 states, all launches of a call, the time
// in four chunks: 490 us forward and 1255 for the gradient; eight lanes to a channel, as many chunks: 650 and 1715, one chunk 709 and 1474;
// one lane, which needs no exchange, in four times the chunks for as many wavefronts: 548 and 8990, where the gradient's registers go to memory.
#include <type_traits>

#include "memory_device.h"
#include "memory_kernels.h"

namespace bps {

namespace {

// Steps whose inputs are loaded together.  8 of them hold twice the states in memory: 8 x 4096 x 2048 bf16, 16 states, 582 us forward with
// held states and 1411 for the gradient, 495 and 1255 with 16.
constexpr int kTile = (int)kHeldSteps;
// Tiles whose sums over time the gradient adds up in registers; joining those in memory costs 1 or 2 %: 8 x 4096 x 2048 bf16 1268 us, 1024 x 32 x 512 float32
// 316, without it 1255, as in the comparisons of other choices here, and 309.
constexpr uint32_t kSumTiles = 16;

// A tensor of sequences as kernels have it.
struct Seq {
    void* at;
    int64_t batch;
    uint32_t step;
};

struct ScanArgs {
    Seq x, delta, gate, B, C, out, grad_out, grad_x, grad_delta, grad_gate, grad_B, grad_C;
    const float *A, *D, *delta_bias;
    bps_starts starts;
    const int32_t* lengths;
    const float* state;
    float* state_out;
    int64_t state_stride, state_out_stride;
    float* held;
    float *grad_A, *grad_D, *grad_delta_bias;
    uint32_t batch, steps, channels, states, groups;
    int32_t softplus;
    uint32_t waves, tiles;                // wavefronts of a work-group, of 64 / L channels each; work-groups for a group's channels
    uint32_t chunks, chunk_steps;
    uint32_t parts;                       // the gradient's work-groups that share the pieces of a tile among them
    float *ends, *spans;                  // [chunks][batch][states][channels], [chunks][batch][2][channels]: with more than one chunk
    float *sums, *shared;                 // the gradient's: [parts][states + 2][channels], [tiles][batch][steps][groups][2][L M]
};

// Where a lane is: its channel, whether that is one of its own, and which share of the states it holds.
struct Seat {
    uint32_t group, channel, share;
    bool on;
};
template <int L, int W>
__device__ __forceinline__ Seat seat_of(const ScanArgs& a, uint32_t tile) {
    constexpr uint32_t kLanes = 64 / L;
    const uint32_t each = a.channels / a.groups, group = tile / a.tiles, lane = threadIdx.x % 64;
    const uint32_t c = (tile % a.tiles * W + threadIdx.x / 64) * kLanes + lane % kLanes;
    return {group, group * each + min(c, each - 1), lane / kLanes, c < each};
}

// x, which the compiler takes for a new value: what follows from it is computed where it is used and not kept in registers for a whole
// loop, and a 32-bit place of a lane stays one, beside an address that all lanes share.
__device__ __forceinline__ uint32_t here(uint32_t x) {
    __asm__ volatile("" : "+v"(x));
    return x;
}

// A sequence's rows as a lane meets them: where a tile's rows begin is the same for all lanes, where in them a lane's elements lie
// fits 32 bits, in bytes.
template <class Raw, int L>
struct Rows {
    char* row;
    uint32_t step, mine;                  // from row to row; the lane's channel in the row of its share
    __device__ __forceinline__ Rows(const Seq& s, uint32_t b, int64_t t, const Seat& at)
        : row(static_cast<char*>(s.at) + (b * s.batch + t * s.step) * (int64_t)sizeof(Raw)), step(s.step * sizeof(Raw)), mine(at.channel * sizeof(Raw) + at.share * step) {}
    // of the lane's step among those from j L on
    __device__ __forceinline__ Raw& operator()(int j) const { return *reinterpret_cast<Raw*>(row + (here(mine) + j * L * step)); }
    // of a step of the tile
    __device__ __forceinline__ Raw& of(uint32_t s, const Seat& at) const { return *reinterpret_cast<Raw*>(row + (here(at.channel * sizeof(Raw)) + s * step)); }
    __device__ __forceinline__ void go(int tiles) { row += (int64_t)tiles * kTile * step; }
};

// A lane's inputs of kTile steps: those of steps j L + its share.  Steps behind the last of `left` read as that one.
template <class T, int L>
struct Inputs {
    typename T::raw v[kTile / L];
    __device__ __forceinline__ void load(const Rows<const typename T::raw, L>& s, int left, const Seat& at) {
        if (left >= kTile) {
#pragma unroll
            for (int j = 0; j < kTile / L; ++j) v[j] = s(j);
        } else {
#pragma unroll
            for (int j = 0; j < kTile / L; ++j) v[j] = s.of(min(L * j + (int)at.share, left - 1), at);
        }
    }
    __device__ __forceinline__ float operator[](int j) const { return to_float(v[j]); }
};

// B and C of kTile steps, a work-group's threads' parts of them on their way to LDS as float32, [step][B of L M states, C of L M
// states]; those of states that there are not are 0.
template <class T, int L, int M, int W>
struct Shared {
    static constexpr int kStates = L * M, kRow = 2 * kStates, kThreads = 64 * W, kMost = (kTile * kStates + kThreads - 1) / kThreads;
    typename T::raw v[2][kMost];
    const char* row[2];
    __device__ __forceinline__ Shared(const ScanArgs& a, uint32_t b, int64_t t, uint32_t group) {
#pragma unroll
        for (int of = 0; of < 2; ++of) {
            const Seq& s = of ? a.C : a.B;
            row[of] = static_cast<const char*>(s.at) + (b * s.batch + t * s.step + group * a.states) * (int64_t)sizeof(v[0][0]);
        }
    }
    __device__ __forceinline__ void load(const ScanArgs& a, int left) {
#pragma unroll
        for (int of = 0; of < 2; ++of)
#pragma unroll
            for (int e = 0; e < kMost; ++e) {
                const uint32_t i = e * kThreads + threadIdx.x;
                const uint32_t at = (min((int)(i / kStates), min(left, kTile) - 1) * (of ? a.C : a.B).step + min(i % kStates, a.states - 1)) * sizeof(v[0][0]);
                v[of][e] = *reinterpret_cast<const typename T::raw*>(row[of] + here(at));
            }
    }
    __device__ __forceinline__ void store(const ScanArgs& a, float (*to)[kRow]) const {
#pragma unroll
        for (int of = 0; of < 2; ++of)
#pragma unroll
            for (int e = 0; e < kMost; ++e) {
                const uint32_t i = e * kThreads + threadIdx.x;
                if (i < kTile * kStates) to[i / kStates][of * kStates + i % kStates] = i % kStates < a.states ? to_float(v[of][e]) : 0.0f;
            }
    }
    __device__ __forceinline__ void go(const ScanArgs& a, int tiles) {
        row[0] += (int64_t)tiles * kTile * a.B.step * (int64_t)sizeof(v[0][0]);
        row[1] += (int64_t)tiles * kTile * a.C.step * (int64_t)sizeof(v[0][0]);
    }
};

// Which of kTile steps begin an episode, a bit each.
__device__ __forceinline__ uint32_t load_starts(const bps_starts& s, uint32_t b, int64_t t, int left) {
    if (!s.at) return 0;
    const int lane = threadIdx.x % 64;
    return (uint32_t)__ballot(lane < min(kTile, left) && s.at[b * s.batch_stride + (t + min(lane, left - 1)) * s.step_stride]);
}

// Where state n of a lane's channel lies in [states][channels] floats, in bytes.
__device__ __forceinline__ uint32_t state_place(const ScanArgs& a, const Seat& at, uint32_t n) { return here((n * a.channels + at.channel) * 4); }

// A lane's states of [states][channels] floats, 0 for those that there are not and where there is no s.
template <int M>
__device__ __forceinline__ void load_states(const float* s, const ScanArgs& a, const Seat& at, float (&h)[M]) {
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const uint32_t n = at.share * M + m;
        h[m] = 0.0f;
        if (s && n < a.states) h[m] = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(s) + state_place(a, at, n));
    }
}
// Rates below -1e38, -infinity among them, count as that, whose decays are zero as well: over a step without a size, as those behind a
// sequence's end are, a state has to stay, and infinity times nothing is not a number.
__device__ __forceinline__ float finite(float rate) { return rate < -1e38f ? -1e38f : rate; }
template <int M>
__device__ __forceinline__ void load_rates(const ScanArgs& a, const Seat& at, float (&rate)[M], float factor = 1.0f) {
    load_states<M>(a.A, a, at, rate);
#pragma unroll
    for (int m = 0; m < M; ++m) rate[m] = finite(rate[m]) * factor;
}
template <int M>
__device__ __forceinline__ void store_states(float* s, const ScanArgs& a, const Seat& at, const float (&h)[M]) {
    if (!s || !at.on) return;
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const uint32_t n = at.share * M + m;
        if (n < a.states) *reinterpret_cast<float*>(reinterpret_cast<char*>(s) + state_place(a, at, n)) = h[m];
    }
}

// x and y with the upper half of x's 2 S lanes and the lower half of y's exchanged.
template <int S>
__device__ __forceinline__ void exchange(float& x, float& y) {
    const uint32_t p = __float_as_uint(x), q = __float_as_uint(y);
    if constexpr (S == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(p, q, false, false);
        x = __uint_as_float(r[0]), y = __uint_as_float(r[1]);
    } else if constexpr (S == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(p, q, false, false);
        x = __uint_as_float(r[0]), y = __uint_as_float(r[1]);
    } else {
        // moves by S lanes within 16, written to every other one of the banks of four lanes, or pair of them
        static_assert(S == 8 || S == 4, "banks have four lanes");
        constexpr int kUpper = S == 8 ? 0xC : 0xA;
        x = __uint_as_float(__builtin_amdgcn_update_dpp(p, q, 0x110 + S, 0xF, kUpper, false));
        y = __uint_as_float(__builtin_amdgcn_update_dpp(q, p, 0x100 + S, 0xF, 0xF - kUpper, false));
    }
}
// Sums over both halves of 2 S lanes: of x in the lower one, of y in the upper one.
template <int S>
__device__ __forceinline__ float pair_sum(float x, float y) {
    if constexpr (S >= 4) {
        exchange<S>(x, y);
        return x + y;
    } else {
        // a permutation within four lanes that turns over bit S, and none above it
        const bool upper = threadIdx.x & S;
        return (upper ? y : x) + from_lane_xor<2 * S - 1>(upper ? x : y);
    }
}

// What the L shares hold, to all of them: v[k] is share k's.
template <int L, int S = 32>
__device__ __forceinline__ void to_all(float x, float* v) {
    if constexpr (L == 1) {
        v[0] = x;
    } else {
        float y = x;
        exchange<S>(x, y);
        to_all<L / 2, S / 2>(x, v);
        to_all<L / 2, S / 2>(y, v + L / 2);
    }
}
// Share k gets the sum of v[k] over the shares.
template <int L, int S = 32>
__device__ __forceinline__ float to_own(const float* v) {
    if constexpr (L == 1) {
        return v[0];
    } else {
        float half[L / 2];
#pragma unroll
        for (int k = 0; k < L / 2; ++k) half[k] = pair_sum<S>(v[k], v[k + L / 2]);
        return to_own<L / 2, S / 2>(half);
    }
}
// The sum of x over the shares, to all of them.
template <int L, int S = 32>
__device__ __forceinline__ float share_sum(float x) {
    if constexpr (L == 1)
        return x;
    else
        return share_sum<L / 2, S / 2>(pair_sum<S>(x, x));
}

// The sums over the 2 S lanes of a share of each of K values: lane i of them gets that of value i K / (2 S).
template <int K, int S>
__device__ __forceinline__ float lane_sums(const float* v) {
    if constexpr (K > 1) {
        float half[K / 2];
#pragma unroll
        for (int k = 0; k < K / 2; ++k) half[k] = pair_sum<S>(v[k], v[k + K / 2]);
        return lane_sums<K / 2, S / 2>(half);
    } else {
        static_assert(S < 8, "as many values as halve 16 lanes once, or more");
        float x = v[0];
        if constexpr (S >= 4) x += from_lane_xor<7>(x);
        if constexpr (S >= 2) x += from_lane_xor<3>(x);
        if constexpr (S >= 1) x += from_lane_xor<1>(x);
        return x;
    }
}

// The sums of four steps over the 16 lanes of a share, of 8 values in each lane, by way of LDS: a lane adds up what 8 lanes have of four
// of them, and the two that have the same four exchange.  8 additions and exchanges a step where permutations of lanes take 30: the
// gradient of 8 x 4096 x 2048 bf16, 16 states, takes 1360 us with those and 1255 so, all launches.
struct LaneSums {
    static constexpr int kSteps = 4;
    static constexpr uint32_t kHalf = 64 * 4 + 16, kStep = 2 * kHalf, kWave = kSteps * kStep;      // floats; 16 of them keep halves in different banks
    float* space;                         // kWave floats of the wavefront's own
    // where the fours of lane i of a share lie: a lane's writes, and reads of all shares, meet different banks
    static __device__ __forceinline__ uint32_t place(uint32_t share, uint32_t i) { return (i * 4 + (share ^ (i >> 1 & 3))) * 4; }
    __device__ __forceinline__ void put(int step, const float (&v)[8]) const {
        const uint32_t lane = threadIdx.x % 64;
        float* p = space + step * kStep + place(lane / 16, lane % 16);
        typedef float Four __attribute__((ext_vector_type(4)));
        *reinterpret_cast<Four*>(p) = Four{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<Four*>(p + kHalf) = Four{v[4], v[5], v[6], v[7]};
    }
    // of step lane / 8 % 4 and share lane % 4: values 4 (lane / 4 % 2) + 2 (lane / 32) and the next
    __device__ __forceinline__ void get(float (&sums)[2]) const {
        typedef float Four __attribute__((ext_vector_type(4)));
        const uint32_t lane = threadIdx.x % 64, share = lane % 4;
        const float* p = space + lane / 8 % 4 * kStep + lane / 4 % 2 * kHalf;
        Four sum{};
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const Four x = *reinterpret_cast<const Four*>(p + place(share, lane / 32 * 8 + i));
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = i ? sum[e] + x[e] : x[e];
        }
        sums[0] = pair_sum<32>(sum[0], sum[2]), sums[1] = pair_sum<32>(sum[1], sum[3]);
    }
};

// What a wavefront wrote to LDS can be read by all of its lanes, whose accesses are in order there.
__device__ __forceinline__ void in_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Nothing is moved across this: left alone, the compiler would have all of a tile's loads from LDS on their way at once, in as many
// registers.
__device__ __forceinline__ void apart() {
    __asm__ volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// What a work-group works on: a chunk of a sequence.
struct Piece {
    uint32_t b, chunk;
    int64_t first, last, length, end;     // steps of the chunk, of the sequence, and the chunk's end within the sequence
    __device__ __forceinline__ Piece(const ScanArgs& a, uint32_t part, uint32_t chunks, uint32_t from = 0) {
        chunk = part % chunks + from, b = part / chunks;
        first = (int64_t)chunk * a.chunk_steps, last = min(first + a.chunk_steps, (int64_t)a.steps);
        length = steps_of(a.lengths, b, a.steps), end = min(last, length);
    }
    __device__ __forceinline__ uint64_t cell(const ScanArgs& a) const { return (uint64_t)chunk * a.batch + b; }
    __device__ __forceinline__ int64_t top() const { return first + (end - first - 1) / kTile * kTile; }      // the last tile's first step
};

// Step sizes of a lane's steps, 0 from `left` on.
template <class T, int L>
__device__ __forceinline__ void step_sizes(const Inputs<T, L>& delta, float bias, bool soft, int left, const Seat& at, float (&d)[kTile / L]) {
#pragma unroll
    for (int j = 0; j < kTile / L; ++j) d[j] = delta[j] + bias;
    if (soft) {
#pragma unroll
        for (int j = 0; j < kTile / L; ++j) d[j] = softplus(d[j]);
    }
    if (left < kTile) {
#pragma unroll
        for (int j = 0; j < kTile / L; ++j) d[j] = L * j + (int)at.share < left ? d[j] : 0.0f;
    }
}

// f of std::true_type where `some`, else of std::false_type
template <class F>
__device__ __forceinline__ void either(bool some, F f) {
    if (some)
        f(std::true_type());
    else
        f(std::false_type());
}

// FIRST: what each chunk makes of states of zero, and its steps' sum.  Otherwise the outputs.  The next tile's inputs are on their way while
// a tile is gone through.  16384 steps of 2048 channels, bf16, 16 states: 125 us and 170 us, the units issuing all the time; 1024 x 32 x 512
// float32: 109 us, 3.8 TB/s.
template <class T, int L, int M, int W, bool FIRST>
__global__ __launch_bounds__(64 * W) void k_scan(const ScanArgs a) {
    using raw = typename T::raw;
    constexpr int kRow = Shared<T, L, M, W>::kRow, kOwn = kTile / L;
    __shared__ float shared[2][kTile][kRow];
    const uint32_t all_tiles = a.tiles * a.groups;
    // the last chunk's end is nothing that another one begins with
    const Piece w(a, blockIdx.x / all_tiles, FIRST ? a.chunks - 1 : a.chunks);
    const Seat at = seat_of<L, W>(a, blockIdx.x % all_tiles);
    const uint32_t b = w.b, c = at.channel;
    float h[M], rate[M];
    load_rates<M>(a, at, rate, kLog2e);
    const float bias = a.delta_bias ? a.delta_bias[c] : 0.0f, skip = !FIRST && a.D ? a.D[c] : 0.0f;
    if constexpr (FIRST)
        load_states<M>(nullptr, a, at, h);
    else
        load_states<M>(a.chunks > 1 ? a.ends + w.cell(a) * a.states * a.channels : a.state ? a.state + b * a.state_stride : nullptr, a, at, h);
    float span = 0.0f, keeps = 1.0f;
    Rows<const raw, L> x_rows(a.x, b, w.first, at), delta_rows(a.delta, b, w.first, at), gate_rows(a.gate, b, w.first, at);
    Rows<raw, L> out_rows(a.out, b, w.first, at);
    float* held = FIRST || !a.held ? nullptr : a.held + ((uint64_t)b * ((a.steps + kTile - 1) / kTile) + w.first / kTile) * a.states * a.channels;
    Inputs<T, L> next_x, next_delta, next_gate;
    Shared<T, L, M, W> next_shared(a, b, w.first, at.group);
    uint32_t next_starts = 0;
    auto load = [&](int64_t t) {
        const int left = (int)(w.end - t);
        next_x.load(x_rows, left, at);
        next_delta.load(delta_rows, left, at);
        if (!FIRST && a.gate.at) next_gate.load(gate_rows, left, at);
        next_shared.load(a, left);
        next_starts = load_starts(a.starts, b, t, left);
        x_rows.go(1), delta_rows.go(1), gate_rows.go(1), next_shared.go(a, 1);
    };
    if (w.first < w.end) load(w.first);
    int turn = 0;
    for (int64_t t = w.first; t < w.end; t += kTile, turn ^= 1) {
        const uint32_t starts = next_starts;
        const int left = (int)(w.end - t), rest = (int)(w.last - t);
        float d_mine[kOwn], x_mine[kOwn], f_mine[kOwn];
        next_shared.store(a, shared[turn]);
        step_sizes<T, L>(next_delta, bias, a.softplus, left, at, d_mine);
#pragma unroll
        for (int j = 0; j < kOwn; ++j) x_mine[j] = next_x[j], f_mine[j] = 1.0f;
        if (left < kTile) {
            // steps behind the end leave the states as they are
#pragma unroll
            for (int j = 0; j < kOwn; ++j) x_mine[j] = L * j + (int)at.share < left ? x_mine[j] : 0.0f;
        }
        if (!FIRST && a.gate.at) {
#pragma unroll
            for (int j = 0; j < kOwn; ++j) f_mine[j] = next_gate[j] * sigmoid(next_gate[j]);
        }
        __syncthreads();
        if (t + kTile < w.end) load(t + kTile);
        if (held) {
            store_states<M>(held, a, at, h);
            held += (uint64_t)a.states * a.channels;
        }
        either(starts, [&](auto some) {
#pragma unroll
            for (int j = 0; j < kOwn; ++j) {
                apart();
                if (L * j >= left) {      // nothing but zeros behind the end
                    if (!FIRST && at.on && L * j + (int)at.share < rest) out_rows(j) = rounded<T>(0.0f);
                    continue;
                }
                float d[L], in[L], y[L];
                to_all<L>(d_mine[j], d);
                to_all<L>(d_mine[j] * x_mine[j], in);
                span += d_mine[j];
#pragma unroll
                for (int k = 0; k < L; ++k) {
                    const float* bc = &shared[turn][L * j + k][at.share * M];
                    if (decltype(some)::value && (starts >> (L * j + k) & 1)) {
                        keeps = 0.0f;
#pragma unroll
                        for (int m = 0; m < M; ++m) h[m] = 0.0f;
                    }
                    y[k] = 0.0f;
#pragma unroll
                    for (int m = 0; m < M; ++m) {
                        h[m] = __builtin_fmaf(h[m], __builtin_amdgcn_exp2f(d[k] * rate[m]), in[k] * bc[m]);
                        if constexpr (!FIRST) y[k] = m ? __builtin_fmaf(h[m], bc[kRow / 2 + m], y[k]) : h[m] * bc[kRow / 2 + m];
                    }
                }
                if constexpr (!FIRST) {
                    const int mine = L * j + (int)at.share;
                    const float sum = __builtin_fmaf(skip, x_mine[j], to_own<L>(y)) * f_mine[j];
                    if (at.on && mine < rest) out_rows(j) = rounded<T>(mine < left ? sum : 0.0f);
                }
            }
        });
        out_rows.go(1);
    }
    if constexpr (FIRST) {
        store_states<M>(a.ends + w.cell(a) * a.states * a.channels, a, at, h);
        span = share_sum<L>(span);
        if (at.on && at.share == 0) {
            a.spans[w.cell(a) * 2 * a.channels + c] = span;
            a.spans[(w.cell(a) * 2 + 1) * a.channels + c] = keeps;
        }
    } else {
        if (w.chunk == a.chunks - 1) store_states<M>(a.state_out ? a.state_out + b * a.state_out_stride : nullptr, a, at, h);
        for (int64_t t = w.first < w.end ? w.top() + kTile : w.first; t < w.last; t += kTile, out_rows.go(1))
#pragma unroll
            for (int j = 0; j < kOwn; ++j)
                if (at.on && t + L * j + at.share < w.last) out_rows(j) = rounded<T>(0.0f);
    }
}

// One step of every sequence, whose states are what is read and written: a lane holds four channels of every fourth state, a row of 256
// channels to a wavefront, so that all of a lane's loads of 16 bytes are on their way at once; the wavefronts' sums meet in LDS.  Bound by memory:
// 1024 x 512 float32 with 16 states 14.5 us, 5.2 TB/s, 192 x 4096 bf16 23 us, 4.6 TB/s (28 and 40 us by the kernel for sequences).
template <class T, int M>
__global__ __launch_bounds__(256) void k_scan_step(const ScanArgs a) {
    using raw = typename T::raw;
    constexpr uint32_t kChannels = 256;
    __shared__ __attribute__((aligned(16))) float sizes[kChannels], inputs[kChannels], sums[4][kChannels];
    const uint32_t each = a.channels / a.groups, tiles = (each + kChannels - 1) / kChannels, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const uint32_t tile = blockIdx.x % tiles, group = blockIdx.x / tiles % a.groups, b = blockIdx.x / tiles / a.groups;
    const uint32_t base = group * each, left = each - tile * kChannels;                     // of the group, and its channels from this tile on
    const uint32_t four = lane * 4, n4 = four < left ? left - four : 0, c4 = base + tile * kChannels + (n4 ? four : 0);
    const bool on = steps_of(a.lengths, b, 1), begins = on && a.starts.at && a.starts.at[b * a.starts.batch_stride];
    float h[M][4], rate[M][4], write[M], read[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const uint32_t n = m * 4 + wave;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[m][e] = rate[m][e] = 0.0f;
        write[m] = read[m] = 0.0f;
        if (n < a.states) {
            if (a.state && !begins) load_part<F32, 4>(a.state + b * a.state_stride + (uint64_t)n * a.channels + c4, n4, h[m]);
            load_part<F32, 4>(a.A + (uint64_t)n * a.channels + c4, n4, rate[m]);
            if (on) {
                write[m] = to_float((static_cast<const raw*>(a.B.at) + b * a.B.batch)[group * a.states + n]);
                read[m] = to_float((static_cast<const raw*>(a.C.at) + b * a.C.batch)[group * a.states + n]);
            }
        }
    }
    const uint32_t c = base + tile * kChannels + threadIdx.x;
    const bool mine = threadIdx.x < left && on;
    float x = 0.0f, d = 0.0f, f = 1.0f;
    if (mine) {
        x = to_float((static_cast<const raw*>(a.x.at) + b * a.x.batch)[c]);
        d = to_float((static_cast<const raw*>(a.delta.at) + b * a.delta.batch)[c]) + (a.delta_bias ? a.delta_bias[c] : 0.0f);
        if (a.gate.at) f = to_float((static_cast<const raw*>(a.gate.at) + b * a.gate.batch)[c]);
    }
    const float skip = mine && a.D ? a.D[c] : 0.0f;
    if (a.softplus && mine) d = softplus(d);
    sizes[threadIdx.x] = d;
    inputs[threadIdx.x] = d * x;
    __syncthreads();
    float y[4] = {};
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const uint32_t n = m * 4 + wave;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[m][e] = __builtin_fmaf(h[m][e], __builtin_amdgcn_exp2f(sizes[four + e] * (finite(rate[m][e]) * kLog2e)), inputs[four + e] * write[m]);
            y[e] = __builtin_fmaf(h[m][e], read[m], y[e]);
        }
        if (n < a.states && a.state_out) store_part<F32, 4>(a.state_out + b * a.state_out_stride + (uint64_t)n * a.channels + c4, n4, h[m]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[wave][four + e] = y[e];
    __syncthreads();
    if (threadIdx.x >= left) return;
    float sum = skip * x;
#pragma unroll
    for (int k = 0; k < 4; ++k) sum += sums[k][threadIdx.x];
    if (a.gate.at) sum *= f * sigmoid(f);
    (static_cast<raw*>(a.out.at) + b * a.out.batch)[c] = rounded<T>(on ? sum : 0.0f);
}

// What the first pass left of each chunk but the last becomes what the next one begins with: REVERSE from the last chunk to the first,
// with nothing behind the last.
template <bool REVERSE>
__global__ __launch_bounds__(256) void k_scan_join(const ScanArgs a) {
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x, per = (uint64_t)a.states * a.channels;
    if (id >= a.batch * per) return;
    const uint32_t b = (uint32_t)(id / per), c = (uint32_t)(id % a.channels);
    const float rate = finite(a.A[id % per]) * kLog2e;
    float h = !REVERSE && a.state ? a.state[b * a.state_stride + id % per] : 0.0f;
    constexpr uint32_t kAhead = 8;        // chunks whose inputs are on their way together
    for (uint32_t i = 0; i < a.chunks; i += kAhead) {
        float end[kAhead], span[kAhead], keeps[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) {
            const uint32_t n = min(i + k, a.chunks - 1);
            const uint64_t cell = (uint64_t)(REVERSE ? a.chunks - 1 - n : n) * a.batch + b;
            end[k] = span[k] = keeps[k] = 0.0f;
            if (n < a.chunks - 1) end[k] = a.ends[cell * per + id % per], span[k] = a.spans[cell * 2 * a.channels + c], keeps[k] = a.spans[(cell * 2 + 1) * a.channels + c];
        }
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) {
            if (i + k >= a.chunks) break;
            a.ends[((uint64_t)(REVERSE ? a.chunks - 1 - i - k : i + k) * a.batch + b) * per + id % per] = h;
            // Where states grow, a chunk's growth may be over what a float32 holds and the state behind it not: its root is applied
            // twice, and a state of zero stays one under a growth of any size, as it does step by step.
            const float root = __builtin_amdgcn_exp2f(span[k] * rate * 0.5f);
            h = keeps[k] != 0.0f && h != 0.0f ? __builtin_fmaf(h * root, root, end[k]) : end[k];
        }
    }
}

// What reaches the states in front of each chunk of what is behind its last step: zero there.
template <class T, int L, int M, int W>
__global__ __launch_bounds__(64 * W) void k_scan_grad_first(const ScanArgs a) {
    using raw = typename T::raw;
    constexpr int kRow = Shared<T, L, M, W>::kRow, kOwn = kTile / L;
    __shared__ float shared[2][kTile][kRow];
    const uint32_t all_tiles = a.tiles * a.groups;
    // nothing reaches the steps in front of the first chunk
    const Piece w(a, blockIdx.x / all_tiles, a.chunks - 1, 1);
    const Seat at = seat_of<L, W>(a, blockIdx.x % all_tiles);
    const uint32_t b = w.b, c = at.channel;
    float g[M] = {}, rate[M];
    load_rates<M>(a, at, rate, kLog2e);
    const float bias = a.delta_bias ? a.delta_bias[c] : 0.0f;
    float span = 0.0f, keeps = 1.0f;
    const int64_t top = w.top();
    Rows<const raw, L> delta_rows(a.delta, b, top, at), gate_rows(a.gate, b, top, at), grad_rows(a.grad_out, b, top, at);
    Inputs<T, L> next_delta, next_gate, next_grad;
    Shared<T, L, M, W> next_shared(a, b, top, at.group);
    uint32_t next_starts = 0;
    auto load = [&](int64_t t) {
        const int left = (int)(w.end - t);
        next_delta.load(delta_rows, left, at);
        next_grad.load(grad_rows, left, at);
        if (a.gate.at) next_gate.load(gate_rows, left, at);
        next_shared.load(a, left);
        next_starts = load_starts(a.starts, b, t, left);
        delta_rows.go(-1), grad_rows.go(-1), gate_rows.go(-1), next_shared.go(a, -1);
    };
    if (w.first < w.end) load(top);
    int turn = 0;
    for (int64_t t = top; t >= w.first && w.first < w.end; t -= kTile, turn ^= 1) {
        const uint32_t starts = next_starts;
        const int left = (int)(w.end - t);
        float d_mine[kOwn], dy_mine[kOwn];
        next_shared.store(a, shared[turn]);
        step_sizes<T, L>(next_delta, bias, a.softplus, left, at, d_mine);
#pragma unroll
        for (int j = 0; j < kOwn; ++j) dy_mine[j] = next_grad[j];
        if (a.gate.at) {
#pragma unroll
            for (int j = 0; j < kOwn; ++j) dy_mine[j] *= next_gate[j] * sigmoid(next_gate[j]);
        }
        if (left < kTile) {
#pragma unroll
            for (int j = 0; j < kOwn; ++j) dy_mine[j] = L * j + (int)at.share < left ? dy_mine[j] : 0.0f;
        }
        __syncthreads();
        if (t > w.first) load(t - kTile);
        either(starts, [&](auto some) {
#pragma unroll
            for (int j = kOwn - 1; j >= 0; --j) {
                apart();
                if (L * j >= left) continue;
                float d[L], dy[L];
                to_all<L>(d_mine[j], d);
                to_all<L>(dy_mine[j], dy);
                span += d_mine[j];
#pragma unroll
                for (int k = L - 1; k >= 0; --k) {
                    const float* bc = &shared[turn][L * j + k][at.share * M];
#pragma unroll
                    for (int m = 0; m < M; ++m) g[m] = __builtin_fmaf(bc[kRow / 2 + m], dy[k], g[m]) * __builtin_amdgcn_exp2f(d[k] * rate[m]);
                    if (decltype(some)::value && (starts >> (L * j + k) & 1)) {
                        keeps = 0.0f;
#pragma unroll
                        for (int m = 0; m < M; ++m) g[m] = 0.0f;
                    }
                }
            }
        });
    }
    store_states<M>(a.ends + w.cell(a) * a.states * a.channels, a, at, g);
    span = share_sum<L>(span);
    if (at.on && at.share == 0) {
        a.spans[w.cell(a) * 2 * a.channels + c] = span;
        a.spans[(w.cell(a) * 2 + 1) * a.channels + c] = keeps;
    }
}

// The gradient.  With dy = grad_out silu(gate) and g the gradient of the states behind a step,
//   g = C dy + (decay of the step behind) (g behind);   grad_C = sum over channels of dy h;   grad_B = sum over channels of g d x
//   grad_x = d sum of g B + D dy;   grad_d = x sum of g B + sum of A g a h before;   grad_A = sum over time of d g a h before
// kTile steps at a time from the last to the first: forward from the states held before them, with all of their states and decays kept
// in registers, then backward.  Sums over channels are sums over the lanes of a share, joined over the work-group's wavefronts in LDS
// and left for each tile of channels.  Decays of 16 steps of 4 states do not fit beside the states (registers that go to memory make all
// launches 2160 us instead of 1255): they are computed again.  8 x 4096 x 2048 bf16, 16 states: 1020 us in its work-groups of four
// wavefronts, two to a SIMD; 1024 x 32 x 512 float32 330 us.  In work-groups of one wavefront 9 to 16 states take 48 registers more than there are,
// 196 bytes of memory a lane (see args_of); no other form takes any.
template <class T, int L, int M, int W>
__global__ __launch_bounds__(64 * W, 2) void k_scan_grad(const ScanArgs a) {
    using raw = typename T::raw;
    constexpr int kRow = Shared<T, L, M, W>::kRow, kOwn = kTile / L;
    // decays of 4 states of a lane would leave no room for a second wavefront: they are computed again
    constexpr bool kKeep = M <= 2;
    __shared__ float shared[kTile][kRow];
    __shared__ float across[W][kTile][kRow];
    // sums over lanes by way of LDS
    constexpr bool kSpace = L == LaneSums::kSteps && M == 4;
    __shared__ __attribute__((aligned(16))) float space[kSpace ? W * 2 * LaneSums::kWave : 1];
    const uint32_t all_tiles = a.tiles * a.groups, tile = blockIdx.x % all_tiles, part = blockIdx.x / all_tiles;
    const Seat at = seat_of<L, W>(a, tile);
    const uint32_t c = at.channel, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    float rate[M], d_rate[M] = {};
    load_rates<M>(a, at, rate);
    const float bias = a.delta_bias ? a.delta_bias[c] : 0.0f, skip = a.D ? a.D[c] : 0.0f;
    float d_skip = 0.0f, d_bias = 0.0f;
    // The sums of kSumTiles tiles join those of the tiles before, in memory: one after another over all steps of a work-group their roundings would be
    // those of thousands of additions (64 x 512 x 512 float32, 4096 for each: grad_A 20 x 2^-24 off instead of 7).
    float* all_sums = a.sums + (uint64_t)part * (a.states + 2) * a.channels;
    uint32_t summed = 0;
    bool begun = false;
    auto leave = [&]() {
        float before[M];
        load_states<M>(begun && at.on ? all_sums : nullptr, a, at, before);
#pragma unroll
        for (int m = 0; m < M; ++m) d_rate[m] += before[m];
        store_states<M>(all_sums, a, at, d_rate);
        d_skip = share_sum<L>(d_skip), d_bias = share_sum<L>(d_bias);
        if (at.on && at.share == 0) {
            float* s = all_sums + a.states * (uint64_t)a.channels + c;
            s[0] = begun ? s[0] + d_skip : d_skip;
            s[a.channels] = begun ? s[a.channels] + d_bias : d_bias;
        }
#pragma unroll
        for (int m = 0; m < M; ++m) d_rate[m] = 0.0f;
        d_skip = d_bias = 0.0f, summed = 0, begun = true;
    };
    for (uint32_t item = part; item < a.batch * a.chunks; item += a.parts) {
        const Piece w(a, item, a.chunks);
        const uint32_t b = w.b;
        const int64_t top = w.first < w.end ? w.top() : w.first - kTile;
        Rows<const raw, L> x_rows(a.x, b, top, at), delta_rows(a.delta, b, top, at), gate_rows(a.gate, b, top, at), grad_rows(a.grad_out, b, top, at);
        Rows<raw, L> dx_rows(a.grad_x, b, top + kTile, at), dd_rows(a.grad_delta, b, top + kTile, at), dz_rows(a.grad_gate, b, top + kTile, at);
        for (int64_t t = top + kTile; t < w.last; t += kTile, dx_rows.go(1), dd_rows.go(1), dz_rows.go(1))
#pragma unroll
            for (int j = 0; j < kOwn; ++j)
                if (at.on && t + L * j + at.share < w.last) {
                    dx_rows(j) = dd_rows(j) = rounded<T>(0.0f);
                    if (a.gate.at) dz_rows(j) = rounded<T>(0.0f);
                }
        if (w.first >= w.end) continue;
        dx_rows = Rows<raw, L>(a.grad_x, b, top, at), dd_rows = Rows<raw, L>(a.grad_delta, b, top, at), dz_rows = Rows<raw, L>(a.grad_gate, b, top, at);
        Shared<T, L, M, W> next_shared(a, b, top, at.group);
        const float* held = a.held + ((uint64_t)b * ((a.steps + kTile - 1) / kTile) + top / kTile) * a.states * a.channels;
        float* sums = a.shared + ((((uint64_t)(tile % a.tiles) * a.batch + b) * a.steps + top) * a.groups + at.group) * kRow;
        float g[M];                       // of the states before the step behind
        // nothing for the lanes behind the last channel, which have no part in the sums over channels
        load_states<M>(a.chunks > 1 && at.on ? a.ends + w.cell(a) * a.states * a.channels : nullptr, a, at, g);
        Inputs<T, L> next_x, next_delta, next_gate, next_grad;
        float next_h[M];
        uint32_t next_starts = 0;
        auto load = [&](int64_t t) {
            const int left = (int)(w.end - t);
            next_x.load(x_rows, left, at);
            next_delta.load(delta_rows, left, at);
            next_grad.load(grad_rows, left, at);
            if (a.gate.at) next_gate.load(gate_rows, left, at);
            next_shared.load(a, left);
            load_states<M>(held, a, at, next_h);
            next_starts = load_starts(a.starts, b, t, left);
            x_rows.go(-1), delta_rows.go(-1), gate_rows.go(-1), grad_rows.go(-1), next_shared.go(a, -1);
            held -= (uint64_t)a.states * a.channels;
        };
        load(top);
        for (int64_t t = top; t >= w.first; t -= kTile) {
            if (summed == kSumTiles) leave();
            ++summed;
            const int left = (int)(w.end - t), rest = (int)(w.last - t);
            const uint32_t starts = next_starts;
            float h[kTile + 1][M], decay[kKeep ? kTile : 1][M];
            float d_mine[kOwn], x_mine[kOwn], dy_mine[kOwn], z_mine[kOwn], slope_mine[kOwn];
#pragma unroll
            for (int m = 0; m < M; ++m) h[0][m] = next_h[m];
            next_shared.store(a, shared);
            step_sizes<T, L>(next_delta, bias, a.softplus, left, at, d_mine);
#pragma unroll
            for (int j = 0; j < kOwn; ++j) {
                // steps behind the end leave states and gradients as they are
                const bool inside = L * j + (int)at.share < left;
                x_mine[j] = inside ? next_x[j] : 0.0f;
                dy_mine[j] = inside && at.on ? next_grad[j] : 0.0f;
                slope_mine[j] = inside ? 1.0f : 0.0f;
                z_mine[j] = next_gate[j];
            }
            if (a.softplus) {
#pragma unroll
                for (int j = 0; j < kOwn; ++j) slope_mine[j] *= sigmoid(next_delta[j] + bias);
            }
            if (left < kTile && a.gate.at) {
#pragma unroll
                for (int j = 0; j < kOwn; ++j) z_mine[j] = L * j + (int)at.share < left ? z_mine[j] : 0.0f;
            }
            __syncthreads();
            if (t > w.first) load(t - kTile);
            // the first kGo of the lane's steps, behind which the sequence ends: short ones have no more than a few
            auto walk = [&](auto some, auto go) {
                constexpr bool kSome = decltype(some)::value;
                constexpr int kGo = decltype(go)::value;
#pragma unroll
                for (int j = kGo; j < kOwn; ++j)
                    if (at.on && L * j + (int)at.share < rest) {
                        dx_rows(j) = dd_rows(j) = rounded<T>(0.0f);
                        if (a.gate.at) dz_rows(j) = rounded<T>(0.0f);
                    }
#pragma unroll
                for (int j = 0; j < kGo; ++j) {
                    apart();
                    const int mine = L * j + (int)at.share;
                    float d[L], in[L], y[L];
                    to_all<L>(d_mine[j], d);
                    to_all<L>(d_mine[j] * x_mine[j], in);
#pragma unroll
                    for (int k = 0; k < L; ++k) {
                        const int s = L * j + k;
                        const float* bc = &shared[s][at.share * M];
                        const bool begins = kSome && (starts >> s & 1);
                        y[k] = 0.0f;
#pragma unroll
                        for (int m = 0; m < M; ++m) {
                            const float f = __builtin_amdgcn_exp2f(d[k] * (rate[m] * kLog2e));
                            if constexpr (kKeep) decay[s][m] = f;
                            h[s + 1][m] = __builtin_fmaf(begins ? 0.0f : h[s][m], f, in[k] * bc[m]);
                            y[k] = m ? __builtin_fmaf(h[s + 1][m], bc[kRow / 2 + m], y[k]) : h[s + 1][m] * bc[kRow / 2 + m];
                        }
                    }
                    if (a.gate.at) {
                        const float z = z_mine[j], s = sigmoid(z), sum = __builtin_fmaf(skip, x_mine[j], to_own<L>(y));
                        if (at.on && mine < rest) dz_rows(j) = rounded<T>(dy_mine[j] * sum * silu_slope(z, s));
                        dy_mine[j] *= z * s;
                    }
                }
                // the sums over lanes of L steps, while the next ones are under way
                auto add_up = [&](int j) {
                    float sums_mine[2];
                    LaneSums{space + (wave * 2 + j % 2) * LaneSums::kWave}.get(sums_mine);
                    float* to = &across[wave][L * j + lane / 8 % 4][lane / 4 % 2 * (kRow / 2) + lane % 4 * M + lane / 32 * 2];
                    to[0] = sums_mine[0], to[1] = sums_mine[1];
                };
#pragma unroll
                for (int j = kGo - 1; j >= 0; --j) {
                    apart();
                    if constexpr (kSpace)
                        if (j + 1 < kGo) add_up(j + 1);
                    // handed out again rather than kept for all steps since the way forward
                    __asm__ volatile("" : "+v"(d_mine[j]), "+v"(x_mine[j]));
                    float d[L], in[L], dy[L], gb[L], dd[L];
                    to_all<L>(d_mine[j], d);
                    to_all<L>(d_mine[j] * x_mine[j], in);
                    to_all<L>(dy_mine[j], dy);
#pragma unroll
                    for (int k = L - 1; k >= 0; --k) {
                        const int s = L * j + k;
                        const float* bc = &shared[s][at.share * M];
                        const bool begins = kSome && (starts >> s & 1);
                        float both[2 * M];
#pragma unroll
                        for (int m = 0; m < M; ++m) {
                            g[m] = __builtin_fmaf(bc[kRow / 2 + m], dy[k], g[m]);
                            both[m] = g[m] * in[k];
                            both[M + m] = dy[k] * h[s + 1][m];
                            gb[k] = m ? __builtin_fmaf(g[m], bc[m], gb[k]) : g[m] * bc[m];
                            if constexpr (kKeep)
                                g[m] *= decay[s][m];
                            else
                                g[m] *= __builtin_amdgcn_exp2f(d[k] * (rate[m] * kLog2e));
                            if (begins) g[m] = 0.0f;
                            const float q = begins ? 0.0f : g[m] * h[s][m];
                            d_rate[m] = __builtin_fmaf(q, d[k], d_rate[m]);
                            dd[k] = m ? __builtin_fmaf(q, rate[m], dd[k]) : q * rate[m];
                        }
                        if constexpr (kSpace) {
                            LaneSums{space + (wave * 2 + j % 2) * LaneSums::kWave}.put(k, both);
                        } else {
                            const float sum = lane_sums<2 * M, 32 / L>(both);
                            constexpr uint32_t kLanes = 64 / L, kEach = kLanes / (2 * M);
                            const uint32_t v = lane % kLanes / kEach;
                            if (lane % kEach == 0) across[wave][s][v / M * (kRow / 2) + at.share * M + v % M] = sum;
                        }
                    }
                    if constexpr (kSpace) in_order();
                    const int mine = L * j + (int)at.share;
                    const float gb_mine = to_own<L>(gb);
                    const float dd_mine = __builtin_fmaf(gb_mine, x_mine[j], to_own<L>(dd)) * slope_mine[j];
                    d_skip = __builtin_fmaf(dy_mine[j], x_mine[j], d_skip);
                    d_bias += dd_mine;
                    if (at.on && mine < rest) {
                        dx_rows(j) = rounded<T>(__builtin_fmaf(d_mine[j], gb_mine, skip * dy_mine[j]));
                        dd_rows(j) = rounded<T>(dd_mine);
                    }
                }
                if constexpr (kSpace) add_up(0);
            };
            either(starts, [&](auto some) {
                if (left <= L)
                    walk(some, std::integral_constant<int, 1>());
                else if (kOwn > 2 && left <= 2 * L)
                    walk(some, std::integral_constant<int, 2>());
                else
                    walk(some, std::integral_constant<int, kOwn>());
            });
            __syncthreads();
#pragma unroll
            for (uint32_t i = threadIdx.x; i < kTile * kRow; i += 64 * W) {
                float sum = across[0][i / kRow][i % kRow];
#pragma unroll
                for (int k = 1; k < W; ++k) sum += across[k][i / kRow][i % kRow];
                if ((int)(i / kRow) < left) sums[(uint64_t)(i / kRow) * a.groups * kRow + i % kRow] = sum;
            }
            dx_rows.go(-1), dd_rows.go(-1), dz_rows.go(-1);
            sums -= (uint64_t)kTile * a.groups * kRow;
        }
    }
    leave();
}

// grad_B and grad_C: the sums of all tiles of a group, zero behind a sequence's end.
template <class T, int P>
__global__ __launch_bounds__(256) void k_scan_grad_shared(const ScanArgs a) {
    using raw = typename T::raw;
    constexpr uint32_t kRow = 2 * P;
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x, row = id / kRow, size = (uint64_t)a.batch * a.steps * a.groups;
    const uint32_t i = id % kRow, n = i % P;
    if (row >= size || n >= a.states) return;
    const uint32_t group = (uint32_t)(row % a.groups), b = (uint32_t)(row / a.groups / a.steps);
    const int64_t t = (int64_t)(row / a.groups % a.steps);
    float sum = 0.0f;
    if (t < steps_of(a.lengths, b, a.steps))
        for (uint32_t k = 0; k < a.tiles; ++k) sum += a.shared[(k * size + row) * kRow + i];
    const Seq& s = i < P ? a.grad_B : a.grad_C;
    (static_cast<raw*>(s.at) + b * s.batch + t * s.step)[group * a.states + n] = rounded<T>(sum);
}

// Work-groups that a launch has, where there is time to be cut for as many, forward and in the gradient: 256 / 512 / 768 / 1024 / 1536, 16 states
// bf16, all launches: 8 x 4096 x 2048 585 / 554 / 500 / 490 / 485 and 1632 / 1282 / 1362 / 1255 / 1263 us, 16384 x 2048 480 / 320 / 292 / 277 / 275 and
// 1030 / 691 / 730 / 670 / 682.
constexpr uint32_t kGroups = 1024;
constexpr uint32_t kParts = 1024;         // work-groups of the gradient: 512 are on the card at a time
constexpr uint32_t kLeast = 64;           // steps of a chunk

// states that the kernels have room for
uint32_t room(uint32_t states) { return states <= 4 ? 4 : states <= 8 ? 8 : states <= 16 ? 16 : 32; }

// Lanes of a channel, as scan_of chooses them.
uint32_t lanes_of(uint32_t states, bool grad) { return grad && states > 16 ? 8 : 4; }

ScanArgs args_of(const bps_scan& s, bool grad) {
    auto seq = [](const bps_sequence& q) { return Seq{q.at, q.batch_stride, (uint32_t)q.step_stride}; };
    ScanArgs a{seq(s.x), seq(s.delta), seq(s.gate), seq(s.B), seq(s.C), seq(s.out), seq(s.grad_out), seq(s.grad_x), seq(s.grad_delta), seq(s.grad_gate), seq(s.grad_B), seq(s.grad_C),
               s.A, s.D, s.delta_bias, s.starts, s.lengths, s.state, s.state_out, s.state_stride, s.state_out_stride, s.held, s.grad_A, s.grad_D, s.grad_delta_bias,
               s.batch, s.steps, s.channels, s.states, s.groups, s.softplus, 0, 0, 0, 0, 0, nullptr, nullptr, nullptr, nullptr};
    // work-groups of 64 channels, or of one wavefront where a quarter of their wavefronts or more would have none: 1623 x 3 x 20 bf16, 32 states in
    // 4 groups, scan and gradient, 72 us instead of 226; 1817 x 14 x 71 with 4 / 8 / 32 states 63 / 75 / 159 instead of 71 / 84 / 210.  With 9 to 16
    // states, where registers of the gradient go to memory so, 145 instead of 108, and 2048 x 32 x 24 118 instead of 113
    const uint32_t lanes = lanes_of(s.states, grad), channels = a.channels / a.groups, wide = (channels + 63) / 64, narrow = (channels * lanes + 63) / 64;
    a.waves = narrow * 4 > wide * lanes * 3 ? lanes : 1;
    a.tiles = a.waves == 1 ? narrow : wide;
    const uint64_t groups = (uint64_t)a.batch * a.tiles * a.groups, most_groups = a.waves == 1 ? kGroups * lanes : kGroups;
    const uint64_t want = groups ? most_groups / groups : 1, most = a.steps / kLeast;
    const uint32_t chunks = (uint32_t)(want < most ? want : most);
    a.chunk_steps = chunks > 1 ? ((a.steps + chunks - 1) / chunks + kTile - 1) / kTile * kTile : a.steps ? a.steps : 1;
    a.chunks = a.steps ? (a.steps + a.chunk_steps - 1) / a.chunk_steps : 1;
    const uint64_t items = (uint64_t)a.batch * a.chunks, part = (a.waves == 1 ? kParts * lanes : kParts) / (a.tiles * a.groups);
    a.parts = (uint32_t)(items < part ? items : part ? part : 1);
    return a;
}
size_t chunk_floats(const ScanArgs& a) { return a.chunks > 1 ? (size_t)a.chunks * a.batch * (a.states + 2) * a.channels : 0; }
// the parts of a workspace, each in whole vectors
size_t whole(size_t floats) { return (floats + 3) / 4 * 4; }

void place_chunks(ScanArgs& a, float* space) {
    a.ends = space;
    a.spans = space + (size_t)a.chunks * a.batch * a.states * a.channels;
}

template <class T, int L, int M, int W>
hipError_t scan(const ScanArgs& a, hipStream_t stream) {
    if (a.steps == 1 && !a.held) {
        k_scan_step<T, L * M / 4><<<a.batch * a.groups * ((a.channels / a.groups + 255) / 256), 256, 0, stream>>>(a);
        return hipGetLastError();
    }
    const uint32_t each = a.batch * a.tiles * a.groups;
    if (a.chunks > 1) {
        k_scan<T, L, M, W, true><<<each * (a.chunks - 1), 64 * W, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
        k_scan_join<false><<<(uint32_t)(((uint64_t)a.batch * a.states * a.channels + 255) / 256), 256, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    k_scan<T, L, M, W, false><<<each * a.chunks, 64 * W, 0, stream>>>(a);
    return hipGetLastError();
}

template <class T, int L, int M, int W>
hipError_t scan_grad(const ScanArgs& a, hipStream_t stream) {
    if (a.chunks > 1) {
        k_scan_grad_first<T, L, M, W><<<a.batch * a.tiles * a.groups * (a.chunks - 1), 64 * W, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
        k_scan_join<true><<<(uint32_t)(((uint64_t)a.batch * a.states * a.channels + 255) / 256), 256, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (a.batch && a.steps) {
        k_scan_grad<T, L, M, W><<<a.parts * a.tiles * a.groups, 64 * W, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
        k_scan_grad_shared<T, L * M><<<(uint32_t)(((uint64_t)a.batch * a.steps * a.groups * 2 * L * M + 255) / 256), 256, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    const uint32_t count = a.batch && a.steps ? a.parts : 0;      // sums of nothing are zero
    JoinJobs jobs;
    jobs.add(a.sums, a.channels * a.states, 1, BPS_F32, a.grad_A);
    if (a.D) jobs.add(a.sums + (size_t)a.states * a.channels, a.channels, 1, BPS_F32, a.grad_D);
    if (a.delta_bias) jobs.add(a.sums + (size_t)(a.states + 1) * a.channels, a.channels, 1, BPS_F32, a.grad_delta_bias);
    return launch_join_parts(jobs, count, (size_t)(a.states + 2) * a.channels, stream);
}

template <class T, int L, int M>
hipError_t one_scan(const ScanArgs& a, bool grad, hipStream_t stream) {
    if (grad) return a.waves == 1 ? scan_grad<T, L, M, 1>(a, stream) : scan_grad<T, L, M, L>(a, stream);
    return a.waves == 1 ? scan<T, L, M, 1>(a, stream) : scan<T, L, M, L>(a, stream);
}

template <class T>
hipError_t scan_of(const ScanArgs& a, bool grad, hipStream_t stream) {
    switch (room(a.states)) {
        case 4: return one_scan<T, 4, 1>(a, grad, stream);
        case 8: return one_scan<T, 4, 2>(a, grad, stream);
        case 16: return one_scan<T, 4, 4>(a, grad, stream);
        // 16 steps' states of 8 states a lane do not fit its registers in the gradient: 8 x 1024 x 1024 bf16 with 32 states takes 671 us with four
        // lanes to a channel and 359 with eight; forward, where only the present ones are held, 123 and 135
        default:
            if (grad) return a.waves == 1 ? scan_grad<T, 8, 4, 1>(a, stream) : scan_grad<T, 8, 4, 8>(a, stream);
            return a.waves == 1 ? scan<T, 4, 8, 1>(a, stream) : scan<T, 4, 8, 4>(a, stream);
    }
}
hipError_t any_scan(const bps_scan& s, const ScanArgs& a, bool grad, hipStream_t stream) {
    return s.dtype == BPS_F32 ? scan_of<F32>(a, grad, stream) : s.dtype == BPS_BF16 ? scan_of<Bf16>(a, grad, stream) : scan_of<F16>(a, grad, stream);
}

}  // namespace

size_t scan_workspace(const bps_scan& s) { return chunk_floats(args_of(s, false)) * sizeof(float); }

hipError_t launch_scan(const bps_scan& s, void* workspace, hipStream_t stream) {
    ScanArgs a = args_of(s, false);
    place_chunks(a, static_cast<float*>(workspace));
    return any_scan(s, a, false, stream);
}

size_t scan_grad_workspace(const bps_scan& s) {
    const ScanArgs a = args_of(s, true);
    return (whole(chunk_floats(a)) + whole((size_t)a.parts * (a.states + 2) * a.channels) + (size_t)a.tiles * a.batch * a.steps * a.groups * 2 * room(a.states)) * sizeof(float);
}

hipError_t launch_scan_grad(const bps_scan& s, void* workspace, hipStream_t stream) {
    ScanArgs a = args_of(s, true);
    float* space = static_cast<float*>(workspace);
    place_chunks(a, space);
    a.sums = space + whole(chunk_floats(a));
    a.shared = a.sums + whole((size_t)a.parts * (a.states + 2) * a.channels);
    return any_scan(s, a, true, stream);
}

}  // namespace bps
