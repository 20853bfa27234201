// Log probabilities of given tokens, with entropy and best alternatives, and their gradient.
//
//   y = scale x over the entries that take part (allowed by the mask, x > -inf);  m = max x
//   z = sum e^(scale (x - m)),  s = sum e^(scale (x - m)) scale (x - m)
//   lse = scale m + ln z,  logp = scale (x_t - m) - ln z,  entropy = ln z - s / z
//   d logp / dx_j = scale (d_jt - p_j),  d entropy / dx_j = -scale p_j (ln p_j + entropy)
//
// All sums are held in float32 and exponents taken to the base 2.  A lane keeps m, z and s of what it has seen,
// and rescales z and s when m grows, so that one pass over the logits is enough; lanes, wavefronts and pieces
// of a row are joined by the same rule.  m and ln z are kept apart for the gradient: their sum, lse, loses ln z
// where logits are large (rows of a type's lowest value).
//
// What bounds it, on one MI355X (median kernel times): long rows the memory, 8192 x 131072 bf16 in 361 us (5.9
// TB/s, with what the Infinity Cache still holds) and their gradient in 730 to 750 us (5.8 TB/s of 4.3 GB); the
// pass itself is near the vector units' limit too, with nine instructions and one exponential (four times the
// issue slots) an entry.  Short rows the launch: 32768 x 6 float32 3.5 us, the gradient 3.1.  Alternatives cost
// what ordering the candidates costs: 192 x 50257 f16 with 5 of them 17 us, 10 without; 1 x 131072 with 20 in
// pieces 7 us and their join 5.
#include <type_traits>

#include "policy_device.h"
#include "policy_kernels.h"

namespace bps {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;
// Stands for differences below it where they are multiplied by a probability, which is zero there (2^-149 is
// the least float), so that the product is too: near enough to zero that neither the number of entries nor the
// gradients that come in make it infinite first.
constexpr float kFar = -256.0f;
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

// Adds N entries, and returns the largest of them (or the lowest finite value).
template <int N>
__device__ __forceinline__ float add(Part& p, const float (&x)[N], float c) {
    float top = kLowest;
#pragma unroll
    for (int k = 0; k < N; ++k) top = fmaxf(top, x[k]);
    const float m = fmaxf(p.m, top);
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
    return top;
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

// N bytes of a mask that lie anywhere, in two words.
template <int N>
__device__ __forceinline__ auto mask_bytes(const uint8_t* p) {
    typedef uint32_t Bytes __attribute__((ext_vector_type(2)));
    const Pack<uint8_t, N> q = *reinterpret_cast<const Pack<uint8_t, N>*>(p);
    if constexpr (N == 8)
        return __builtin_bit_cast(Bytes, q);
    else
        return Bytes{__builtin_bit_cast(uint32_t, q), 0u};
}

// U times N entries of a row, the u-th from first + u * apart + lane * N on; `all`: the same for all lanes of
// the wavefront, says that none of them lies behind the row's end.  Loads under a condition of their own would
// each be waited for before the next.
template <class T, int U, int N, bool MASK>
__device__ __forceinline__ void row_blocks(const typename T::raw* row, const uint8_t* mask, uint32_t first, uint32_t apart, uint32_t lane, uint32_t end, bool all, float (&x)[U * N]) {
    if (all) {
        Pack<typename T::raw, N> q[U];
        Pack<uint8_t, N> may[MASK ? U : 1];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = *reinterpret_cast<const Pack<typename T::raw, N>*>(row + first + u * apart + lane * N);
        if (MASK) {
#pragma unroll
            for (int u = 0; u < U; ++u) may[u] = *reinterpret_cast<const Pack<uint8_t, N>*>(mask + first + u * apart + lane * N);
        }
#pragma unroll
        for (int e = 0; e < U * N; ++e) {
            const float y = to_float(q[e / N].v[e % N]);
            x[e] = !MASK || may[e / N].v[e % N] ? y : -kInf;
        }
        return;
    }
    // -inf, and allowed, where nothing is loaded; the one lane that the row ends in takes its entries one by one
    constexpr uint32_t kNone = sizeof(typename T::raw) == 4 ? 0xFF800000u : std::is_same_v<T, Bf16> ? 0xFF80FF80u : 0xFC00FC00u;
    typedef uint32_t Bytes __attribute__((ext_vector_type(2)));
    Words q[U];
    Bytes may[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * apart + lane * N;
        q[u] = Words{kNone, kNone, kNone, kNone};
        may[u] = Bytes{0x01010101u, 0x01010101u};
        if (at + N <= end) {
            q[u] = load_words<T>(row + at);
            if (MASK) may[u] = mask_bytes<N>(mask + at);
        }
    }
#pragma unroll
    for (int e = 0; e < U * N; ++e) {
        const float y = word_float<T>(q[e / N], e % N);
        x[e] = !MASK || (may[e / N][e % N / 4] >> (8 * (e % 4)) & 255u) ? y : -kInf;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * apart + lane * N;
        if (at < end && at + N > end) {
#pragma unroll
            for (int k = 0; k < N; ++k) x[u * N + k] = at + k < end && (!MASK || mask[at + k]) ? to_float(row[at + k]) : -kInf;
        }
    }
}

// What decides the order of alternatives: the entry as a number that grows with it (NaN above all, -0 as 0), then
// the lower index.  No entry that takes part has the number 0.
__device__ __forceinline__ uint64_t order_of(float x, uint32_t at) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t up = x != x ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return (uint64_t)up << 32 | (uint32_t)~at;
}

template <int X>
__device__ __forceinline__ Part from_lane_xor(const Part& p) {
    return {bps::from_lane_xor<X>(p.m), bps::from_lane_xor<X>(p.z), bps::from_lane_xor<X>(p.s)};
}
template <int G>
__device__ __forceinline__ Part group_part(Part p, float c) {
    if constexpr (G > 1) p = joined(p, from_lane_xor<1>(p), c);
    if constexpr (G > 2) p = joined(p, from_lane_xor<2>(p), c);
    if constexpr (G > 4) p = joined(p, from_lane_xor<4>(p), c);
    if constexpr (G > 8) p = joined(p, from_lane_xor<8>(p), c);
    if constexpr (G > 16) p = joined(p, from_lane_xor<16>(p), c);
    if constexpr (G > 32) p = joined(p, from_lane_xor<32>(p), c);
    return p;
}

// What a row's sums say, written by one lane.
template <class T>
__device__ __forceinline__ void write_row(const ScoreArgs& a, uint64_t r, const Part& p, float ln_z, const typename T::raw* row, const uint8_t* mask) {
    const bool empty = p.z == 0.0f;
    a.largest[r] = p.m;
    a.ln_z[r] = ln_z;
    a.lse[r] = empty ? -kInf : fmaf(a.scale, p.m, ln_z);
    a.entropy[r] = empty ? 0.0f : ln_z - kLn2 * (p.s / p.z);
    const int64_t t = token_at(a.tokens, a.tokens64, r);
    float lp = 0.0f;
    if (t < -1 || t >= (int64_t)a.entries) {
        lp = __builtin_nanf("");
    } else if (t >= 0) {
        const float x = !mask || mask[t] ? to_float(row[t]) : -kInf;
        lp = empty ? -kInf : fmaf(x - p.m, a.scale, -ln_z);
    }
    a.logp[r] = lp;
}
template <class T>
__device__ __forceinline__ void write_alternative(const ScoreArgs& a, uint64_t to, uint64_t order, const Part& p, float ln_z, const typename T::raw* row) {
    const uint32_t at = ~(uint32_t)order;
    a.top_ids[to] = order ? (int32_t)at : -1;
    a.top_logp[to] = order ? fmaf(to_float(row[at]) - p.m, a.scale, -ln_z) : -kInf;
}

// ---- rows of up to G * N entries: G lanes for a row, N entries of it in each; alternatives one after the other

template <class T, bool MASK, bool TOP, int G, int N>
__global__ __launch_bounds__(256) void k_score_short(ScoreArgs a) {
    const uint32_t lane = threadIdx.x & (G - 1);
    const uint64_t r = (uint64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    if (r >= a.rows) return;
    const float c = a.scale * kLog2e;
    const typename T::raw* row = static_cast<const typename T::raw*>(a.logits) + (int64_t)r * a.row_stride;
    const uint8_t* mask = MASK ? a.mask + (int64_t)r * a.mask_stride : nullptr;
    float x[N];
    row_entries<T, N, MASK>(row, mask, lane * N, a.entries, x);
    Part p = nothing();
    add(p, x, c);
    p = group_part<G>(p, c);
    const float ln_z = logf(p.z);
    if (lane == 0) write_row<T>(a, r, p, ln_z, row, mask);
    if constexpr (TOP) {
        uint64_t below = ~0ull;
        for (uint32_t k = 0; k < a.top_k; ++k) {
            uint64_t b = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint64_t o = order_of(x[e], lane * N + e);
                if (x[e] != -kInf && o < below && o > b) b = o;
            }
            b = group_reduce<G>(b, [](uint64_t u, uint64_t v) { return u > v ? u : v; });
            if (lane == 0) write_alternative<T>(a, r * a.top_k + k, b, p, ln_z, row);
            below = b;
        }
    }
}

// ---- longer rows: a wavefront, or a work-group, streams a row or a piece of one

// The best 64 of what a wavefront has seen, one in each lane in descending order; 0 = none. A bitonic network:
// halves that are sorted are joined by a comparison with the mirrored lane, then with lanes at falling
// distances.
template <int X>
__device__ __forceinline__ uint64_t exchanged(uint64_t v, bool keep_larger) {
    const uint64_t o = bps::from_lane_xor<X>(v);
    return (o > v) == keep_larger ? o : v;
}
template <int X>
__device__ __forceinline__ uint64_t settled(uint64_t v, uint32_t lane) {      // comparisons at the distances X, X / 2 .. 1
    v = exchanged<X>(v, (lane & X) == 0);
    if constexpr (X > 1) v = settled<X / 2>(v, lane);
    return v;
}
__device__ __forceinline__ uint64_t sorted(uint64_t v, uint32_t lane) {
    v = exchanged<1>(v, (lane & 1) == 0);
    v = settled<1>(exchanged<3>(v, (lane & 2) == 0), lane);
    v = settled<2>(exchanged<7>(v, (lane & 4) == 0), lane);
    v = settled<4>(exchanged<15>(v, (lane & 8) == 0), lane);
    v = settled<8>(exchanged<31>(v, (lane & 16) == 0), lane);
    return settled<16>(exchanged<63>(v, (lane & 32) == 0), lane);
}
// the best 64 of two lists that are sorted
__device__ __forceinline__ uint64_t merged(uint64_t a, uint64_t b, uint32_t lane) {
    const uint64_t o = bps::from_lane_xor<63>(b);
    return settled<32>(o > a ? o : a, lane);
}
// The best of WAVES lists, in the first wavefront: half of the lists are joined to the other half, until one is left.
template <int WAVES>
__device__ __forceinline__ uint64_t merged_waves(uint64_t list, uint64_t* held, uint32_t stride, uint32_t wave, uint32_t lane) {
    held[wave * stride + lane] = list;
#pragma unroll
    for (uint32_t half = WAVES / 2; half; half /= 2) {
        __syncthreads();
        if (wave < half) {
            list = merged(list, held[(wave + half) * stride + lane], lane);
            held[wave * stride + lane] = list;
        }
    }
    return list;
}

// A number that k of the wavefront's reach, and no more than the k-th largest's upper 16 bits are above it.
__device__ __forceinline__ uint32_t reached_by(uint32_t v, uint32_t k) {
    uint32_t bar = 0;
#pragma unroll
    for (int b = 31; b >= 16; --b) {
        const uint32_t trial = bar | 1u << b;
        bar = (uint32_t)__popcll(__ballot(v >= trial)) >= k ? trial : bar;
    }
    return bar;
}

// The upper half of an order (see order_of), which the float alone decides, and the float that it stands for.
__device__ __forceinline__ uint32_t rank_of(float x) { return (uint32_t)(order_of(x, 0u) >> 32); }
__device__ __forceinline__ float value_of(uint32_t rank) { return rank < 0x00800000u ? kLowest : __uint_as_float((rank & 0x80000000u) ? rank & 0x7FFFFFFFu : ~rank); }

constexpr uint32_t kWaiting = 128;     // candidates that wait for a sort, per wavefront
constexpr uint32_t kCounted = 40;      // up to so many are put in order by counting

struct Best {
    uint64_t list;            // sorted, one per lane
    uint64_t* waiting;        // LDS, kWaiting of this wavefront
    uint32_t count;           // of them, below 64 between calls
    bool any;                 // in the list
    float least;              // finite, or NaN, or +inf: entries below it, or as large and behind least_at, are no candidates (nor is -inf ever)
    uint32_t least_at;

    __device__ __forceinline__ void raise(float to, uint32_t at) {
        if (to > least || to != to || (to == least && at < least_at)) {
            least = to;
            least_at = at;
        }
    }
    __device__ __forceinline__ void take_in(uint32_t lane, uint32_t k, uint32_t n) {
        // the wavefront's own stores, in order before its loads
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        uint64_t v = lane < n ? waiting[lane] : 0;
        if (n <= kCounted) {
            // few: each goes where the number of larger ones says
            uint32_t larger = 0;
            for (uint32_t j = 0; j < n; ++j) {
                const uint64_t o = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), (int)j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, (int)j);
                larger += o > v ? 1u : 0u;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (lane < n) waiting[larger] = v;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            v = lane < n ? waiting[lane] : 0;
        } else {
            v = sorted(v, lane);
        }
        list = any ? merged(list, v, lane) : v;
        any = true;
        const uint64_t last = __shfl((unsigned long long)list, (int)k - 1, 64);
        if (last) raise(value_of((uint32_t)(last >> 32)), ~(uint32_t)last);
    }
    // Entries base + place(e); most wavefronts hold few candidates or none, so that each lane's are told first
    // and then taken one at a time.
    template <int N, class Place>
    __device__ __forceinline__ void offer(const float (&x)[N], uint32_t lane, uint32_t k, Place&& place) {
        uint32_t hit = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) hit += hit + (x[e] < least ? 0u : 1u);
        hit <<= 32 - N;
        while (__ballot(hit != 0)) {
            const uint32_t e = (uint32_t)__builtin_clz(hit | 1u);
            float y = x[0];
#pragma unroll
            for (int j = 1; j < N; ++j) y = e == (uint32_t)j ? x[j] : y;
            const uint32_t at = place(e);
            const bool is = hit != 0 && (y > least || (y == least && at <= least_at) || y != y);
            hit &= 0x7FFFFFFFu >> e;
            const uint64_t who = __ballot(is);
            if (!who) continue;
            if (is) waiting[count + lanes_before(who)] = order_of(y, at);
            count += (uint32_t)__popcll(who);
            if (count >= 64) {
                take_in(lane, k, 64);
                count -= 64;
                const uint64_t v = waiting[64 + lane];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                if (lane < count) waiting[lane] = v;
            }
        }
    }
    __device__ __forceinline__ void finish(uint32_t lane, uint32_t k) {
        if (count) take_in(lane, k, count);
        count = 0;
    }
};

// Entries [from, to) of a row, by WAVES wavefronts; bars: LDS, 2 * WAVES numbers.
template <class T, bool MASK, bool TOP, int WAVES>
__device__ __forceinline__ Part stream(const typename T::raw* row, const uint8_t* mask, uint32_t from, uint32_t to, uint32_t tid, float c, Best& best, uint32_t k,
                                       uint32_t* bars) {
    constexpr int N = T::kPer16, U = 4, kThreads = 64 * WAVES;
    const uint32_t lane = tid & 63u, wave = tid >> 6;
    Part p = nothing();
    bool first = true;
    for (uint32_t base = from; base < to; base += kThreads * N * U) {
        float x[U * N];
        row_blocks<T, U, N, MASK>(row, mask, base, kThreads * N, tid, to, base + kThreads * N * U <= to, x);
        const float top = add(p, x, c);
        if constexpr (TOP) {
            if (first) {
                // Where at least k lanes' own best reach a bar, the k-th best of all does: the k-th of any
                // wavefront's lanes, and what the k / WAVES best lanes of every wavefront reach.
                const uint32_t own = rank_of(top);
                uint32_t bar = reached_by(own, k);
                if constexpr (WAVES > 1) {
                    const uint32_t all = reached_by(own, (k + WAVES - 1) / WAVES);
                    if (lane == 0) {
                        bars[wave] = bar;
                        bars[WAVES + wave] = all;
                    }
                    __syncthreads();
                    uint32_t least = 0xFFFFFFFFu;
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) {
                        bar = bars[w] > bar ? bars[w] : bar;
                        least = bars[WAVES + w] < least ? bars[WAVES + w] : least;
                    }
                    bar = least > bar ? least : bar;
                }
                best.least = value_of(bar);
                first = false;
            }
            if (__ballot(top >= best.least || p.z != p.z))
                best.offer(x, lane, k, [&](uint32_t e) { return base + ((e / N) * kThreads + tid) * N + e % N; });
        }
    }
    return p;
}

// WAVES wavefronts for a row, four or more to a work-group.
template <class T, bool MASK, bool TOP, int WAVES>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void k_score(ScoreArgs a) {
    constexpr uint32_t kGroup = WAVES > 4 ? WAVES * 64 : 256, kWaves = kGroup / 64;
    __shared__ uint64_t waiting[TOP ? kWaves * kWaiting : 1];
    __shared__ uint32_t bars[2 * kWaves];
    __shared__ Part parts[kWaves];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t r = (uint64_t)blockIdx.x * (kWaves / WAVES) + wave / WAVES;
    const float c = a.scale * kLog2e;
    if (r >= a.rows) return;        // whole wavefronts, and where they share a row whole work-groups
    const typename T::raw* row = static_cast<const typename T::raw*>(a.logits) + (int64_t)r * a.row_stride;
    const uint8_t* mask = MASK ? a.mask + (int64_t)r * a.mask_stride : nullptr;
    Best best = {0, waiting + (TOP ? wave * kWaiting : 0), 0, false, kLowest, 0xFFFFFFFFu};
    Part p = stream<T, MASK, TOP, WAVES>(row, mask, 0, a.entries, threadIdx.x % (64 * WAVES), c, best, a.top_k, bars);
    p = group_part<64>(p, c);
    if constexpr (TOP) best.finish(lane, a.top_k);
    if constexpr (WAVES > 1) {
        if (lane == 0) parts[wave] = p;
        if (TOP)
            best.list = merged_waves<WAVES>(best.list, waiting, kWaiting, wave, lane);
        else
            __syncthreads();
        if (wave) return;
        p = group_part<WAVES>(parts[lane % WAVES], c);
    }
    const float ln_z = logf(p.z);
    if (lane == 0) write_row<T>(a, r, p, ln_z, row, mask);
    if (TOP && lane < a.top_k) write_alternative<T>(a, r * a.top_k + lane, best.list, p, ln_z, row);
}

// ---- few long rows: a work-group for each piece of a row, and one for each row that joins them

struct Pieces {
    uint32_t count, length;      // of a row; length in entries
};
struct __align__(16) PieceSums {
    Part p;
    float pad;
};

template <class T, bool MASK, bool TOP>
__global__ __launch_bounds__(256) void k_score_piece(ScoreArgs a, Pieces pieces, PieceSums* sums, uint64_t* lists) {
    __shared__ uint64_t waiting[TOP ? 4 * kWaiting : 1];
    __shared__ uint32_t bars[8];
    __shared__ Part parts[4];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t r = blockIdx.x / pieces.count;
    const uint32_t piece = blockIdx.x % pieces.count, from = piece * pieces.length;
    const uint32_t to = a.entries - from < pieces.length ? a.entries : from + pieces.length;
    const float c = a.scale * kLog2e;
    const typename T::raw* row = static_cast<const typename T::raw*>(a.logits) + (int64_t)r * a.row_stride;
    const uint8_t* mask = MASK ? a.mask + (int64_t)r * a.mask_stride : nullptr;
    Best best = {0, waiting + (TOP ? wave * kWaiting : 0), 0, false, kLowest, 0xFFFFFFFFu};
    Part p = stream<T, MASK, TOP, 4>(row, mask, from, to, threadIdx.x, c, best, a.top_k, bars);
    p = group_part<64>(p, c);
    if constexpr (TOP) best.finish(lane, a.top_k);
    if (lane == 0) parts[wave] = p;
    if (TOP)
        best.list = merged_waves<4>(best.list, waiting, kWaiting, wave, lane);
    else
        __syncthreads();
    if (wave) return;
    p = group_part<4>(parts[lane % 4], c);
    if (lane == 0) sums[blockIdx.x] = {p, 0.0f};
    if (TOP && lane < a.top_k) lists[(uint64_t)blockIdx.x * a.top_k + lane] = best.list;
}

constexpr uint32_t kMaxPieces = 64;

template <class T, bool TOP>
__global__ __launch_bounds__(TOP ? 1024 : 64) void k_score_join(ScoreArgs a, Pieces pieces, const PieceSums* sums, const uint64_t* lists) {
    constexpr uint32_t kWaves = TOP ? 16 : 1;
    __shared__ uint64_t held[kWaves * 64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t r = blockIdx.x;
    const float c = a.scale * kLog2e;
    const typename T::raw* row = static_cast<const typename T::raw*>(a.logits) + (int64_t)r * a.row_stride;
    const uint8_t* mask = a.mask ? a.mask + (int64_t)r * a.mask_stride : nullptr;
    uint64_t list = 0;
    if constexpr (TOP) {
        const uint32_t n = pieces.count * a.top_k;
        for (uint32_t at = wave * 64; at < n; at += kWaves * 64) {
            const uint64_t v = at + lane < n ? lists[r * n + at + lane] : 0;
            list = merged(list, sorted(v, lane), lane);
        }
        list = merged_waves<kWaves>(list, held, 64, wave, lane);
        if (wave) return;
    }
    Part p = lane < pieces.count ? sums[r * pieces.count + lane].p : nothing();
    p = group_part<64>(p, c);
    const float ln_z = logf(p.z);
    if (lane == 0) write_row<T>(a, r, p, ln_z, row, mask);
    if (TOP && lane < a.top_k) write_alternative<T>(a, r * a.top_k + lane, list, p, ln_z, row);
}

// ---- gradient

// With l = log2 p_j = c (x_j - m) - log2 z, the gradient is p_j (slope l + base), and token_grad more for the
// token's entry.  An entry that takes no part has p = 0 and so the gradient 0, but where the bracket may not be
// finite: odd, where that has to be asked for, and p multiplied first.
struct RowGrad {
    float m, log2_z, slope, base, token_grad;
    int64_t t;
    bool odd;
};
__device__ __forceinline__ RowGrad row_grad(const ScoreGradArgs& a, uint64_t r) {
    RowGrad g;
    g.m = a.largest[r];
    const float ln_z = a.ln_z[r];
    g.log2_z = ln_z == -kInf ? 0.0f : ln_z * kLog2e;      // nothing takes part: all entries are -inf
    g.t = token_at(a.tokens, a.tokens64, r);
    const float gh = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
    const float gl = !a.grad_logp || g.t == -1 || a.logp[r] == -kInf ? 0.0f : g.t < -1 || g.t >= (int64_t)a.entries ? __builtin_nanf("") : a.grad_logp[r];
    g.slope = -gh * a.scale * kLn2;
    g.base = -fmaf(gh, a.entropy[r], gl) * a.scale;
    g.token_grad = gl * a.scale;
    g.odd = !(fabsf(g.log2_z) < kInf && fmaf(fabsf(g.slope), -kFar, fabsf(g.base)) < kInf);
    return g;
}
template <int N>
__device__ __forceinline__ void gradient(const RowGrad& g, float c, uint32_t at, const float* x, float (&d)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float l = fmaf(x[k] - g.m, c, -g.log2_z);
        d[k] = __builtin_amdgcn_exp2f(l) * fmaf(g.slope, fmaxf(l, kFar), g.base);
    }
    if (g.odd) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float l = fmaf(x[k] - g.m, c, -g.log2_z), p = __builtin_amdgcn_exp2f(l);
            d[k] = x[k] == -kInf ? 0.0f : fmaf(p * g.slope, fmaxf(l, kFar), p * g.base);
        }
    }
    if ((uint64_t)g.t - at < (uint64_t)N) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (at + k == (uint64_t)g.t && x[k] != -kInf) d[k] += g.token_grad;
    }
}
template <class T, int N>
__device__ __forceinline__ void store_entries(typename T::raw* out, uint32_t at, uint32_t end, const float (&d)[N], bool past) {
    if (at + N <= end) {
        store<T, N>(out + at, d, past);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (at + k < end) out[at + k] = rounded<T>(d[k]);
    }
}

template <class T, int G, int N>
__global__ __launch_bounds__(256) void k_score_grad_short(ScoreGradArgs a) {
    const uint32_t lane = threadIdx.x & (G - 1);
    const uint64_t r = (uint64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    if (r >= a.rows) return;
    const RowGrad g = row_grad(a, r);
    float x[N], d[N];
    const typename T::raw* row = static_cast<const typename T::raw*>(a.logits) + (int64_t)r * a.row_stride;
    if (a.mask)
        row_entries<T, N, true>(row, a.mask + (int64_t)r * a.mask_stride, lane * N, a.entries, x);
    else
        row_entries<T, N, false>(row, nullptr, lane * N, a.entries, x);
    gradient<N>(g, a.scale * kLog2e, lane * N, x, d);
    store_entries<T, N>(static_cast<typename T::raw*>(a.out) + (int64_t)r * a.out_stride, lane * N, a.entries, d, false);
}

// Work-groups take pieces of rows, the last row first: what of the logits the forward pass read last may still
// be in a cache.
template <class T, bool MASK, int GROUP>
__global__ __launch_bounds__(GROUP) void k_score_grad(ScoreGradArgs a, uint32_t pieces) {
    constexpr int N = T::kPer16, U = 4;
    const uint64_t r = a.rows - 1 - blockIdx.x / pieces;
    const uint32_t from = blockIdx.x % pieces * (GROUP * N * U);
    const RowGrad g = row_grad(a, r);
    const typename T::raw* row = static_cast<const typename T::raw*>(a.logits) + (int64_t)r * a.row_stride;
    const uint8_t* mask = MASK ? a.mask + (int64_t)r * a.mask_stride : nullptr;
    typename T::raw* out = static_cast<typename T::raw*>(a.out) + (int64_t)r * a.out_stride;
    const float c = a.scale * kLog2e;
    float x[U * N], d[N];
    row_blocks<T, U, N, MASK>(row, mask, from, GROUP * N, threadIdx.x, a.entries, from + GROUP * N * U <= a.entries, x);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t at = from + (u * GROUP + threadIdx.x) * N;
        gradient<N>(g, c, at, x + u * N, d);
        store_entries<T, N>(out, at, a.entries, d, a.past != 0);
    }
}

// ---- which kernel

// Rows of up to kShort entries are held by few lanes, those of up to kWide by a wavefront, 8 entries to a lane,
// if not many alternatives are asked for, which cost a pass over the lanes each; longer ones are streamed.
// Measured with 32768 rows of bf16, held / streamed by a wavefront each: 32 entries 3.8 / 25.7 us, 128 5.4 /
// 25.2 (with 16 alternatives 22 / 68, with 32 37 / 90, but 300 rows of 100 with 32 17 / 11), 256 15.7 / 24.2
// (with 3 alternatives 29 / 41; float32 29 / 29, with 5 36 / 30).
constexpr uint32_t kShort = 128, kShortTop = 16, kManyRows = 8192, kShortTopOfMany = 32, kWide = 512, kWideTop = 3;
bool held(uint64_t rows, uint32_t entries, uint32_t top_k) {
    return entries <= kShort ? top_k <= (rows < kManyRows ? kShortTop : kShortTopOfMany) : entries <= kWide && top_k <= kWideTop;
}
// Rows of up to kWaveRow entries have one wavefront, where there are kWaveRows rows or more those of up to
// kLongWaveRow too.  Measured with bf16, one wavefront / four: 4096 x 2048 6.0 / 14.6 us, 4096 x 4096 8.5 /
// 14.9, 4096 x 8192 15.1 / 15.4, 512 x 4096 4.3 / 5.2 (with 20 alternatives 10.0 / 8.9), 1024 x 8192 6.3 / 6.1
// (16.1 / 12.4).
constexpr uint32_t kWaveRow = 2048, kLongWaveRow = 8192, kWaveRows = 2048;
// Longer ones have four wavefronts, or sixteen where they are longer than kLongWaveRow and there is a compute
// unit for each row.  Four / sixteen, and with 20 alternatives: 64 x 8192 3.8 / 6.2 us, 192 x 50257 9.2 / 9.0
// (20.0 / 15.9), 256 x 131072 18.0 / 15.8 (36.8 / 25.6), 384 x 50257 13.5 / 14.7 (24.5 / 29.1), 512 x 131072
// 23.7 / 27.8 (43.4 / 45.9).
constexpr uint32_t kComputeUnits = 256;
// Of up to kPieceRows rows, those longer than kLongRow are cut, so that there are up to kGroups pieces, and as
// many of a row at most as it has blocks of kPieceEntries, what a work-group loads at once of 16-bit entries
// (half of that of float32 ones).  Sixteen wavefronts / pieces: 1 x 32768 5.4 / 5.2 us (9.9 / 11.2), 1 x 131072
// 11.2 / 5.5 (21.0 / 11.2), 32 x 131072 11.6 / 6.6 (21.8 / 12.9), 64 x 50257 8.7 / 7.4 (15.3 / 13.6), 128 x
// 50257 8.9 / 8.4 (15.5 / 16.1).
constexpr uint32_t kPieceRows = 64, kLongRow = 32768, kGroups = 512, kPieceEntries = 8192;

Pieces pieces_of(uint64_t rows, uint32_t entries) {
    if (entries <= kLongRow || rows > kPieceRows || rows == 0) return {1, entries};
    uint32_t n = kGroups / (uint32_t)rows;
    const uint32_t most = (entries + kPieceEntries - 1) / kPieceEntries;
    if (n > most) n = most;
    if (n > kMaxPieces) n = kMaxPieces;
    const uint32_t length = ((entries + n - 1) / n + 63) / 64 * 64;
    return {(entries + length - 1) / length, length};
}

#define BPS_ROWS(kernel, per_group, threads, ...) \
    hipLaunchKernelGGL((kernel<T, __VA_ARGS__>), dim3((uint32_t)((a.rows + (per_group) - 1) / (per_group))), dim3(threads), 0, stream, a)

// all: rows of the whole call, which decide for each of its launches: the workspace was sized for them
template <class T, bool MASK, bool TOP>
hipError_t score(const ScoreArgs& a, uint64_t all, hipStream_t stream) {
    const Pieces pieces = pieces_of(all, a.entries);
    if (held(all, a.entries, a.top_k)) {
        if (a.entries <= 8)
            BPS_ROWS(k_score_short, 64, 256, MASK, TOP, 4, 2);
        else if (a.entries <= 32)
            BPS_ROWS(k_score_short, 32, 256, MASK, TOP, 8, 4);
        else if (a.entries <= kShort)
            BPS_ROWS(k_score_short, 16, 256, MASK, TOP, 16, 8);
        else
            BPS_ROWS(k_score_short, 4, 256, MASK, TOP, 64, 8);
    } else if (pieces.count > 1) {
        PieceSums* sums = static_cast<PieceSums*>(a.workspace);
        uint64_t* lists = reinterpret_cast<uint64_t*>(sums + a.rows * pieces.count);
        hipLaunchKernelGGL((k_score_piece<T, MASK, TOP>), dim3((uint32_t)(a.rows * pieces.count)), dim3(256), 0, stream, a, pieces, sums, lists);
        hipLaunchKernelGGL((k_score_join<T, TOP>), dim3((uint32_t)a.rows), dim3(TOP ? 1024 : 64), 0, stream, a, pieces, sums, lists);
    } else if (a.entries <= (all < kWaveRows ? kWaveRow : kLongWaveRow)) {
        BPS_ROWS(k_score, 4, 256, MASK, TOP, 1);
    } else if (a.entries <= kLongWaveRow || all > kComputeUnits) {
        BPS_ROWS(k_score, 1, 256, MASK, TOP, 4);
    } else {
        BPS_ROWS(k_score, 1, 1024, MASK, TOP, 16);
    }
    return hipGetLastError();
}
template <class T>
hipError_t score(const ScoreArgs& a, uint64_t all, hipStream_t stream) {
    if (a.mask) return a.top_k ? score<T, true, true>(a, all, stream) : score<T, true, false>(a, all, stream);
    return a.top_k ? score<T, false, true>(a, all, stream) : score<T, false, false>(a, all, stream);
}

template <class T, bool MASK>
hipError_t score_grad_masked(const ScoreGradArgs& a, hipStream_t stream) {
    if (a.entries <= 8) {
        BPS_ROWS(k_score_grad_short, 64, 256, 4, 2);
    } else if (a.entries <= 32) {
        BPS_ROWS(k_score_grad_short, 32, 256, 8, 4);
    } else if (a.entries <= kShort) {
        BPS_ROWS(k_score_grad_short, 16, 256, 16, 8);
    } else if (a.entries <= kWide) {
        BPS_ROWS(k_score_grad_short, 4, 256, 64, 8);
    } else {
        const uint32_t wave = 64 * T::kPer16 * 4, group = 4 * wave;
        const uint32_t pieces = a.entries <= wave ? 1 : (a.entries + group - 1) / group;
        if (a.entries <= wave)
            hipLaunchKernelGGL((k_score_grad<T, MASK, 64>), dim3((uint32_t)a.rows), dim3(64), 0, stream, a, pieces);
        else
            hipLaunchKernelGGL((k_score_grad<T, MASK, 256>), dim3((uint32_t)(a.rows * pieces)), dim3(256), 0, stream, a, pieces);
    }
    return hipGetLastError();
}
#undef BPS_ROWS
template <class T>
hipError_t score_grad(const ScoreGradArgs& a, hipStream_t stream) {
    return a.mask ? score_grad_masked<T, true>(a, stream) : score_grad_masked<T, false>(a, stream);
}

}  // namespace

namespace {

// Work-groups of one launch; a grid has to have less than 2^32 threads.
constexpr uint64_t kMaxGroups = 1u << 21;

template <class A>
A rows_of(const A& a, int32_t dtype, uint64_t first, uint64_t rows) {
    A s = a;
    s.rows = rows;
    s.logits = static_cast<const char*>(a.logits) + (int64_t)first * a.row_stride * (dtype == BPS_F32 ? 4 : 2);
    s.tokens = static_cast<const char*>(a.tokens) + first * (a.tokens64 ? 8 : 4);
    if (a.mask) s.mask = a.mask + (int64_t)first * a.mask_stride;
    s.logp = a.logp + first;
    s.entropy = a.entropy + first;
    s.largest = a.largest + first;
    s.ln_z = a.ln_z + first;
    return s;
}

}  // namespace

size_t score_workspace(int32_t, uint64_t rows, uint32_t entries, uint32_t top_k) {
    const Pieces pieces = pieces_of(rows, entries);
    return pieces.count > 1 ? rows * pieces.count * (sizeof(PieceSums) + top_k * sizeof(uint64_t)) : 0;
}

hipError_t launch_score(int32_t dtype, const ScoreArgs& a, hipStream_t stream) {
    // rows of a call that cuts them into pieces are few, so that it has one launch of all of them; others have
    // at most one work-group each
    static_assert(kPieceRows <= kMaxGroups, "calls that need the workspace are not split");
    for (uint64_t first = 0; first < a.rows; first += kMaxGroups) {
        ScoreArgs s = rows_of(a, dtype, first, a.rows - first < kMaxGroups ? a.rows - first : kMaxGroups);
        s.lse = a.lse + first;
        if (a.top_k) {
            s.top_ids = a.top_ids + first * a.top_k;
            s.top_logp = a.top_logp + first * a.top_k;
        }
        const hipError_t e = dtype == BPS_F32 ? score<F32>(s, a.rows, stream) : dtype == BPS_BF16 ? score<Bf16>(s, a.rows, stream) : score<F16>(s, a.rows, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_score_grad(int32_t dtype, const ScoreGradArgs& a, hipStream_t stream) {
    const uint64_t each = kMaxGroups / (1 + a.entries / 4096);
    const size_t size = dtype == BPS_F32 ? 4 : 2;
    const int32_t past = past_caches(a.out, a.out_stride, size, a.rows, a.entries);
    for (uint64_t left = a.rows; left;) {      // the last rows first, as within a launch
        const uint64_t n = left < each ? left : each;
        left -= n;
        ScoreGradArgs s = rows_of(a, dtype, left, n);
        if (a.grad_logp) s.grad_logp = a.grad_logp + left;
        if (a.grad_entropy) s.grad_entropy = a.grad_entropy + left;
        s.out = static_cast<char*>(a.out) + (int64_t)left * a.out_stride * (int64_t)size;
        s.past = past;
        const hipError_t e = dtype == BPS_F32 ? score_grad<F32>(s, stream) : dtype == BPS_BF16 ? score_grad<Bf16>(s, stream) : score_grad<F16>(s, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace bps
