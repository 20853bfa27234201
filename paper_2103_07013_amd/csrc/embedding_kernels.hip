// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Gradient: (row, token) pairs are sorted by row, stably, by digits of a few bits from the lowest up; the
// sorted order is cut into pieces of equal length, and one group of lanes walks a piece, adding up gradient
// rows in float32 in that order.  A row that lies within one piece is written at once.  One that is cut by a
// piece's bounds leaves a partial sum per piece, which are added in order by a second kernel.  The sort marks
// the rows that have a token; the others are written as zeros next to the sums, or all of a table that is
// little used is cleared next to the sort.  Tables of up to 16 rows need no sort: sums of all rows fit in LDS.
//
// What bounds it, on one MI355X (median kernel times): long batches the memory, the lookup of 262144 rows of
// 2048 bf16 290 us (5.8 TB/s of what it moves), their sums into 131072 float32 rows 415 us (5.3 TB/s), sorting
// 40 us, joining cut rows 40 us.  Middling ones the launches one after the other, each waiting for a few memory
// round trips: 16384 tokens and 50257 rows of 769, 23 us of sort, 30 us of sums (6.3 TB/s), 13 us of joining (8
// MB; each work-group lists the cut rows first).  Few rows: 32768 tokens of 5 rows of 32 4.8 us and 2.9 us.
#include <type_traits>

#include "policy_device.h"
#include "policy_kernels.h"

namespace bps {

namespace {

constexpr uint32_t kSortGroup = 512, kSortTile = 2048, kMaxDigit = 9;
// Up to this many tokens are sorted by one work-group, in one launch.  Measured at 50257 rows (two passes), one
// work-group / two launches a pass: 4096 tokens 13 / 21 us, 8192 20 / 21, without what the launches take apart.
constexpr uint32_t kSortOne = 8192, kSortOneGroup = 1024;
// Up to this many tiles each work-group adds up the counts of those before its own by itself; for more a launch
// in between does.
constexpr uint32_t kSumTiles = 32;

uint32_t bits_of(uint32_t v) {
    uint32_t b = 0;
    while (b < 32 && (v >> b)) ++b;
    return b;
}
struct SortPlan {
    uint32_t passes, digit, tiles, row;
};
// keys are 0..rows, where `rows` stands for no row
SortPlan sort_plan(uint32_t count, uint32_t rows) {
    const uint32_t bits = bits_of(rows);
    SortPlan p;
    p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
    p.digit = (bits + p.passes - 1) / p.passes;
    p.tiles = (count + kSortTile - 1) / kSortTile;
    p.row = (p.tiles + 3) / 4 * 4;
    return p;
}

__device__ __forceinline__ uint32_t key_at(const void* tokens, int tokens64, uint32_t i, uint32_t rows) {
    const int64_t t = token_at(tokens, tokens64, i);
    return t < 0 || t >= (int64_t)rows ? rows : (uint32_t)t;
}

// The lanes whose digit is the same as this lane's, among those that hold one.
__device__ __forceinline__ uint64_t peers_of(uint32_t digit, uint32_t bits, bool held) {
    uint64_t same = __ballot(held);
    for (uint32_t b = 0; b < bits; ++b) {
        const uint64_t with = __ballot((digit >> b) & 1u);
        same &= (digit >> b) & 1u ? with : ~with;
    }
    return same;
}

struct SortArgs {
    const void* tokens;       // of the first pass, where keys is null
    const uint32_t *keys, *places;
    uint32_t *out_keys, *out_places;
    uint32_t* counts;         // [digit][row of tiles], tiles in whole words of 16 bytes; then the digits' totals
    uint8_t* marks;           // [rows, in whole words], 1 where a row has a token; or null
    void* fill;               // the gradient, where the first launch writes zeros into all of it; or null
    uint64_t fill_bytes;
    int32_t tokens64;
    uint32_t count, rows, shift, bits, tiles, row, passes, last;
};

constexpr uint32_t kFill = 4096;      // of 16 bytes
// Zeros into all of a.fill, 16 bytes at a time, by the threads of `groups` work-groups, 64 KiB after 64 KiB: 1
// GiB takes 210 us so, 255 with all work-groups side by side along it, 286 so and past the caches.
__device__ __forceinline__ void fill_zeros(const SortArgs& a, uint32_t group, uint32_t groups) {
    char* p = static_cast<char*>(a.fill);
    const uint32_t head = (uint32_t)(-reinterpret_cast<uintptr_t>(p) & 15u);
    const uint64_t at = (uint64_t)group * blockDim.x + threadIdx.x, threads = (uint64_t)groups * blockDim.x;
    if (a.fill_bytes <= head) {
        for (uint64_t i = 2 * at; i < a.fill_bytes; i += 2 * threads) *reinterpret_cast<uint16_t*>(p + i) = 0;
        return;
    }
    const uint64_t words = (a.fill_bytes - head) / 16, tail = head + words * 16;
    if (2 * at < head) *reinterpret_cast<uint16_t*>(p + 2 * at) = 0;
    if (tail + 2 * at < a.fill_bytes) *reinterpret_cast<uint16_t*>(p + tail + 2 * at) = 0;
    typedef uint32_t word __attribute__((ext_vector_type(4)));
    const word zero = {0, 0, 0, 0};
    for (uint64_t from = (uint64_t)group * kFill; from < words; from += (uint64_t)groups * kFill)
        for (uint64_t i = from + threadIdx.x; i < words && i < from + kFill; i += blockDim.x) reinterpret_cast<word*>(p + head)[i] = zero;
}

__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, uint32_t i) { return a.keys ? a.keys[i] : key_at(a.tokens, a.tokens64, i, a.rows); }

// (Counted by the pass before, with an atomic addition for each pair, the second pass's counts cost 20 to 230
// us: tokens in frequent use meet.)
__global__ __launch_bounds__(kSortGroup) void k_sort_count(SortArgs a) {
    __shared__ uint32_t hist[1u << kMaxDigit];
    if (blockIdx.x >= a.tiles) {
        fill_zeros(a, blockIdx.x - a.tiles, gridDim.x - a.tiles);
        return;
    }
    const uint32_t bins = 1u << a.bits;
    for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) hist[b] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * kSortTile;
    uint32_t key[kSortTile / kSortGroup];
#pragma unroll
    for (uint32_t k = 0; k < kSortTile / kSortGroup; ++k) {
        const uint32_t i = first + k * kSortGroup + threadIdx.x;
        key[k] = i < a.count ? sort_key(a, i) : 0u;
    }
#pragma unroll
    for (uint32_t k = 0; k < kSortTile / kSortGroup; ++k)
        if (first + k * kSortGroup + threadIdx.x < a.count) atomicAdd(&hist[(key[k] >> a.shift) & (bins - 1)], 1u);
    // marks are cleared by the first pass and set by the last
    if (!a.keys && a.marks)
        for (uint32_t r = blockIdx.x * kSortGroup + threadIdx.x; r < (a.rows + 3) / 4; r += a.tiles * kSortGroup) reinterpret_cast<uint32_t*>(a.marks)[r] = 0;
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) a.counts[(size_t)b * a.row + blockIdx.x] = hist[b];
}

// Many tiles: a wavefront for each digit turns its counts into the number of equal digits in tiles before.
__global__ __launch_bounds__(256) void k_sort_sum(SortArgs a) {
    const uint32_t bins = 1u << a.bits, b = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63u;
    if (b >= bins) return;
    uint32_t* counts = a.counts + (size_t)b * a.row;
    uint32_t sum = 0;
    for (uint32_t t = 0; t < a.tiles; t += 64) {
        const uint32_t n = t + lane < a.tiles ? counts[t + lane] : 0u;
        uint32_t with = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t x = __shfl_up(with, d, 64);
            if (lane >= (uint32_t)d) with += x;
        }
        if (t + lane < a.tiles) counts[t + lane] = sum + with - n;
        sum += __shfl(with, 63, 64);
    }
    if (lane == 0) a.counts[(size_t)bins * a.row + b] = sum;
}

// Exclusive sums over `bins` numbers in LDS, by a work-group of GROUP threads; `sums`: GROUP / 64 numbers.
template <uint32_t GROUP>
__device__ __forceinline__ void exclusive_sums(uint32_t* v, uint32_t bins, uint32_t* sums) {
    constexpr uint32_t kEach = ((1u << kMaxDigit) + GROUP - 1) / GROUP;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    uint32_t n[kEach], sum = 0;
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
        n[k] = tid * kEach + k < bins ? v[tid * kEach + k] : 0u;
        sum += n[k];
    }
    uint32_t before = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t x = __shfl_up(before, d, 64);
        if (lane >= (uint32_t)d) before += x;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    before -= sum;
    for (uint32_t w = 0; w < wave; ++w) before += sums[w];
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
        if (tid * kEach + k < bins) v[tid * kEach + k] = before;
        before += n[k];
    }
    __syncthreads();
}

// Where the pairs of ROUNDS * 64 consecutive places that a wavefront holds go, 64 at a time: among the lanes of
// equal digits the rank is the number of lanes before, so that pairs of equal digits keep their order.
// at[wave][digit]: first how many the wavefront has, then, after `spread` has turned counts into places, the
// next free one.
template <uint32_t ROUNDS>
struct Ranks {
    uint64_t same[ROUNDS];

    __device__ __forceinline__ void count(const uint32_t (&digit)[ROUNDS], const bool (&held)[ROUNDS], uint32_t bits, uint32_t lane, uint32_t* at) {
#pragma unroll
        for (uint32_t j = 0; j < ROUNDS; ++j) {
            same[j] = peers_of(digit[j], bits, held[j]);
            if (held[j] && lanes_before(same[j]) == 0) atomicAdd(&at[digit[j]], (uint32_t)__popcll(same[j]));
        }
    }
    __device__ __forceinline__ void places(const uint32_t (&digit)[ROUNDS], const bool (&held)[ROUNDS], uint32_t* at, uint32_t (&to)[ROUNDS]) {
#pragma unroll
        for (uint32_t j = 0; j < ROUNDS; ++j) {
            const uint32_t before = lanes_before(same[j]);
            to[j] = held[j] ? at[digit[j]] + before : 0u;
            // the wavefront's LDS accesses are carried out in order; they only have to stay in it
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (held[j] && before == 0) at[digit[j]] = to[j] + (uint32_t)__popcll(same[j]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
};

__global__ __launch_bounds__(kSortGroup) void k_sort_place(SortArgs a) {
    constexpr uint32_t kWaves = kSortGroup / 64, kEach = kSortTile / kWaves, kRounds = kEach / 64;
    __shared__ uint32_t at[kWaves][1u << kMaxDigit];
    __shared__ uint32_t start[1u << kMaxDigit];
    __shared__ uint32_t sums[kWaves];
    const uint32_t bins = 1u << a.bits, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t first = blockIdx.x * kSortTile + wave * kEach;
    uint32_t key[kRounds], place[kRounds], digit[kRounds], to[kRounds];
    bool held[kRounds];
#pragma unroll
    for (uint32_t j = 0; j < kRounds; ++j) {
        const uint32_t i = first + 64 * j + lane;
        held[j] = i < a.count;
        key[j] = held[j] ? sort_key(a, i) : 0u;
        place[j] = held[j] && a.places ? a.places[i] : i;
        digit[j] = (key[j] >> a.shift) & (bins - 1);
    }
    // how many pairs of equal digits are in tiles before this one, and how many pairs have lower digits
    constexpr uint32_t kBins = (1u << kMaxDigit) / kSortGroup;
    uint32_t before[kBins] = {};
#pragma unroll
    for (uint32_t k = 0; k < kBins; ++k) {
        const uint32_t b = threadIdx.x + k * kSortGroup;
        if (b >= bins) continue;
        uint32_t total;
        if (a.tiles > kSumTiles) {
            before[k] = a.counts[(size_t)b * a.row + blockIdx.x];
            total = a.counts[(size_t)bins * a.row + b];
        } else {
            uint4 n[kSumTiles / 4];
#pragma unroll
            for (uint32_t t = 0; t < kSumTiles / 4; ++t)
                n[t] = 4 * t < a.tiles ? *reinterpret_cast<const uint4*>(a.counts + (size_t)b * a.row + 4 * t) : make_uint4(0, 0, 0, 0);
            total = 0;
#pragma unroll
            for (uint32_t t = 0; t < kSumTiles; ++t) {
                const uint32_t m = t >= a.tiles ? 0u : t % 4 == 0 ? n[t / 4].x : t % 4 == 1 ? n[t / 4].y : t % 4 == 2 ? n[t / 4].z : n[t / 4].w;
                if (t < blockIdx.x) before[k] += m;
                total += m;
            }
        }
        start[b] = total;
        for (uint32_t w = 0; w < kWaves; ++w) at[w][b] = 0;
    }
    __syncthreads();
    Ranks<kRounds> ranks;
    ranks.count(digit, held, a.bits, lane, at[wave]);
    exclusive_sums<kSortGroup>(start, bins, sums);
#pragma unroll
    for (uint32_t k = 0; k < kBins; ++k) {
        const uint32_t b = threadIdx.x + k * kSortGroup;
        if (b >= bins) continue;
        uint32_t next = start[b] + before[k];
        for (uint32_t w = 0; w < kWaves; ++w) {
            const uint32_t n = at[w][b];
            at[w][b] = next;
            next += n;
        }
    }
    __syncthreads();
    ranks.places(digit, held, at[wave], to);
#pragma unroll
    for (uint32_t j = 0; j < kRounds; ++j) {
        if (!held[j]) continue;
        a.out_keys[to[j]] = key[j];
        a.out_places[to[j]] = place[j];
        if (a.last && a.marks && key[j] < a.rows) a.marks[key[j]] = 1;
    }
}

// All passes by one work-group, the pairs in LDS between them; kRounds pairs to a thread.
template <uint32_t kRounds>
__global__ __launch_bounds__(kSortOneGroup) void k_sort_one(SortArgs a) {
    constexpr uint32_t kWaves = kSortOneGroup / 64, kEach = 64 * kRounds;
    __shared__ uint32_t at[kWaves][1u << kMaxDigit];
    __shared__ uint32_t start[1u << kMaxDigit];
    __shared__ uint32_t sums[kWaves];
    __shared__ uint64_t pairs[kWaves * kEach];
    if (blockIdx.x) {
        fill_zeros(a, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    const uint32_t bins = 1u << a.bits, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t first = wave * kEach;
    uint32_t key[kRounds], place[kRounds], digit[kRounds], to[kRounds];
    bool held[kRounds];
#pragma unroll
    for (uint32_t j = 0; j < kRounds; ++j) {
        const uint32_t i = first + 64 * j + lane;
        held[j] = i < a.count;
        key[j] = held[j] ? sort_key(a, i) : 0u;
        place[j] = i;
    }
    if (a.marks)
        for (uint32_t r = threadIdx.x; r < (a.rows + 3) / 4; r += kSortOneGroup) reinterpret_cast<uint32_t*>(a.marks)[r] = 0;
    for (uint32_t p = 0; p < a.passes; ++p) {
        for (uint32_t b = threadIdx.x; b < kWaves * bins; b += kSortOneGroup) at[b >> a.bits][b & (bins - 1)] = 0;
#pragma unroll
        for (uint32_t j = 0; j < kRounds; ++j) digit[j] = (key[j] >> (p * a.bits)) & (bins - 1);
        __syncthreads();
        Ranks<kRounds> ranks;
        ranks.count(digit, held, a.bits, lane, at[wave]);
        __syncthreads();
        for (uint32_t b = threadIdx.x; b < bins; b += kSortOneGroup) {
            uint32_t sum = 0;
            for (uint32_t w = 0; w < kWaves; ++w) {
                const uint32_t n = at[w][b];
                at[w][b] = sum;
                sum += n;
            }
            start[b] = sum;
        }
        __syncthreads();
        exclusive_sums<kSortOneGroup>(start, bins, sums);
        for (uint32_t b = threadIdx.x; b < kWaves * bins; b += kSortOneGroup) at[b >> a.bits][b & (bins - 1)] += start[b & (bins - 1)];
        __syncthreads();
        ranks.places(digit, held, at[wave], to);
#pragma unroll
        for (uint32_t j = 0; j < kRounds; ++j)
            if (held[j]) pairs[to[j]] = (uint64_t)key[j] << 32 | place[j];
        __syncthreads();
#pragma unroll
        for (uint32_t j = 0; j < kRounds; ++j)
            if (held[j]) {
                const uint64_t v = pairs[first + 64 * j + lane];
                key[j] = (uint32_t)(v >> 32);
                place[j] = (uint32_t)v;
            }
    }
#pragma unroll
    for (uint32_t j = 0; j < kRounds; ++j) {
        const uint32_t i = first + 64 * j + lane;
        if (!held[j]) continue;
        a.out_keys[i] = key[j];
        a.out_places[i] = place[j];
        // the clearing above lies behind the barriers of at least one pass
        if (a.marks && key[j] < a.rows) a.marks[key[j]] = 1;
    }
}

// GROUP lanes for a row, four blocks of GROUP * N columns at a time.
template <class T, int GROUP>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a) {
    constexpr int N = T::kPer16, kRows = 256 / GROUP, kAhead = 4;
    const uint64_t n = (uint64_t)blockIdx.x * kRows + threadIdx.x / GROUP;
    if (n >= a.count) return;
    const int64_t t = token_at(a.tokens, a.tokens64, n);
    const bool row = t >= 0 && t < (int64_t)a.rows;
    const float other = t == -1 ? 0.0f : __builtin_nanf("");
    const typename T::raw* from = static_cast<const typename T::raw*>(a.weight) + (row ? t : 0) * a.weight_stride;
    typename T::raw* to = static_cast<typename T::raw*>(a.out) + (int64_t)n * a.out_stride;
    for (uint32_t base = threadIdx.x % GROUP * N; base < a.width; base += kAhead * GROUP * N) {
        Words w[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            w[u] = Words{0, 0, 0, 0};
            if (base + (u * GROUP + 1) * N <= a.width) w[u] = load_words<T>(from + base + u * GROUP * N);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t at = base + u * GROUP * N;
            if (at + N <= a.width) {
                float x[N];
#pragma unroll
                for (int k = 0; k < N; ++k) x[k] = row ? word_float<T>(w[u], k) * a.scale : other;
                store<T, N>(to + at, x, a.past != 0);
            } else {
                for (uint32_t k = at; k < a.width; ++k) to[k] = rounded<T>(row ? to_float(from[k]) * a.scale : other);
            }
        }
    }
}

// ---- gradient

// Tokens of a piece: so many that there are about 2048 pieces, 4096 of narrow rows, which take few lanes each,
// so that all compute units have some; but no fewer than 8, to keep partial sums few, and from 64 on as many as
// kMaxPieces allow.  Up to 32 tokens are one piece: nothing is cut.
constexpr uint32_t kPiece = 64, kMaxPieces = 4096, kNarrow = 64;
uint32_t piece_length(uint32_t count, uint32_t width) {
    uint32_t n = count <= 32 ? 32 : 8;
    while ((count + (uint64_t)n - 1) / n > (n < kPiece && width > kNarrow ? kMaxPieces / 2 : kMaxPieces)) n *= 2;
    return n;
}

// A piece's last row goes on in the next piece: it began in this one, or before it.
enum : uint8_t { kGoesOn = 1, kThrough = 2 };

struct SumArgs {
    const uint32_t *keys, *places;
    const uint8_t* marks;     // null where no zeros are to be written
    const void* grad;
    void* out;
    uint8_t* cuts;            // [piece] what its last row is: kGoesOn, kThrough or 0
    float* partial;           // [piece][2][width]: of the row that began before the piece, of the row that goes on behind it
    int64_t grad_stride, out_stride;
    uint32_t count, rows, width, pieces, length;
    uint32_t sum_groups, blocks;      // work-groups that add up, the others write zeros; groups of columns of a row
    uint32_t zero_rows;
    float scale;
    int32_t accumulate, past;
    uint32_t join_bits;               // 2^join_bits lanes join 4 columns each
};

template <class O, int N>
__device__ __forceinline__ void write_sum(const SumArgs& a, uint32_t row, uint32_t at, const float (&sum)[N]) {
    typename O::raw* to = static_cast<typename O::raw*>(a.out) + (int64_t)row * a.out_stride + at;
    if (at + N <= a.width) {
        float y[N];
        if (a.accumulate) {
            load<O, N>(to, y);
#pragma unroll
            for (int k = 0; k < N; ++k) y[k] = fmaf(sum[k], a.scale, y[k]);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) y[k] = sum[k] * a.scale;
        }
        store<O, N>(to, y, a.past != 0);
    } else {
        for (uint32_t k = 0; at + k < a.width; ++k) to[k] = rounded<O>(a.accumulate ? fmaf(sum[k], a.scale, to_float(to[k])) : sum[k] * a.scale);
    }
}

// Zeros in rows that are not marked, GROUP lanes to a row; a work-group takes zero_rows rows that follow one another.
template <class O, int GROUP>
__device__ __forceinline__ void write_zeros(const SumArgs& a, uint32_t group) {
    constexpr int N = O::kPer16, kRows = 256 / GROUP;
    float zero[N] = {};
    const uint64_t first = (uint64_t)group * a.zero_rows, last = first + a.zero_rows < a.rows ? first + a.zero_rows : a.rows;
    for (uint64_t row = first + threadIdx.x / GROUP; row < last; row += kRows) {
        if (a.marks && a.marks[row]) continue;      // no marks: no tokens at all
        typename O::raw* to = static_cast<typename O::raw*>(a.out) + (int64_t)row * a.out_stride;
        for (uint32_t at = threadIdx.x % GROUP * N; at < a.width; at += GROUP * N) {
            if (at + N <= a.width) {
                store<O, N>(to + at, zero, a.past != 0);
            } else {
                for (uint32_t k = at; k < a.width; ++k) to[k] = rounded<O>(0.0f);
            }
        }
    }
}
// How many rows that is: 64 KiB at least.
template <class O>
uint32_t zero_rows(uint32_t width, uint32_t together) {
    const uint32_t bytes = width * (uint32_t)sizeof(typename O::raw), n = bytes < (64u << 10) ? (64u << 10) / bytes : 1u;
    return (n + together - 1) / together * together;
}
template <class O>
__global__ __launch_bounds__(256) void k_embed_zero(SumArgs a) { write_zeros<O, 64>(a, blockIdx.x); }

// 16 bytes of AHEAD rows, of which `left` columns are the row's, as they lie there: all loads are on their way
// before the first value is converted.  (A load and its conversion under one condition are waited for there:
// 519 instead of 429 us for 262144 rows of 2048 bf16.)
template <class T, int AHEAD>
__device__ __forceinline__ void rows_ahead(const typename T::raw* const (&g)[AHEAD], uint32_t left, Words (&x)[AHEAD]) {
    constexpr int N = T::kPer16, kInWord = N / 4;
    using bits = std::conditional_t<kInWord == 1, uint32_t, uint16_t>;
    if (left >= (uint32_t)N) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) x[u] = load_words<T>(g[u]);
    } else {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) x[u] = Words{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < N - 1; ++k)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                x[u][k / kInWord] |= (uint32_t)((uint32_t)k < left ? __builtin_bit_cast(bits, g[u][k]) : bits(0)) << (16 * (k % kInWord));
    }
}

// GROUP lanes for N columns each of a piece; 256 / GROUP pieces (or column blocks of one) to a work-group.
// Keys and places are fetched 64 at a time, rows kAhead at a time, so that that many are on their way at once.
template <class T, class O, int GROUP>
__global__ __launch_bounds__(256) void k_embed_sum(SumArgs a) {
    constexpr int N = T::kPer16, kSlots = 256 / GROUP, kAhead = 8;
    __shared__ uint32_t keys[kSlots][kPiece + 1], places[kSlots][kPiece];
    if (blockIdx.x >= a.sum_groups) {
        write_zeros<O, GROUP>(a, blockIdx.x - a.sum_groups);
        return;
    }
    const uint32_t lane = threadIdx.x % GROUP, slot = threadIdx.x / GROUP;
    const uint32_t work = blockIdx.x * kSlots + slot;
    const uint32_t piece = work / a.blocks, at = (work % a.blocks * GROUP + lane) * N;
    const uint32_t from = piece * a.length;
    const uint32_t end = piece >= a.pieces ? from : a.count - from < a.length ? a.count : from + a.length;
    bool began_before = piece < a.pieces && from > 0 && a.keys[from - 1] == a.keys[from];
    if (at == 0 && piece < a.pieces) {
        const uint32_t last = a.keys[end - 1];
        a.cuts[piece] = last >= a.rows || end == a.count || a.keys[end] != last ? 0 : began_before && a.keys[from] == last ? kThrough : kGoesOn;
    }
    float sum[N];
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.0f;
    for (uint32_t batch = 0; batch < a.length; batch += kPiece) {
        const uint32_t base = from + batch, n = base >= end ? 0u : end - base < kPiece ? end - base : kPiece;
        __syncthreads();
        for (uint32_t k = lane; k < n; k += GROUP) {
            keys[slot][k] = a.keys[base + k];
            places[slot][k] = a.places[base + k];
        }
        if (lane == 0 && n) keys[slot][n] = base + n < a.count ? a.keys[base + n] : 0xFFFFFFFFu;
        __syncthreads();
        if (at >= a.width) continue;
        for (uint32_t j = 0; j < n; j += kAhead) {
            Words x[kAhead];
            const typename T::raw* g[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                g[u] = static_cast<const typename T::raw*>(a.grad) + (j + u < n ? (int64_t)places[slot][j + u] * a.grad_stride : 0) + at;
            rows_ahead<T, kAhead>(g, a.width - at, x);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (j + u >= n) continue;
                const uint32_t key = keys[slot][j + u];
                if (key >= a.rows) continue;
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] += word_float<T>(x[u], k);
                const bool ends = keys[slot][j + u + 1] != key;
                if (!ends && base + j + u + 1 != end) continue;
                if (ends && !began_before) {
                    write_sum<O, N>(a, key, at, sum);
                } else {
                    float* p = a.partial + ((size_t)piece * 2 + (began_before ? 0 : 1)) * a.width + at;
                    if (at + N <= a.width) {
                        store<F32, N>(p, sum);
                    } else {
                        for (uint32_t k = 0; at + k < a.width; ++k) p[k] = sum[k];
                    }
                }
                began_before = false;
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] = 0.0f;
            }
        }
    }
}

// The rows that are cut.  Each work-group lists the pieces in which such a row begins, those of few partial
// sums and those of many.  2^join_bits lanes, 4 columns each, add up the sums of a row with few; of rows with
// many all lanes of a work-group do, each such share of them a part of the sums in order, and then those parts
// in a fixed order.
template <class O>
__global__ __launch_bounds__(1024) void k_embed_join(SumArgs a) {
    constexpr uint32_t kFew = 8, kTogether = 8, kWords = kMaxPieces / 64, kRounds = kMaxPieces / 1024;
    __shared__ uint64_t through[kWords];
    __shared__ uint16_t list[kMaxPieces];      // of few from the front, of many from the back
    __shared__ uint32_t counts[2][kWords];
    __shared__ float part[16][256];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    uint64_t begin_here[kRounds];
#pragma unroll
    for (uint32_t k = 0; k < kRounds; ++k) {
        const uint32_t piece = k * 1024 + tid;
        const uint32_t cut = piece < a.pieces ? a.cuts[piece] : 0u;
        begin_here[k] = __ballot(cut == kGoesOn);
        const uint64_t with = __ballot(cut == kThrough);
        if (lane == 0) through[piece / 64] = with;
    }
    __syncthreads();
    // partial sums of the row that begins in a piece: of this one, of those that it goes through, and of the
    // one that it ends in
    auto partial_sums = [&](uint32_t piece) {
        const uint32_t at = piece + 1;
        for (uint32_t word = at / 64; word < kWords; ++word) {
            const uint64_t ends = ~through[word] & (word == at / 64 ? ~0ull << (at % 64) : ~0ull);
            if (ends) return word * 64 + (uint32_t)__builtin_ctzll(ends) + 1 - piece;
        }
        return kMaxPieces - piece;
    };
    uint64_t many_here[kRounds];
#pragma unroll
    for (uint32_t k = 0; k < kRounds; ++k) {
        const uint32_t piece = k * 1024 + tid;
        many_here[k] = __ballot((begin_here[k] >> lane & 1u) && partial_sums(piece) > kFew);
        begin_here[k] &= ~many_here[k];
        if (lane == 0) {
            counts[0][piece / 64] = (uint32_t)__popcll(begin_here[k]);
            counts[1][piece / 64] = (uint32_t)__popcll(many_here[k]);
        }
    }
    __syncthreads();
    if (wave < 2) {
        uint32_t with = counts[wave][lane];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t x = __shfl_up(with, d, 64);
            if (lane >= (uint32_t)d) with += x;
        }
        counts[wave][lane] = with;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < kRounds; ++k) {
        const uint32_t piece = k * 1024 + tid, word = piece / 64;
        if (begin_here[k] >> lane & 1u) list[(word ? counts[0][word - 1] : 0u) + lanes_before(begin_here[k])] = (uint16_t)piece;
        if (many_here[k] >> lane & 1u) list[kMaxPieces - 1 - (word ? counts[1][word - 1] : 0u) - lanes_before(many_here[k])] = (uint16_t)piece;
    }
    __syncthreads();
    auto add = [&](uint32_t piece, uint32_t from, uint32_t to, uint32_t at, float (&sum)[4]) {
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] = 0.0f;
        for (uint32_t k = from; k < to; k += kTogether) {
            float x[kTogether][4];
#pragma unroll
            for (uint32_t u = 0; u < kTogether; ++u) {
                const float* p = a.partial + ((size_t)(piece + (k + u < to ? k + u : from)) * 2 + ((k + u < to ? k + u : from) == 0)) * a.width + at;
                if (at + 4 <= a.width) {
                    load<F32, 4>(p, x[u]);
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[u][c] = at + c < a.width ? p[c] : 0.0f;
                }
            }
#pragma unroll
            for (uint32_t u = 0; u < kTogether; ++u)
                if (k + u < to) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) sum[c] += x[u][c];
                }
        }
    };
    const uint32_t lanes = 1u << a.join_bits, shares = 1024u >> a.join_bits, share = tid >> a.join_bits, column = (tid & (lanes - 1)) * 4;
    const uint32_t blocks = (a.width + 4 * lanes - 1) / (4 * lanes);
    // a gradient of `count` rows fits in memory, so that this and the like stay below 2^32
    const uint32_t few = counts[0][kWords - 1] * blocks, many = counts[1][kWords - 1] * blocks;
    // up to half of the work-groups have rows of many sums alone, so that those of few do not wait
    const uint32_t apart = many < gridDim.x / 2 ? many : 0u;
    if (blockIdx.x >= apart) {
        for (uint32_t work = share * (gridDim.x - apart) + blockIdx.x - apart; work < few; work += shares * (gridDim.x - apart)) {
            const uint32_t piece = list[work / blocks], at = work % blocks * 4 * lanes + column;
            if (at >= a.width) continue;
            float sum[4];
            add(piece, 0, partial_sums(piece), at, sum);
            write_sum<O, 4>(a, a.keys[(piece + 1) * a.length - 1], at, sum);
        }
        if (apart) return;
    }
    for (uint32_t work = blockIdx.x; work < many; work += gridDim.x) {
        const uint32_t piece = list[kMaxPieces - 1 - work / blocks], n = partial_sums(piece), at = work % blocks * 4 * lanes + column;
        const uint32_t each = (n + shares - 1) / shares, begin = share * each < n ? share * each : n, stop = begin + each < n ? begin + each : n;
        float sum[4] = {};
        if (at < a.width) add(piece, begin, stop, at, sum);
        for (uint32_t d = lanes; d < 64; d <<= 1) {      // the shares of a wavefront, then the wavefronts
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] += __shfl_xor(sum[c], (int)d, 64);
        }
        __syncthreads();
        if (lane < lanes) store<F32, 4>(&part[wave][column], sum);
        __syncthreads();
        if (share == 0 && at < a.width) {
#pragma unroll
            for (uint32_t w = 1; w < 16; ++w) {
#pragma unroll
                for (int c = 0; c < 4; ++c) sum[c] += part[w][column + c];
            }
            write_sum<O, 4>(a, a.keys[(piece + 1) * a.length - 1], at, sum);
        }
    }
}

// ---- gradient of tables of few rows

// A policy's moves, say: every row has many tokens, and sums of all rows fit in LDS, so that nothing is sorted.
// GROUP lanes for N columns each; the groups of a work-group add up a part of its tokens each, in order, into
// sums of their own, which are joined in order, and the work-groups' sums by a second kernel.
struct FewArgs {
    const void *tokens, *grad;
    void* out;
    uint32_t* used;           // [part][wavefront], with accumulate: bit r is set where row r had a token
    float* partial;           // [part][row][width]
    int64_t grad_stride, out_stride;
    uint32_t count, rows, width, parts, length;      // parts: work-groups side by side, length: tokens of one
    float scale;
    int32_t tokens64, accumulate;
};

template <class T, int GROUP>
__global__ __launch_bounds__(256) void k_embed_few(FewArgs a) {
    constexpr int N = T::kPer16, kSlots = 256 / GROUP, kAhead = 8;
    extern __shared__ float sums[];                  // [row][slot][GROUP][N]
    const uint32_t lane = threadIdx.x % GROUP, slot = threadIdx.x / GROUP, at = (blockIdx.y * GROUP + lane) * N;
    float zero[N] = {};
    for (uint32_t r = 0; r < a.rows; ++r) store<F32, N>(sums + ((size_t)r * 256 + threadIdx.x) * N, zero);
    const uint32_t first = blockIdx.x * a.length, last = a.count - first < a.length ? a.count : first + a.length;
    uint32_t used = 0;
    const uint32_t each = (a.length + kSlots - 1) / kSlots, from = first + slot * each < last ? first + slot * each : last, to = last - from < each ? last : from + each;
    if (at < a.width) {
        for (uint32_t i = from; i < to; i += kAhead) {
            Words x[kAhead];
            int64_t t[kAhead];
            const typename T::raw* g[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t n = i + u < to ? i + u : i;
                t[u] = i + u < to ? token_at(a.tokens, a.tokens64, n) : -1;
                g[u] = static_cast<const typename T::raw*>(a.grad) + (int64_t)n * a.grad_stride + at;
            }
            rows_ahead<T, kAhead>(g, a.width - at, x);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (t[u] < 0 || t[u] >= (int64_t)a.rows) continue;
                used |= 1u << t[u];
                float* sum = sums + ((uint32_t)t[u] * 256 + threadIdx.x) * N;
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] += word_float<T>(x[u], k);
            }
        }
    }
    if (a.accumulate && blockIdx.y == 0) {      // a slot's first lane has seen all of its tokens
        used = group_reduce<64>(used, [](uint32_t u, uint32_t v) { return u | v; });
        if ((threadIdx.x & 63u) == 0) a.used[blockIdx.x * 4 + threadIdx.x / 64] = used;
    }
    __syncthreads();
    // lane (r, column) of the joined sums: N consecutive columns of one row to a thread
    for (uint32_t w = threadIdx.x; w < a.rows * GROUP; w += 256) {
        const uint32_t r = w / GROUP, l = w % GROUP, column = (blockIdx.y * GROUP + l) * N;
        if (column >= a.width) continue;
        float sum[N] = {};
#pragma unroll 4
        for (uint32_t g = 0; g < kSlots; ++g) {
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] += sums[(r * 256 + g * GROUP + l) * N + k];
        }
        float* p = a.partial + ((size_t)blockIdx.x * a.rows + r) * a.width + column;
        for (int k = 0; k < N; ++k)
            if (column + k < a.width) p[k] = sum[k];
    }
}

// 16 lanes for a column of a row, each of which adds up every 16th part's sum.  With accumulate, rows that had
// no token are not written.
template <class O>
__global__ __launch_bounds__(256) void k_embed_few_join(FewArgs a) {
    __shared__ float part[16][16];
    __shared__ uint32_t used;
    if (a.accumulate) {
        uint32_t mine = 0;
        for (uint32_t i = threadIdx.x; i < 4 * a.parts; i += 256) mine |= a.used[i];
        if (threadIdx.x == 0) used = 0;
        __syncthreads();
        if (mine) atomicOr(&used, mine);
    }
    const uint32_t cells = a.rows * a.width, cell = blockIdx.x * 16 + (threadIdx.x & 15u), share = threadIdx.x >> 4;
    float sum = 0.0f;
    if (cell < cells) {
#pragma unroll 8
        for (uint32_t p = share; p < a.parts; p += 16) sum += a.partial[(size_t)p * cells + cell];
    }
    part[share][threadIdx.x & 15u] = sum;
    __syncthreads();
    if (share || cell >= cells) return;
#pragma unroll
    for (uint32_t w = 1; w < 16; ++w) sum += part[w][threadIdx.x];
    const uint32_t r = cell / a.width;
    if (a.accumulate && !(used >> r & 1u)) return;
    typename O::raw* to = static_cast<typename O::raw*>(a.out) + (int64_t)r * a.out_stride + cell % a.width;
    *to = rounded<O>(a.accumulate ? fmaf(sum, a.scale, to_float(*to)) : sum * a.scale);
}

// Sums of so many bytes are held by a work-group, two to a compute unit.
constexpr uint32_t kFewBytes = 64 << 10, kFewParts = 256;
// How many work-groups share the tokens of a table of few rows (0: the table has more): for sums not much
// larger than the gradients, no fewer than 64 tokens for each.
uint32_t few_parts(uint32_t count, uint32_t rows, bool wide) {
    if (rows > 16 || rows * 256u * (wide ? 16u : 32u) > kFewBytes) return 0;
    const uint32_t n = (count + 63) / 64;
    return n < kFewParts ? n : kFewParts;
}

// Columns of one launch: a grid has less than 2^32 threads, and up to 65535 work-groups along its second axis.
constexpr uint32_t kFewColumns = 1u << 22;
template <class T, class O, int GROUP>
void few(const FewArgs& a, hipStream_t stream) {
    FewArgs f = a;
    for (uint32_t first = 0; first < a.width; first += kFewColumns) {
        f.width = a.width - first < kFewColumns ? a.width - first : kFewColumns;
        f.grad = static_cast<const typename T::raw*>(a.grad) + first;
        f.out = static_cast<typename O::raw*>(a.out) + first;
        const uint32_t blocks = (f.width + GROUP * T::kPer16 - 1) / (GROUP * T::kPer16);
        hipLaunchKernelGGL((k_embed_few<T, GROUP>), dim3(f.parts, blocks), dim3(256), f.rows * 256 * T::kPer16 * sizeof(float), stream, f);
        hipLaunchKernelGGL((k_embed_few_join<O>), dim3((f.rows * f.width + 15) / 16), dim3(256), 0, stream, f);
    }
}

size_t whole(size_t n) { return (n + 255) / 256 * 256; }

template <class T, class O, int GROUP>
void sum(SumArgs s, hipStream_t stream) {
    constexpr uint32_t kSlots = 256 / GROUP;
    s.blocks = (s.width + GROUP * T::kPer16 - 1) / (GROUP * T::kPer16);
    s.sum_groups = (uint32_t)(((uint64_t)s.pieces * s.blocks + kSlots - 1) / kSlots);
    s.zero_rows = zero_rows<O>(s.width, kSlots);
    const uint32_t zero = s.marks ? (s.rows + s.zero_rows - 1) / s.zero_rows : 0u;
    hipLaunchKernelGGL((k_embed_sum<T, O, GROUP>), dim3(s.sum_groups + zero), dim3(256), 0, stream, s);
}

template <class T, class O>
hipError_t embed_grad(const EmbedGradArgs& a, hipStream_t stream) {
    SumArgs s = {nullptr, nullptr, nullptr, a.grad, a.out, nullptr, nullptr, a.grad_stride, a.out_stride, a.count, a.rows, a.width, 0, 0, 0, 0, 0, a.scale, a.accumulate, past_caches(a.out, a.out_stride, sizeof(typename O::raw), a.rows, a.width), 0};
    while (s.join_bits < 6 && 4u << s.join_bits < a.width) ++s.join_bits;
    if (!a.count) {
        s.zero_rows = zero_rows<O>(a.width, 4);
        if (!a.accumulate) hipLaunchKernelGGL((k_embed_zero<O>), dim3((a.rows + s.zero_rows - 1) / s.zero_rows), dim3(256), 0, stream, s);
        return hipGetLastError();
    }
    const uint32_t lanes = (a.width + T::kPer16 - 1) / T::kPer16;
    if (uint32_t parts = few_parts(a.count, a.rows, T::kPer16 == 4)) {
        const uint32_t length = (a.count + parts - 1) / parts;
        parts = (a.count + length - 1) / length;
        uint32_t* used = static_cast<uint32_t*>(a.workspace);
        const FewArgs f = {a.tokens, a.grad, a.out, used, reinterpret_cast<float*>(used + 4 * parts), a.grad_stride, a.out_stride, a.count, a.rows, a.width, parts, length, a.scale, a.tokens64, a.accumulate};
        if (lanes <= 4)
            few<T, O, 4>(f, stream);
        else if (lanes <= 16)
            few<T, O, 16>(f, stream);
        else
            few<T, O, 64>(f, stream);
        return hipGetLastError();
    }
    const SortPlan plan = sort_plan(a.count, a.rows);
    char* w = static_cast<char*>(a.workspace);
    uint32_t* buffer[4];
    for (auto& b : buffer) {
        b = reinterpret_cast<uint32_t*>(w);
        w += whole((size_t)a.count * 4);
    }
    uint32_t* counts = reinterpret_cast<uint32_t*>(w);
    w += whole(((size_t)(plan.row + 1) << plan.digit) * 4);
    uint8_t* marks = reinterpret_cast<uint8_t*>(w);
    w += whole(a.rows);
    s.cuts = reinterpret_cast<uint8_t*>(w);
    w += kMaxPieces;
    s.partial = reinterpret_cast<float*>(w);
    // Where most rows have no token the whole table is cleared by work-groups of the sort's first launch, a
    // contiguous one in whole cache lines; else the rows that have none are, next to the sums.
    const bool cleared = !a.accumulate && a.out_stride == a.width && a.count < a.rows / 4;
    const uint64_t bytes = (uint64_t)a.rows * a.width * sizeof(typename O::raw);
    SortArgs sort = {a.tokens, nullptr, nullptr, buffer[0], buffer[1], counts, cleared || a.accumulate ? nullptr : marks, cleared ? a.out : nullptr, bytes, a.tokens64, a.count,
                     a.rows, 0, plan.digit, plan.tiles, plan.row, plan.passes, 0};
    const uint64_t fill_groups = !cleared ? 0 : (bytes + 16 * kFill - 1) / (16 * kFill);
    const uint32_t fill = (uint32_t)(fill_groups < 2048 ? fill_groups : 2048);
    if (a.count <= kSortOne) {
        const auto kernel = a.count <= kSortOneGroup ? &k_sort_one<1> : a.count <= 4 * kSortOneGroup ? &k_sort_one<4> : &k_sort_one<8>;
        hipLaunchKernelGGL(kernel, dim3(1 + fill), dim3(kSortOneGroup), 0, stream, sort);
    } else {
        for (uint32_t p = 0; p < plan.passes; ++p) {
            sort.shift = p * plan.digit;
            sort.last = p + 1 == plan.passes;
            sort.out_keys = buffer[2 * (p & 1)];
            sort.out_places = buffer[2 * (p & 1) + 1];
            hipLaunchKernelGGL(k_sort_count, dim3(plan.tiles + (p == 0 ? fill : 0u)), dim3(kSortGroup), 0, stream, sort);
            if (plan.tiles > kSumTiles) hipLaunchKernelGGL(k_sort_sum, dim3(((1u << plan.digit) + 3) / 4), dim3(256), 0, stream, sort);
            hipLaunchKernelGGL(k_sort_place, dim3(plan.tiles), dim3(kSortGroup), 0, stream, sort);
            sort.keys = sort.out_keys;
            sort.places = sort.out_places;
        }
    }
    s.keys = sort.out_keys;
    s.places = sort.out_places;
    s.marks = sort.marks;
    s.length = piece_length(a.count, a.width);
    s.pieces = (uint32_t)((a.count + (uint64_t)s.length - 1) / s.length);
    if (lanes <= 4)
        sum<T, O, 4>(s, stream);
    else if (lanes <= 16)
        sum<T, O, 16>(s, stream);
    else
        sum<T, O, 64>(s, stream);
    if (s.pieces > 1) {
        // no more rows are cut than there are rows, or places to cut at
        const uint64_t cut = (uint64_t)(s.pieces - 1 < a.rows ? s.pieces - 1 : a.rows) * ((a.width + 255) / 256);
        hipLaunchKernelGGL((k_embed_join<O>), dim3(cut < 256 ? (uint32_t)cut : 256u), dim3(1024), 0, stream, s);
    }
    return hipGetLastError();
}

template <class T>
hipError_t embed_grad_to(int32_t out_dtype, const EmbedGradArgs& a, hipStream_t stream) {
    return out_dtype == BPS_F32 ? embed_grad<T, F32>(a, stream) : out_dtype == BPS_BF16 ? embed_grad<T, Bf16>(a, stream) : embed_grad<T, F16>(a, stream);
}

// Launches of at most this many rows: a grid has to have less than 2^32 threads.
constexpr uint64_t kMaxRows = 1u << 22;

template <class T, int GROUP>
void embed_rows(const EmbedArgs& a, hipStream_t stream) {
    constexpr uint32_t kRows = 256 / GROUP;
    hipLaunchKernelGGL((k_embed<T, GROUP>), dim3((uint32_t)((a.count + kRows - 1) / kRows)), dim3(256), 0, stream, a);
}
template <class T>
hipError_t embed(const EmbedArgs& a, hipStream_t stream) {
    const uint32_t lanes = (a.width + T::kPer16 - 1) / T::kPer16;
    const int32_t past = past_caches(a.out, a.out_stride, sizeof(typename T::raw), a.count, a.width);
    for (uint64_t first = 0; first < a.count; first += kMaxRows) {
        EmbedArgs s = a;
        s.count = a.count - first < kMaxRows ? a.count - first : kMaxRows;
        s.tokens = static_cast<const char*>(a.tokens) + first * (a.tokens64 ? 8 : 4);
        s.out = static_cast<typename T::raw*>(a.out) + (int64_t)first * a.out_stride;
        s.past = past;
        if (lanes <= 4)
            embed_rows<T, 4>(s, stream);
        else if (lanes <= 16)
            embed_rows<T, 16>(s, stream);
        else
            embed_rows<T, 64>(s, stream);
    }
    return hipGetLastError();
}

}  // namespace

size_t embed_grad_workspace(uint32_t count, uint32_t rows, uint32_t width) {
    if (!count) return 0;
    const SortPlan plan = sort_plan(count, rows);
    const uint32_t length = piece_length(count, width);
    // the gradient's type is not known here: enough for either way
    const size_t few = (size_t)few_parts(count, rows, true) * ((size_t)rows * (width < kFewColumns ? width : kFewColumns) * 4 + 16);
    const size_t sorted = 4 * whole((size_t)count * 4) + whole(((size_t)(plan.row + 1) << plan.digit) * 4) + whole(rows) + kMaxPieces + (count + (size_t)length - 1) / length * 2 * width * 4;
    return few > sorted ? few : sorted;
}

hipError_t launch_embed(int32_t dtype, const EmbedArgs& a, hipStream_t stream) {
    return dtype == BPS_F32 ? embed<F32>(a, stream) : dtype == BPS_BF16 ? embed<Bf16>(a, stream) : embed<F16>(a, stream);
}
hipError_t launch_embed_grad(int32_t grad_dtype, int32_t out_dtype, const EmbedGradArgs& a, hipStream_t stream) {
    return grad_dtype == BPS_F32 ? embed_grad_to<F32>(out_dtype, a, stream)
                                 : grad_dtype == BPS_BF16 ? embed_grad_to<Bf16>(out_dtype, a, stream) : embed_grad_to<F16>(out_dtype, a, stream);
}

}  // namespace bps
