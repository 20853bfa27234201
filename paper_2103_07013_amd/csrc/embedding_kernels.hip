// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Gradient: (row, token) pairs are sorted by row, stably, by digits of a few bits from the lowest up; the sorted order
// is cut into pieces of equal length, and one group of lanes walks a piece, adding up gradient rows in float32 in
// that order.  A row that lies within one piece is written at once.  One that is cut by a piece's bounds leaves a
// partial sum per piece, which are added in order by a second kernel.  Rows without a token are found by search.
#include "policy_device.h"
#include "policy_kernels.h"

namespace bps {

namespace {

constexpr uint32_t kSortGroup = 256, kSortTile = 2048, kMaxDigit = 9;

uint32_t bits_of(uint32_t v) {
    uint32_t b = 0;
    while (b < 32 && (v >> b)) ++b;
    return b;
}
struct SortPlan {
    uint32_t passes, digit, tiles;
};
// keys are 0..rows, where `rows` stands for no row
SortPlan sort_plan(uint32_t count, uint32_t rows) {
    const uint32_t bits = bits_of(rows);
    SortPlan p;
    p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
    p.digit = (bits + p.passes - 1) / p.passes;
    p.tiles = (count + kSortTile - 1) / kSortTile;
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

// counts[digit][tile]
__global__ __launch_bounds__(kSortGroup) void k_sort_count(const void* tokens, int tokens64, const uint32_t* keys, uint32_t count, uint32_t rows,
                                                           uint32_t shift, uint32_t bits, uint32_t tiles, uint32_t* counts) {
    __shared__ uint32_t hist[1u << kMaxDigit];
    const uint32_t bins = 1u << bits;
    for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) hist[b] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * kSortTile;
    for (uint32_t k = threadIdx.x; k < kSortTile; k += kSortGroup) {
        const uint32_t i = first + k;
        if (i < count) atomicAdd(&hist[((keys ? keys[i] : key_at(tokens, tokens64, i, rows)) >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) counts[(size_t)b * tiles + blockIdx.x] = hist[b];
}

// exclusive sums in place, by one work-group
__global__ __launch_bounds__(1024) void k_sort_scan(uint32_t* counts, uint32_t n) {
    __shared__ uint32_t sums[16];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const uint32_t each = (n + 1023u) / 1024u, from = tid * each < n ? tid * each : n, to = from + each < n ? from + each : n;
    uint32_t sum = 0;
    for (uint32_t i = from; i < to; ++i) sum += counts[i];
    uint32_t before = sum;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t x = __shfl_up(before, d, 64);
        if (lane >= (uint32_t)d) before += x;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    before -= sum;
    for (uint32_t w = 0; w < wave; ++w) before += sums[w];
    for (uint32_t i = from; i < to; ++i) {
        const uint32_t x = counts[i];
        counts[i] = before;
        before += x;
    }
}

// A wavefront takes kSortTile / 4 consecutive pairs, 64 at a time; among the lanes of equal digits the rank is the number of
// lanes before, so that pairs of equal digits keep their order.
__global__ __launch_bounds__(kSortGroup) void k_sort_place(const void* tokens, int tokens64, const uint32_t* keys, const uint32_t* places, uint32_t count,
                                                           uint32_t rows, uint32_t shift, uint32_t bits, uint32_t tiles, const uint32_t* starts,
                                                           uint32_t* out_keys, uint32_t* out_places) {
    constexpr uint32_t kWaves = kSortGroup / 64, kEach = kSortTile / kWaves, kRounds = kEach / 64;
    __shared__ uint32_t at[kWaves][1u << kMaxDigit];
    const uint32_t bins = 1u << bits, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    for (uint32_t b = threadIdx.x; b < kWaves * bins; b += kSortGroup) at[b / bins][b % bins] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * kSortTile + wave * kEach;
    uint32_t key[kRounds];
    uint64_t same[kRounds];
#pragma unroll
    for (uint32_t j = 0; j < kRounds; ++j) {
        const uint32_t i = first + 64 * j + lane;
        key[j] = i < count ? (keys ? keys[i] : key_at(tokens, tokens64, i, rows)) : 0u;
    }
#pragma unroll
    for (uint32_t j = 0; j < kRounds; ++j) {
        const bool held = first + 64 * j + lane < count;
        const uint32_t digit = (key[j] >> shift) & (bins - 1);
        same[j] = peers_of(digit, bits, held);
        if (held && (same[j] & ((1ull << lane) - 1)) == 0) atomicAdd(&at[wave][digit], (uint32_t)__popcll(same[j]));
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) {
        uint32_t to = starts[(size_t)b * tiles + blockIdx.x];
        for (uint32_t w = 0; w < kWaves; ++w) {
            const uint32_t n = at[w][b];
            at[w][b] = to;
            to += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kRounds; ++j) {
        const uint32_t i = first + 64 * j + lane, digit = (key[j] >> shift) & (bins - 1);
        const bool held = i < count;
        const uint32_t before = (uint32_t)__popcll(same[j] & ((1ull << lane) - 1));
        uint32_t to = 0;
        if (held) to = at[wave][digit] + before;
        __builtin_amdgcn_wave_barrier();
        if (held && before == 0) at[wave][digit] += (uint32_t)__popcll(same[j]);
        __builtin_amdgcn_wave_barrier();
        if (held) {
            out_keys[to] = key[j];
            out_places[to] = places ? places[i] : i;
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a) {
    constexpr int N = T::kPer16;
    const uint32_t per_row = (a.width + N - 1) / N;
    const uint64_t all = a.count * per_row;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 256) {
        const uint64_t n = i / per_row;
        const uint32_t at = (uint32_t)(i - n * per_row) * N;
        const int64_t t = token_at(a.tokens, a.tokens64, n);
        const bool row = t >= 0 && t < (int64_t)a.rows;
        const float other = t == -1 ? 0.0f : __builtin_nanf("");
        const typename T::raw* from = static_cast<const typename T::raw*>(a.weight) + (row ? t : 0) * a.weight_stride + at;
        typename T::raw* to = static_cast<typename T::raw*>(a.out) + (int64_t)n * a.out_stride + at;
        if (at + N <= a.width) {
            float x[N];
            load<T, N>(from, x);
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = row ? x[k] * a.scale : other;
            store<T, N>(to, x);
        } else {
            for (uint32_t k = 0; at + k < a.width; ++k) to[k] = rounded<T>(row ? to_float(from[k]) * a.scale : other);
        }
    }
}

// ---- gradient

constexpr uint32_t kPiece = 64;

struct SumArgs {
    const uint32_t *keys, *places;
    const void* grad;
    void* out;
    float* partial;           // [piece][2][width]: of the row that began before the piece, of the row that goes on behind it
    int64_t grad_stride, out_stride;
    uint32_t count, rows, width, pieces;
    float scale;
    int32_t accumulate;
};

template <class O, int N>
__device__ __forceinline__ void write_row(const SumArgs& a, uint32_t row, uint32_t at, float (&sum)[N]) {
    typename O::raw* to = static_cast<typename O::raw*>(a.out) + (int64_t)row * a.out_stride + at;
    const uint32_t n = a.width - at < (uint32_t)N ? a.width - at : (uint32_t)N;
#pragma unroll
    for (int k = 0; k < N; ++k)
        if ((uint32_t)k < n) to[k] = rounded<O>(a.accumulate ? fmaf(sum[k], a.scale, to_float(to[k])) : sum[k] * a.scale);
}

// One thread for N columns of a piece.
template <class T, class O>
__global__ __launch_bounds__(256) void k_embed_sum(SumArgs a) {
    constexpr int N = T::kPer16;
    const uint32_t per_row = (a.width + N - 1) / N;
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint32_t piece = (uint32_t)(i / per_row);
    if (piece >= a.pieces) return;
    const uint32_t at = (uint32_t)(i - (uint64_t)piece * per_row) * N;
    const uint32_t from = piece * kPiece, to = from + kPiece < a.count ? from + kPiece : a.count;
    bool began_before = piece > 0 && a.keys[from - 1] == a.keys[from];
    float sum[N];
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.0f;
    for (uint32_t j = from; j < to; ++j) {
        const uint32_t key = a.keys[j];
        if (key >= a.rows) break;
        const typename T::raw* g = static_cast<const typename T::raw*>(a.grad) + (int64_t)a.places[j] * a.grad_stride + at;
        if (at + N <= a.width) {
            float x[N];
            load<T, N>(g, x);
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] += x[k];
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (at + k < a.width) sum[k] += to_float(g[k]);
        }
        const bool last = j + 1 == to, ends = j + 1 == a.count || a.keys[j + 1] != key;
        if (!last && !ends) continue;
        if (ends && !began_before) {
            write_row<O, N>(a, key, at, sum);
        } else {
            float* p = a.partial + ((size_t)piece * 2 + (began_before ? 0 : 1)) * a.width + at;
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (at + k < a.width) p[k] = sum[k];
        }
        began_before = false;
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] = 0.0f;
    }
}

// The rows that are cut: a thread for each column of the piece that such a row begins in.
template <class O>
__global__ __launch_bounds__(256) void k_embed_join(SumArgs a) {
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint32_t piece = (uint32_t)(i / a.width), at = (uint32_t)(i - (uint64_t)piece * a.width);
    if (piece + 1 >= a.pieces) return;
    const uint32_t from = piece * kPiece, next = from + kPiece, key = a.keys[next - 1];
    if (key >= a.rows || a.keys[next] != key) return;
    if (a.keys[from] == key && piece > 0 && a.keys[from - 1] == key) return;      // it began before this piece
    float sum[1] = {a.partial[((size_t)piece * 2 + 1) * a.width + at]};
    for (uint32_t p = piece + 1; p < a.pieces && a.keys[p * kPiece] == key; ++p) sum[0] += a.partial[(size_t)p * 2 * a.width + at];
    typename O::raw* to = static_cast<typename O::raw*>(a.out) + (int64_t)key * a.out_stride + at;
    *to = rounded<O>(a.accumulate ? fmaf(sum[0], a.scale, to_float(*to)) : sum[0] * a.scale);
}

// Zeros in rows without a token: a wavefront looks for each row among the sorted keys.
template <class O>
__global__ __launch_bounds__(256) void k_embed_zero(SumArgs a) {
    const uint32_t lane = threadIdx.x & 63u;
    for (uint32_t row = blockIdx.x * 4u + (threadIdx.x >> 6); row < a.rows; row += gridDim.x * 4u) {
        uint32_t lo = 0, hi = a.count;      // the first key >= row is in [lo, hi]
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (a.keys[mid] < row) lo = mid + 1; else hi = mid;
        }
        if (lo < a.count && a.keys[lo] == row) continue;
        typename O::raw* to = static_cast<typename O::raw*>(a.out) + (int64_t)row * a.out_stride;
        for (uint32_t at = lane; at < a.width; at += 64) to[at] = rounded<O>(0.0f);
    }
}

uint32_t groups_of(uint64_t threads) { return (uint32_t)((threads + 255) / 256); }
size_t whole(size_t n) { return (n + 255) / 256 * 256; }

template <class T, class O>
hipError_t embed_grad(const EmbedGradArgs& a, hipStream_t stream) {
    const SortPlan plan = sort_plan(a.count, a.rows);
    char* w = static_cast<char*>(a.workspace);
    uint32_t* buffer[4];
    for (auto& b : buffer) {
        b = reinterpret_cast<uint32_t*>(w);
        w += whole((size_t)a.count * 4);
    }
    uint32_t* counts = reinterpret_cast<uint32_t*>(w);
    w += whole(((size_t)plan.tiles << plan.digit) * 4);
    const uint32_t* keys = nullptr;
    const uint32_t* places = nullptr;
    for (uint32_t p = 0; p < plan.passes && a.count; ++p) {
        const uint32_t shift = p * plan.digit;
        uint32_t *to_keys = buffer[2 * (p & 1)], *to_places = buffer[2 * (p & 1) + 1];
        hipLaunchKernelGGL(k_sort_count, dim3(plan.tiles), dim3(kSortGroup), 0, stream, a.tokens, a.tokens64, keys, a.count, a.rows, shift, plan.digit, plan.tiles, counts);
        hipLaunchKernelGGL(k_sort_scan, dim3(1), dim3(1024), 0, stream, counts, plan.tiles << plan.digit);
        hipLaunchKernelGGL(k_sort_place, dim3(plan.tiles), dim3(kSortGroup), 0, stream, a.tokens, a.tokens64, keys, places, a.count, a.rows, shift, plan.digit, plan.tiles,
                           counts, to_keys, to_places);
        keys = to_keys;
        places = to_places;
    }
    SumArgs s = {keys, places, a.grad, a.out, reinterpret_cast<float*>(w), a.grad_stride, a.out_stride, a.count, a.rows, a.width,
                 (a.count + kPiece - 1) / kPiece, a.scale, a.accumulate};
    if (!a.accumulate) {
        const uint32_t g = (a.rows + 3) / 4;
        hipLaunchKernelGGL((k_embed_zero<O>), dim3(g < 8192 ? g : 8192), dim3(256), 0, stream, s);
    }
    if (a.count) {
        const uint32_t per_row = (a.width + T::kPer16 - 1) / T::kPer16;
        hipLaunchKernelGGL((k_embed_sum<T, O>), dim3(groups_of((uint64_t)s.pieces * per_row)), dim3(256), 0, stream, s);
        if (s.pieces > 1) hipLaunchKernelGGL((k_embed_join<O>), dim3(groups_of((uint64_t)(s.pieces - 1) * a.width)), dim3(256), 0, stream, s);
    }
    return hipGetLastError();
}

template <class T>
hipError_t embed_grad_to(int32_t out_dtype, const EmbedGradArgs& a, hipStream_t stream) {
    return out_dtype == BPS_F32 ? embed_grad<T, F32>(a, stream) : out_dtype == BPS_BF16 ? embed_grad<T, Bf16>(a, stream) : embed_grad<T, F16>(a, stream);
}

template <class T>
hipError_t embed(const EmbedArgs& a, hipStream_t stream) {
    const uint64_t g = (a.count * ((a.width + T::kPer16 - 1) / T::kPer16) + 255) / 256;
    hipLaunchKernelGGL((k_embed<T>), dim3((uint32_t)(g < (1u << 20) ? g : (1u << 20))), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

size_t embed_grad_workspace(uint32_t count, uint32_t rows, uint32_t width) {
    if (!count) return 0;
    const SortPlan plan = sort_plan(count, rows);
    return 4 * whole((size_t)count * 4) + whole(((size_t)plan.tiles << plan.digit) * 4) + (size_t)((count + kPiece - 1) / kPiece) * 2 * width * 4;
}

hipError_t launch_embed(int32_t dtype, const EmbedArgs& a, hipStream_t stream) {
    return dtype == BPS_F32 ? embed<F32>(a, stream) : dtype == BPS_BF16 ? embed<Bf16>(a, stream) : embed<F16>(a, stream);
}
hipError_t launch_embed_grad(int32_t grad_dtype, int32_t out_dtype, const EmbedGradArgs& a, hipStream_t stream) {
    return grad_dtype == BPS_F32 ? embed_grad_to<F32>(out_dtype, a, stream)
                                 : grad_dtype == BPS_BF16 ? embed_grad_to<Bf16>(out_dtype, a, stream) : embed_grad_to<F16>(out_dtype, a, stream);
}

}  // namespace bps
