// Host side of the policy's operators (include/bps.h): checks of arguments, and the handle of an AdamW plan.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <vector>

#include "policy_kernels.h"

using bps::fail_here;

namespace {

constexpr uint32_t kMaxTopK = 64;
constexpr uint32_t kMaxEntries = 1u << 30;

bool known(int32_t dtype) { return dtype == BPS_F32 || dtype == BPS_BF16 || dtype == BPS_F16; }
uint32_t size_of(int32_t dtype) { return dtype == BPS_F32 ? 4u : 2u; }
bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bps_status launched(const char* what, hipError_t e) {
    return e == hipSuccess ? BPS_OK : fail_here(e == hipErrorOutOfMemory ? BPS_ERR_OOM : BPS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// What both directions of the scores ask of their arguments.
bps_status check_scores(const char* what, const void* logits, int32_t dtype, uint32_t entries, const void* tokens, int32_t token_bits, float scale) {
    if (!known(dtype)) return fail_here(BPS_ERR_INVALID_ARG, "%s: unknown element type %d", what, dtype);
    if (token_bits != 32 && token_bits != 64) return fail_here(BPS_ERR_INVALID_ARG, "%s: tokens of %d bits (32 or 64)", what, token_bits);
    if (entries == 0 || entries >= kMaxEntries) return fail_here(BPS_ERR_INVALID_ARG, "%s: entries=%u must be 1 .. 2^30 - 1", what, entries);
    // exponents are taken to the base 2, and scale * log2 e has to be finite
    if (!(scale > 0.0f) || !(scale <= 0x1p127f)) return fail_here(BPS_ERR_INVALID_ARG, "%s: scale must be positive and at most 2^127", what);
    if (!logits || !tokens) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (!aligned(logits, size_of(dtype)) || !aligned(tokens, token_bits / 8)) return fail_here(BPS_ERR_INVALID_ARG, "%s: misaligned logits or tokens", what);
    return BPS_OK;
}

// Whether parameters or masters of a plan share memory, where work-groups would write to it in no order.
bool share_memory(const bps_adamw_config& cfg) {
    struct Span {
        uintptr_t begin, end;
    };
    std::vector<Span> spans;
    spans.reserve(2 * (size_t)cfg.tensors);
    for (uint32_t i = 0; i < cfg.tensors; ++i) {
        const bps_adamw_tensor& t = cfg.tensor[i];
        const uintptr_t param = reinterpret_cast<uintptr_t>(t.param), master = reinterpret_cast<uintptr_t>(t.master);
        spans.push_back({param, param + t.count * size_of(cfg.param_dtype)});
        if (t.master) spans.push_back({master, master + t.count * sizeof(float)});
    }
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.begin < b.begin; });
    for (size_t i = 1; i < spans.size(); ++i)
        if (spans[i].begin < spans[i - 1].end) return true;
    return false;
}

}  // namespace

struct bps_adamw {
    int device = 0;
    int32_t param_dtype = 0, state_bits = 0;
    uint32_t seed = 0;
    uint32_t sums = 0;                     // sums of squares that a launch leaves at most
    uint64_t total = 0;
    std::vector<uint32_t> first_chunk;     // of each tensor, and behind the last
    void* block = nullptr;                 // one allocation: tensors, chunks, sums
    bps::AdamPlan plan{};
};

extern "C" {

size_t bps_log_probs_workspace(int32_t dtype, uint64_t rows, uint32_t entries, uint32_t top_k) {
    if (!known(dtype) || rows == 0 || entries == 0 || entries >= kMaxEntries || top_k > kMaxTopK) return 0;
    return bps::score_workspace(dtype, rows, entries, top_k);
}

bps_status bps_log_probs(const void* logits, int32_t dtype, uint64_t rows, uint32_t entries, int64_t row_stride, const void* tokens, int32_t token_bits,
                         const uint8_t* mask, int64_t mask_stride, float scale, uint32_t top_k, float* logp, float* entropy, float* lse, float* norm,
                         int32_t* top_ids, float* top_logp, void* workspace, size_t workspace_bytes, void* stream) {
    const char* what = "bps_log_probs";
    if (rows == 0) return BPS_OK;
    if (bps_status st = check_scores(what, logits, dtype, entries, tokens, token_bits, scale)) return st;
    if (!logp || !entropy || !lse || !norm) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (top_k > kMaxTopK) return fail_here(BPS_ERR_INVALID_ARG, "%s: top_k=%u exceeds %u", what, top_k, kMaxTopK);
    if (top_k && (!top_ids || !top_logp)) return fail_here(BPS_ERR_INVALID_ARG, "%s: top_k without top_ids and top_logp", what);
    const size_t need = bps::score_workspace(dtype, rows, entries, top_k);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16)))
        return fail_here(BPS_ERR_INVALID_ARG, "%s: needs %zu bytes of workspace, 16-byte aligned (got %zu)", what, need, workspace ? workspace_bytes : 0);
    const bps::ScoreArgs a = {logits, tokens, mask, row_stride, mask_stride, rows, entries, scale, top_k, token_bits == 64, logp, entropy, lse, norm, norm + rows, top_ids, top_logp, workspace};
    return launched(what, bps::launch_score(dtype, a, static_cast<hipStream_t>(stream)));
}

bps_status bps_log_probs_backward(const void* logits, int32_t dtype, uint64_t rows, uint32_t entries, int64_t row_stride, const void* tokens,
                                  int32_t token_bits, const uint8_t* mask, int64_t mask_stride, float scale, const float* logp, const float* entropy,
                                  const float* norm, const float* grad_logp, const float* grad_entropy, void* out, int64_t out_stride, void* stream) {
    const char* what = "bps_log_probs_backward";
    if (rows == 0) return BPS_OK;
    if (bps_status st = check_scores(what, logits, dtype, entries, tokens, token_bits, scale)) return st;
    if (!logp || !entropy || !norm || !out) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (!aligned(out, size_of(dtype))) return fail_here(BPS_ERR_INVALID_ARG, "%s: misaligned out", what);
    if (rows > 1 && (out_stride < 0 ? -out_stride : out_stride) < (int64_t)entries) return fail_here(BPS_ERR_INVALID_ARG, "%s: rows of out overlap", what);
    const bps::ScoreGradArgs a = {logits, tokens, mask, row_stride, mask_stride, out_stride, rows, entries, scale, token_bits == 64,
                                  logp, entropy, norm, norm + rows, grad_logp, grad_entropy, out, 0};
    return launched(what, bps::launch_score_grad(dtype, a, static_cast<hipStream_t>(stream)));
}

bps_status bps_embedding(const void* tokens, int32_t token_bits, uint64_t count, const void* weight, int32_t dtype, uint32_t rows, uint32_t width,
                         int64_t weight_stride, float scale, void* out, int64_t out_stride, void* stream) {
    const char* what = "bps_embedding";
    if (!known(dtype)) return fail_here(BPS_ERR_INVALID_ARG, "%s: unknown element type %d", what, dtype);
    if (token_bits != 32 && token_bits != 64) return fail_here(BPS_ERR_INVALID_ARG, "%s: tokens of %d bits (32 or 64)", what, token_bits);
    if (rows == 0 || rows >= kMaxEntries || width == 0 || width >= kMaxEntries) return fail_here(BPS_ERR_INVALID_ARG, "%s: rows=%u and width=%u must be 1 .. 2^30 - 1", what, rows, width);
    if (count >= 1ull << 40) return fail_here(BPS_ERR_INVALID_ARG, "%s: count must be below 2^40", what);
    if (count == 0) return BPS_OK;
    if (!tokens || !weight || !out) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (!aligned(weight, size_of(dtype)) || !aligned(out, size_of(dtype)) || !aligned(tokens, token_bits / 8)) return fail_here(BPS_ERR_INVALID_ARG, "%s: misaligned argument", what);
    if (count > 1 && (out_stride < 0 ? -out_stride : out_stride) < (int64_t)width) return fail_here(BPS_ERR_INVALID_ARG, "%s: rows of out overlap", what);
    const bps::EmbedArgs a = {tokens, weight, out, weight_stride, out_stride, count, rows, width, scale, token_bits == 64, 0};
    return launched(what, bps::launch_embed(dtype, a, static_cast<hipStream_t>(stream)));
}

size_t bps_embedding_backward_workspace(uint64_t count, uint32_t rows, uint32_t width) {
    if (count >= 1ull << 31 || rows == 0 || rows >= kMaxEntries || width == 0 || width >= kMaxEntries) return 0;
    return bps::embed_grad_workspace((uint32_t)count, rows, width);
}

bps_status bps_embedding_backward(const void* tokens, int32_t token_bits, uint64_t count, const void* grad_out, int32_t grad_dtype, uint32_t rows,
                                  uint32_t width, int64_t grad_stride, float scale, void* grad_weight, int32_t weight_dtype, int64_t weight_stride,
                                  int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    const char* what = "bps_embedding_backward";
    if (!known(grad_dtype) || !known(weight_dtype)) return fail_here(BPS_ERR_INVALID_ARG, "%s: unknown element type %d or %d", what, grad_dtype, weight_dtype);
    if (token_bits != 32 && token_bits != 64) return fail_here(BPS_ERR_INVALID_ARG, "%s: tokens of %d bits (32 or 64)", what, token_bits);
    if (rows == 0 || rows >= kMaxEntries || width == 0 || width >= kMaxEntries) return fail_here(BPS_ERR_INVALID_ARG, "%s: rows=%u and width=%u must be 1 .. 2^30 - 1", what, rows, width);
    if (count >= 1ull << 31) return fail_here(BPS_ERR_INVALID_ARG, "%s: count must be below 2^31", what);
    if (!grad_weight || (count && (!tokens || !grad_out))) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (!aligned(grad_weight, size_of(weight_dtype)) || !aligned(grad_out, size_of(grad_dtype)) || !aligned(tokens, token_bits / 8))
        return fail_here(BPS_ERR_INVALID_ARG, "%s: misaligned argument", what);
    if (rows > 1 && (weight_stride < 0 ? -weight_stride : weight_stride) < (int64_t)width) return fail_here(BPS_ERR_INVALID_ARG, "%s: rows of grad_weight overlap", what);
    const size_t need = bps::embed_grad_workspace((uint32_t)count, rows, width);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16)))
        return fail_here(BPS_ERR_INVALID_ARG, "%s: needs %zu bytes of workspace, 16-byte aligned (got %zu)", what, need, workspace ? workspace_bytes : 0);
    const bps::EmbedGradArgs a = {tokens, grad_out, grad_weight, grad_stride, weight_stride, (uint32_t)count, rows, width, scale, token_bits == 64, accumulate != 0, workspace};
    return launched(what, bps::launch_embed_grad(grad_dtype, weight_dtype, a, static_cast<hipStream_t>(stream)));
}

bps_status bps_adamw_create(const bps_adamw_config* cfg, bps_adamw** out) {
    const char* what = "bps_adamw_create";
    if (!cfg || !out) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    *out = nullptr;
    if (!known(cfg->param_dtype)) return fail_here(BPS_ERR_INVALID_ARG, "%s: unknown element type %d", what, cfg->param_dtype);
    if (cfg->state_bits != 32 && cfg->state_bits != 8) return fail_here(BPS_ERR_INVALID_ARG, "%s: state_bits must be 32 or 8", what);
    if (cfg->tensors == 0 || !cfg->tensor) return fail_here(BPS_ERR_INVALID_ARG, "%s: no tensors", what);
    if (!cfg->exp_avg || !cfg->exp_avg_sq || (cfg->state_bits == 8 && (!cfg->exp_avg_exponent || !cfg->exp_avg_sq_exponent)))
        return fail_here(BPS_ERR_INVALID_ARG, "%s: null state", what);
    if (!aligned(cfg->exp_avg, 16) || !aligned(cfg->exp_avg_sq, 16)) return fail_here(BPS_ERR_INVALID_ARG, "%s: states must be 16-byte aligned", what);
    if (cfg->total % bps::kStateBlock) return fail_here(BPS_ERR_INVALID_ARG, "%s: total must be a multiple of %u", what, bps::kStateBlock);
    uint64_t end = 0, chunks = 0;
    for (uint32_t i = 0; i < cfg->tensors; ++i) {
        const bps_adamw_tensor& t = cfg->tensor[i];
        if (!t.param || t.count == 0) return fail_here(BPS_ERR_INVALID_ARG, "%s: tensor %u is empty", what, i);
        if ((cfg->param_dtype == BPS_F32) != (t.master == nullptr))
            return fail_here(BPS_ERR_INVALID_ARG, "%s: tensor %u: a float32 master goes with 16-bit parameters, and with no others", what, i);
        if (!aligned(t.param, size_of(cfg->param_dtype)) || !aligned(t.master, 4)) return fail_here(BPS_ERR_INVALID_ARG, "%s: tensor %u is misaligned", what, i);
        if (t.start % bps::kStateBlock || t.start < end || t.start > cfg->total || t.count > cfg->total - t.start)
            return fail_here(BPS_ERR_INVALID_ARG, "%s: the states of tensor %u start at %llu: not a multiple of %u, not behind the last tensor's, or not inside", what, i,
                             (unsigned long long)t.start, bps::kStateBlock);
        if (!std::isfinite(t.weight_decay) || !std::isfinite(t.lr_scale)) return fail_here(BPS_ERR_INVALID_ARG, "%s: tensor %u: weight_decay or lr_scale is not finite", what, i);
        end = t.start + (t.count + bps::kStateBlock - 1) / bps::kStateBlock * bps::kStateBlock;
        chunks += (t.count + bps::kAdamChunk - 1) / bps::kAdamChunk;
    }
    if (chunks >= 1ull << 23) return fail_here(BPS_ERR_UNSUPPORTED, "%s: too many elements", what);
    // failures are told by the status; the runtime's last error, which the next launch would be taken to have
    // failed with, is cleared
    int ndev = 0, device = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || ndev <= 0 || hipGetDevice(&device) != hipSuccess) {
        (void)hipGetLastError();
        return fail_here(BPS_ERR_HIP, "%s: no HIP device available (this library has no CPU path)", what);
    }
    try {
        if (share_memory(*cfg)) return fail_here(BPS_ERR_INVALID_ARG, "%s: tensors overlap in memory", what);
        std::unique_ptr<bps_adamw> h(new bps_adamw());
        h->device = device;
        h->param_dtype = cfg->param_dtype;
        h->state_bits = cfg->state_bits;
        h->seed = cfg->seed;
        h->total = cfg->total;
        const uint32_t launches = (cfg->tensors + bps::kAdamGrads - 1) / bps::kAdamGrads;
        h->sums = launches <= bps::kAdamSums / 64 ? bps::kAdamSums / launches : 64;
        std::vector<bps::AdamTensor> tensors(cfg->tensors);
        std::vector<bps::AdamChunk> list;
        list.reserve(chunks);
        h->first_chunk.reserve(cfg->tensors + 1);
        for (uint32_t i = 0; i < cfg->tensors; ++i) {
            const bps_adamw_tensor& t = cfg->tensor[i];
            tensors[i] = {t.param, t.master, t.start, t.count, t.weight_decay, t.lr_scale};
            h->first_chunk.push_back((uint32_t)list.size());
            for (uint64_t c = 0; c * bps::kAdamChunk < t.count; ++c) list.push_back({i, (uint32_t)c});
        }
        h->first_chunk.push_back((uint32_t)list.size());
        // tensors | chunks | sums
        static_assert(sizeof(bps::AdamTensor) % alignof(double) == 0 && sizeof(bps::AdamChunk) % alignof(double) == 0, "the sums are aligned");
        const size_t at_chunks = tensors.size() * sizeof(tensors[0]), at_sums = at_chunks + list.size() * sizeof(list[0]);
        const size_t bytes = at_sums + (size_t)launches * h->sums * sizeof(double);
        hipError_t e = hipMalloc(&h->block, bytes);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            return fail_here(e == hipErrorOutOfMemory ? BPS_ERR_OOM : BPS_ERR_HIP, "%s: hipMalloc(%zu): %s", what, bytes, hipGetErrorString(e));
        }
        char* b = static_cast<char*>(h->block);
        e = hipMemcpy(b, tensors.data(), at_chunks, hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipMemcpy(b + at_chunks, list.data(), list.size() * sizeof(list[0]), hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipDeviceSynchronize();
        if (e != hipSuccess) {
            (void)hipFree(h->block);
            (void)hipGetLastError();
            return launched(what, e);
        }
        h->plan = {reinterpret_cast<bps::AdamTensor*>(b), reinterpret_cast<bps::AdamChunk*>(b + at_chunks), cfg->exp_avg, cfg->exp_avg_sq, cfg->exp_avg_exponent,
                   cfg->exp_avg_sq_exponent, reinterpret_cast<double*>(b + at_sums)};
        *out = h.release();
        return BPS_OK;
    } catch (const std::bad_alloc&) {
        return fail_here(BPS_ERR_OOM, "%s: out of host memory", what);
    }
}

void bps_adamw_destroy(bps_adamw* h) {
    if (!h) return;
    int was = 0;
    const bool known_device = hipGetDevice(&was) == hipSuccess;
    if (hipSetDevice(h->device) == hipSuccess) {
        hipDeviceSynchronize();
        hipFree(h->block);
    }
    if (known_device) (void)hipSetDevice(was);
    delete h;
}

bps_status bps_adamw_step(bps_adamw* h, const void* const* grads, int32_t grad_dtype, uint64_t step, double lr, double beta1, double beta2, double eps,
                          double grad_scale, double max_norm, float* grad_norm, void* stream) {
    const char* what = "bps_adamw_step";
    if (!h || !grads) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (grad_dtype != BPS_F32 && grad_dtype != h->param_dtype) return fail_here(BPS_ERR_INVALID_ARG, "%s: gradients of type %d for parameters of type %d", what, grad_dtype, h->param_dtype);
    if (step == 0) return fail_here(BPS_ERR_INVALID_ARG, "%s: steps are numbered from 1", what);
    if (!std::isfinite(lr) || !std::isfinite(grad_scale) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps) || !(max_norm >= 0.0) ||
        !std::isfinite(max_norm))
        return fail_here(BPS_ERR_INVALID_ARG, "%s: lr and grad_scale must be finite, beta1 and beta2 in [0, 1), eps and max_norm at least 0 and finite", what);
    const uint32_t tensors = (uint32_t)h->first_chunk.size() - 1;
    for (uint32_t i = 0; i < tensors; ++i)
        if (!aligned(grads[i], size_of(grad_dtype))) return fail_here(BPS_ERR_INVALID_ARG, "%s: gradient %u is misaligned", what, i);
    bps::AdamScalars s{};
    s.lr = lr;
    s.step_size = lr / (1.0 - std::pow(beta1, (double)step));
    s.beta1 = (float)beta1;
    s.one_minus_beta1 = (float)(1.0 - beta1);
    s.beta2 = (float)beta2;
    s.one_minus_beta2 = (float)(1.0 - beta2);
    s.root_c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    s.eps = (float)eps;
    s.grad_scale = (float)grad_scale;
    s.max_norm = (float)max_norm;
    s.key = bps::mixed(h->seed + (uint32_t)step * bps::kGolden);
    const bool clipped = max_norm > 0.0;
    // the sums of squares of all gradients first, then the step
    bps::AdamGrads g;
    for (int pass = clipped ? 0 : 1; pass < 2; ++pass)
        for (uint32_t first = 0; first < tensors; first += bps::kAdamGrads) {
            const uint32_t n = tensors - first < bps::kAdamGrads ? tensors - first : bps::kAdamGrads;
            for (uint32_t i = 0; i < bps::kAdamGrads; ++i) g.at[i] = i < n ? grads[first + i] : nullptr;
            const uint32_t chunk = h->first_chunk[first], chunks = h->first_chunk[first + n] - chunk;
            hipError_t e;
            if (pass == 0) {
                const uint32_t groups = (chunks + 3) / 4 < h->sums ? (chunks + 3) / 4 : h->sums;      // four chunks at a time each
                e = bps::launch_adamw_norm(grad_dtype, h->plan, g, first, chunk, chunks, s.partials, groups, s, static_cast<hipStream_t>(stream));
                s.partials += groups;
            } else {
                e = bps::launch_adamw_step(h->param_dtype, grad_dtype, h->state_bits, h->plan, g, first, chunk, chunks, clipped, s, grad_norm, static_cast<hipStream_t>(stream));
            }
            if (e != hipSuccess) return launched(what, e);
        }
    return BPS_OK;
}

bps_status bps_adamw_read_states(bps_adamw* h, float* exp_avg, float* exp_avg_sq, void* stream) {
    const char* what = "bps_adamw_read_states";
    if (!h || !exp_avg || !exp_avg_sq) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (h->state_bits != 8) return fail_here(BPS_ERR_INVALID_ARG, "%s: the states are float32 already", what);
    if (!aligned(exp_avg, 4) || !aligned(exp_avg_sq, 4)) return fail_here(BPS_ERR_INVALID_ARG, "%s: misaligned argument", what);
    return launched(what, bps::launch_adamw_read(h->plan, h->total / bps::kStateBlock, exp_avg, exp_avg_sq, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
