// Operators of a policy that is trained on the renderer's frames (paper Sec. 3.3, 3.4), written for gfx950: the
// scores of the tokens (actions) it takes, the embedding of tokens, and the optimiser's step.
// Launchers only; arguments are checked in policy_api.hip, and every launcher relies on what is said there.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/bps.h"

namespace bps {

// Records `fmt` as the calling thread's last error (bps_last_error(NULL)) and returns `code`.
bps_status fail_here(bps_status code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

struct ScoreArgs {
    const void* logits;
    const void* tokens;       // int32 or int64 [rows]
    const uint8_t* mask;      // or null
    int64_t row_stride, mask_stride;
    uint64_t rows;
    uint32_t entries;         // V
    float scale;
    uint32_t top_k;
    int32_t tokens64;
    float *logp, *entropy, *lse, *largest, *ln_z;
    int32_t* top_ids;
    float* top_logp;
    void* workspace;
};
size_t score_workspace(int32_t dtype, uint64_t rows, uint32_t entries, uint32_t top_k);
hipError_t launch_score(int32_t dtype, const ScoreArgs& a, hipStream_t stream);

struct ScoreGradArgs {
    const void* logits;
    const void* tokens;
    const uint8_t* mask;
    int64_t row_stride, mask_stride, out_stride;
    uint64_t rows;
    uint32_t entries;
    float scale;
    int32_t tokens64;
    const float *logp, *entropy, *largest, *ln_z, *grad_logp, *grad_entropy;   // grad_* may be null (zero)
    void* out;
    int32_t past;             // the launcher's: results are written past the caches
};
hipError_t launch_score_grad(int32_t dtype, const ScoreGradArgs& a, hipStream_t stream);

struct EmbedArgs {
    const void* tokens;
    const void* weight;
    void* out;
    int64_t weight_stride, out_stride;
    uint64_t count;           // tokens
    uint32_t rows, width;     // V, D
    float scale;
    int32_t tokens64;
    int32_t past;             // the launcher's, as above
};
hipError_t launch_embed(int32_t dtype, const EmbedArgs& a, hipStream_t stream);

struct EmbedGradArgs {
    const void* tokens;
    const void* grad;
    void* out;
    int64_t grad_stride, out_stride;
    uint32_t count;
    uint32_t rows, width;
    float scale;
    int32_t tokens64, accumulate;
    void* workspace;
};
size_t embed_grad_workspace(uint32_t count, uint32_t rows, uint32_t width);
hipError_t launch_embed_grad(int32_t grad_dtype, int32_t out_dtype, const EmbedGradArgs& a, hipStream_t stream);

// ---- AdamW

constexpr uint32_t kStateBlock = 256;     // states of a tensor start at a multiple of this; 8-bit states share an exponent over as many
constexpr uint32_t kAdamGroup = 256;      // threads of a work-group
// Elements of a work-group: four to a thread, at once.  Chunks of 1024 / 2048 / 4096: 1.92e8 float32 parameters
// 965 / 1008 / 1012 us, 1.2e8 bf16 ones with 8-bit states 331 / 369 / 378.
constexpr uint32_t kAdamChunk = 1024;
constexpr uint32_t kAdamGrads = 448;      // gradients of one launch: their addresses travel as kernel arguments
// Sums of squares of all gradients, in which every work-group of the step finds the norm for itself: a second
// launch more, or a counter of work-groups with the cache write-backs that it needs (35 us for 5.3e6
// parameters), cost more than reading them does (see k_adamw_norm).
constexpr uint32_t kAdamSums = 1024;

struct AdamTensor {
    void* param;
    float* master;            // null for float32 parameters
    uint64_t start;           // of its states
    uint64_t count;
    float weight_decay, lr_scale;
};
struct AdamChunk {
    uint32_t tensor, index;
};
struct AdamGrads {
    const void* at[kAdamGrads];   // null: the tensor has no gradient in this step
};
struct AdamPlan {             // device memory of a handle
    const AdamTensor* tensors;
    const AdamChunk* chunks;
    void *exp_avg, *exp_avg_sq;
    uint8_t *exp_avg_exponent, *exp_avg_sq_exponent;
    double* partial;          // sums of squares
};
struct AdamScalars {
    double lr, step_size;     // lr, and lr / (1 - beta1^t)
    float beta1, one_minus_beta1, beta2, one_minus_beta2, root_c2, eps, grad_scale, max_norm;   // root_c2: 1 / sqrt(1 - beta2^t)
    uint32_t key;             // of the dither
    uint32_t partials;        // sums of squares
};
hipError_t launch_adamw_norm(int32_t grad_dtype, const AdamPlan& p, const AdamGrads& g, uint32_t first_tensor, uint32_t first_chunk, uint32_t chunks,
                             uint32_t first_sum, uint32_t groups, const AdamScalars& s, hipStream_t stream);
hipError_t launch_adamw_step(int32_t param_dtype, int32_t grad_dtype, int32_t state_bits, const AdamPlan& p, const AdamGrads& g, uint32_t first_tensor,
                             uint32_t first_chunk, uint32_t chunks, bool clipped, const AdamScalars& s, float* norm_out, hipStream_t stream);
hipError_t launch_adamw_read(const AdamPlan& p, uint64_t blocks, float* exp_avg, float* exp_avg_sq, hipStream_t stream);

// 32 bits each of which depends on all bits of h; the factors are odd numbers next to 2^32 times the fractional parts
// of sqrt 2 and sqrt 3, kGolden to that of the golden ratio.
constexpr uint32_t kGolden = 0x9E3779B9u, kRoot2 = 0x6A09E667u, kRoot3 = 0xBB67AE85u;
__host__ __device__ inline uint32_t mixed(uint32_t h) {
    h = (h ^ (h >> 16)) * kRoot2;
    h = (h ^ (h >> 15)) * kRoot3;
    return h ^ (h >> 16);
}

}  // namespace bps
