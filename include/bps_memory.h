/* bps_memory.h - C ABI of libbps_memory.so: operators of a policy's memory, beside those of libbps.so (bps.h), which it needs.
 *
 * The recurrent block between a policy's embedding and its scores (the paper's policies carry a state from step to step, Sec. 3.3).
 * All that bps.h says of the policy's operators holds for these: device memory of the current device, calls that only enqueue,
 * nothing allocated, sums in float32, the same bits every time, failures told by the status and bps_last_error(NULL).
 *
 * Sequences are tensors [batch][steps][channels]: element (b, t, c) lies at + b * batch_stride + t * step_stride + c, in elements;
 * strides are any for inputs, and for results such that no two elements meet.  In a batch of sequences
 *   starts    uint8, or NULL: where it is not 0 an episode begins at that step, which sees nothing of what came before
 *   lengths   int32 [batch], or NULL: sequence b ends before step lengths[b] (0 .. steps; others count as the nearer of the
 *             two).  What inputs hold behind the end does not matter, results and gradients are 0 there.
 * A step of a rollout or of an answer is a call with steps = 1 whose state_out is its state.  Gradients do not go
 * through states from call to call. */
#ifndef BPS_MEMORY_H
#define BPS_MEMORY_H

#include "bps.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    void *at;
    int64_t batch_stride, step_stride;
} bps_sequence;

typedef struct {
    const uint8_t *at;
    int64_t batch_stride, step_stride;   /* bytes */
} bps_starts;

/* Causal convolution, each channel by itself:
 *   u[t] = bias + sum over k < taps of weight[c][k] x[t - taps + 1 + k];   out = u / (1 + e^-u) with silu, else u
 * Inputs before the episode count as 0, those before step 0 are the state's: its last taps - 1 inputs, the oldest first.
 * 1 <= taps <= 8, channels < 2^24. */
typedef struct {
    int32_t dtype;                       /* of x, out, states and their gradients */
    int32_t weight_dtype;                /* of weight, bias and their gradients: dtype or BPS_F32 */
    uint32_t batch, steps, channels, taps;
    int32_t silu;
    bps_sequence x, out;
    const void *weight, *bias;           /* [channels][taps]; [channels] or NULL */
    bps_starts starts;
    const int32_t *lengths;
    const void *state;                   /* [batch][taps - 1][channels], batches state_stride apart; NULL = zeros */
    void *state_out;                     /* the state behind the last step, or NULL; may be `state` where steps <= 1 */
    int64_t state_stride, state_out_stride;
    /* the gradient's */
    bps_sequence grad_out, grad_x;
    void *grad_weight, *grad_bias;       /* grad_bias may be NULL */
} bps_conv;

bps_status bps_causal_conv(const bps_conv *args, void *stream);
/* The gradient of out: reads x, weight, bias, starts, lengths, state and grad_out, writes grad_x, grad_weight and grad_bias.
 *   workspace  bps_causal_conv_backward_workspace bytes, 16-byte aligned */
size_t bps_causal_conv_backward_workspace(const bps_conv *args);
bps_status bps_causal_conv_backward(const bps_conv *args, void *workspace, size_t workspace_bytes, void *stream);

/* Selective scan: a linear recurrence for each channel c and state n, whose decay and input depend on the step.
 *   d = delta + delta_bias, or ln(1 + e^that) with softplus
 *   h[n] = e^(d A[n]) h[n] + d x B[n];   y = sum over n of C[n] h[n] + D x;   out = y gate / (1 + e^-gate), or y without a gate
 * B and C are shared by the channels / groups channels of a group.  h is float32, 0 before an episode, the state's before step 0.
 * Rates A below -1e38, -infinity among them, count as that: their decays are 0 as well.
 * 1 <= states <= 32, channels < 2^24 and a multiple of groups, steps < 2^31, 0 <= step_stride < 2^26. */
typedef struct {
    int32_t dtype;                       /* of x, delta, gate, B, C, out and their gradients */
    int32_t softplus;
    uint32_t batch, steps, channels, states, groups;
    bps_sequence x, delta, gate, B, C, out;   /* B, C: [batch][steps][groups][states]; gate.at may be NULL */
    const float *A, *D, *delta_bias;     /* [states][channels]; [channels] or NULL, both */
    bps_starts starts;
    const int32_t *lengths;
    const float *state;                  /* [batch][states][channels], batches state_stride apart; NULL = zeros */
    float *state_out;                    /* the state behind the last step, or NULL; may be `state` */
    int64_t state_stride, state_out_stride;
    float *held;                         /* [batch][ceil(steps / 16)][states][channels]: states that the gradient needs, or NULL */
    /* the gradient's */
    bps_sequence grad_out, grad_x, grad_delta, grad_gate, grad_B, grad_C;
    float *grad_A, *grad_D, *grad_delta_bias;
} bps_scan;

/*   workspace  bps_selective_scan_workspace bytes, 16-byte aligned; it may be NULL where that is 0 */
size_t bps_selective_scan_workspace(const bps_scan *args);
bps_status bps_selective_scan(const bps_scan *args, void *workspace, size_t workspace_bytes, void *stream);
/* The gradient of out: reads what the scan read, with `held` as the scan left it, and grad_out; writes grad_x, grad_delta, grad_B, grad_C,
 * grad_A, and grad_gate, grad_D and grad_delta_bias where there is a gate, D and delta_bias. */
size_t bps_selective_scan_backward_workspace(const bps_scan *args);
bps_status bps_selective_scan_backward(const bps_scan *args, void *workspace, size_t workspace_bytes, void *stream);

/* A block's end and the next one's beginning, on a residual stream: with N(v; w) = v / sqrt(mean of v^2 + eps) * w over a row,
 *   m = scale * act(gate) * N(block; post_weight);   residual_out = residual + m;   out = N(residual + m; pre_weight)
 * post_weight NULL: the block's output as it is; scale, gate NULL: 1; pre_weight NULL: there is no `out`.
 * act: 0 = 1 / (1 + e^-g), 1 = g / (1 + e^-g).  Rows are *_stride elements apart.  width <= 16384. */
typedef struct {
    int32_t dtype;                       /* of block, gate, out and their gradients */
    int32_t residual_dtype;              /* of residual, residual_out and their gradients: dtype or BPS_F32 */
    int32_t weight_dtype;                /* of the three vectors and their gradients: dtype or BPS_F32 */
    int32_t activation;
    uint64_t rows;
    uint32_t width;
    float eps;                           /* >= 2^-126 */
    const void *residual, *block, *gate;
    int64_t residual_stride, block_stride, gate_stride;
    const void *post_weight, *scale, *pre_weight;   /* [width] */
    void *residual_out, *out;            /* residual_out may be `residual` where the strides are the same */
    int64_t residual_out_stride, out_stride;
    float *roots;                        /* [2][rows]: 1 / sqrt of the block's and of the sum's mean square, for the gradient; or NULL */
    /* the gradient's: what comes in for residual_out and out (NULL = zero), and what goes out */
    const void *grad_residual_out, *grad_out;
    int64_t grad_residual_out_stride, grad_out_stride;
    void *grad_residual, *grad_block, *grad_gate;
    int64_t grad_residual_stride, grad_block_stride, grad_gate_stride;
    void *grad_post_weight, *grad_scale, *grad_pre_weight;
} bps_norm;

bps_status bps_residual_norm(const bps_norm *args, void *stream);
/* The gradient: reads residual, block, gate, the vectors, roots and what comes in; writes the gradients of all of the
 * forward call's inputs that are not NULL.
 *   workspace  bps_residual_norm_backward_workspace bytes, 16-byte aligned; it may be NULL where that is 0 */
size_t bps_residual_norm_backward_workspace(const bps_norm *args);
bps_status bps_residual_norm_backward(const bps_norm *args, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BPS_MEMORY_H */
