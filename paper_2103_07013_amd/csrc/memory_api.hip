// Host side of the operators of the policy's memory (include/bps_memory.h): checks of arguments.
#include <cmath>

#include "memory_kernels.h"

using bps::fail_here;

namespace {

constexpr uint32_t kMaxChannels = 1u << 24;
constexpr int64_t kMaxStride = 1 << 26;          // of a scan's steps: places within 16 rows fit 32 bits
constexpr uint64_t kMaxThreads = 1ull << 32;     // that a launch takes

bool known(int32_t dtype) { return dtype == BPS_F32 || dtype == BPS_BF16 || dtype == BPS_F16; }
uint32_t size_of(int32_t dtype) { return dtype == BPS_F32 ? 4u : 2u; }
bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
uint64_t distance(int64_t stride) { return stride < 0 ? 0 - (uint64_t)stride : (uint64_t)stride; }

bps_status launched(const char* what, hipError_t e) {
    return e == hipSuccess ? BPS_OK : fail_here(e == hipErrorOutOfMemory ? BPS_ERR_OOM : BPS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bps_status check_workspace(const char* what, size_t need, const void* workspace, size_t bytes) {
    if (need && (!workspace || bytes < need || !aligned(workspace, 16)))
        return fail_here(BPS_ERR_INVALID_ARG, "%s: needs %zu bytes of workspace, 16-byte aligned (got %zu)", what, need, workspace ? bytes : 0);
    return BPS_OK;
}

// Of the sequences and vectors of one call
struct Checks {
    const char* what;
    uint32_t batch, steps;
    bps_status status = BPS_OK;

    void fail(const char* name, const char* text) {
        if (status == BPS_OK) status = fail_here(BPS_ERR_INVALID_ARG, "%s: %s %s", what, name, text);
    }
    void pointer(const char* name, const void* p, uint32_t size, bool needed) {
        if (!p && needed) fail(name, "is null");
        if (!aligned(p, size)) fail(name, "is misaligned");
    }
    void input(const char* name, const bps_sequence& s, int32_t dtype, bool needed = true) { pointer(name, s.at, size_of(dtype), needed && batch && steps); }
    // rows of `width` elements that do not meet: steps inside batches, or batches inside steps
    void result(const char* name, const bps_sequence& s, int32_t dtype, uint64_t width) {
        input(name, s, dtype);
        if (!batch || !steps) return;
        uint64_t near = distance(s.step_stride), far = distance(s.batch_stride), count = steps, others = batch;
        if (count == 1 || (others > 1 && far < near)) {
            uint64_t x = near;
            near = far, far = x;
            x = count;
            count = others, others = x;
        }
        // the division, by no less than the width, keeps the product in range
        if ((count > 1 && near < width) || (others > 1 && (far < width || (count > 1 && (far - width) / near < count - 1)))) fail(name, "has rows that overlap");
    }
    void state(const char* name, const void* p, uint32_t size, int64_t stride, uint64_t width, bool written) {
        pointer(name, p, size, false);
        if (p && written && batch > 1 && distance(stride) < width) fail(name, "has batches that overlap");
    }
};

bps_status check_conv(const char* what, const bps_conv& a, bool grad) {
    if (!known(a.dtype)) return fail_here(BPS_ERR_INVALID_ARG, "%s: unknown element type %d", what, a.dtype);
    if (a.weight_dtype != a.dtype && a.weight_dtype != BPS_F32) return fail_here(BPS_ERR_INVALID_ARG, "%s: weights of type %d for inputs of type %d", what, a.weight_dtype, a.dtype);
    if (a.taps == 0 || a.taps > bps::kMaxTaps) return fail_here(BPS_ERR_INVALID_ARG, "%s: taps=%u must be 1 .. %u", what, a.taps, bps::kMaxTaps);
    if (a.channels == 0 || a.channels >= kMaxChannels) return fail_here(BPS_ERR_INVALID_ARG, "%s: channels=%u must be 1 .. 2^24 - 1", what, a.channels);
    if (a.steps >= 1u << 31) return fail_here(BPS_ERR_INVALID_ARG, "%s: steps must be below 2^31", what);
    // a thread has at least 4 channels of at most 8 steps
    if ((uint64_t)a.batch * ((a.steps + 7) / 8 + 1) * ((a.channels + 3) / 4) >= kMaxThreads) return fail_here(BPS_ERR_UNSUPPORTED, "%s: too many elements for one launch", what);
    Checks c{what, a.batch, a.steps};
    const uint64_t kept = (uint64_t)(a.taps - 1) * a.channels;
    c.pointer("weight", a.weight, size_of(a.weight_dtype), true);
    c.pointer("bias", a.bias, size_of(a.weight_dtype), false);
    c.pointer("lengths", a.lengths, 4, false);
    c.input("x", a.x, a.dtype);
    c.state("state", a.state, size_of(a.dtype), a.state_stride, kept, false);
    if (grad) {
        c.input("grad_out", a.grad_out, a.dtype);
        c.result("grad_x", a.grad_x, a.dtype, a.channels);
        c.pointer("grad_weight", a.grad_weight, size_of(a.weight_dtype), true);
        c.pointer("grad_bias", a.grad_bias, size_of(a.weight_dtype), false);
    } else {
        c.result("out", a.out, a.dtype, a.channels);
        c.state("state_out", a.state_out, size_of(a.dtype), a.state_out_stride, kept, true);
        if (a.state_out && a.state_out == a.state && (a.steps > 1 || a.state_stride != a.state_out_stride)) c.fail("state_out", "may be the state in calls of one step only, with its stride");
    }
    return c.status;
}

bps_status check_scan(const char* what, const bps_scan& a, bool grad) {
    if (!known(a.dtype)) return fail_here(BPS_ERR_INVALID_ARG, "%s: unknown element type %d", what, a.dtype);
    if (a.states == 0 || a.states > bps::kMaxStates) return fail_here(BPS_ERR_INVALID_ARG, "%s: states=%u must be 1 .. %u", what, a.states, bps::kMaxStates);
    if (a.channels == 0 || a.channels >= kMaxChannels) return fail_here(BPS_ERR_INVALID_ARG, "%s: channels=%u must be 1 .. 2^24 - 1", what, a.channels);
    if (a.groups == 0 || a.channels % a.groups) return fail_here(BPS_ERR_INVALID_ARG, "%s: channels=%u must be a multiple of groups=%u", what, a.channels, a.groups);
    if (a.steps >= 1u << 31) return fail_here(BPS_ERR_INVALID_ARG, "%s: steps must be below 2^31", what);
    // at most 8 wavefronts for 64 channels of a group; time is cut where there are few of those only
    const uint64_t tiles = (uint64_t)a.groups * ((a.channels / a.groups + 63) / 64);
    if (a.batch * tiles >= kMaxThreads / 512 || (grad && (uint64_t)a.batch * a.steps * a.groups * 2 * bps::kMaxStates >= kMaxThreads - 256))
        return fail_here(BPS_ERR_UNSUPPORTED, "%s: too many elements for one launch", what);
    Checks c{what, a.batch, a.steps};
    for (const bps_sequence* s : {&a.x, &a.delta, &a.gate, &a.B, &a.C, &a.out, &a.grad_out, &a.grad_x, &a.grad_delta, &a.grad_gate, &a.grad_B, &a.grad_C})
        if (s->at && a.steps > 1 && (s->step_stride < 0 || s->step_stride >= kMaxStride)) return fail_here(BPS_ERR_INVALID_ARG, "%s: step strides must be 0 .. 2^26 - 1", what);
    const uint64_t kept = (uint64_t)a.states * a.channels, shared = (uint64_t)a.groups * a.states;
    c.pointer("A", a.A, 4, true);
    c.pointer("D", a.D, 4, false);
    c.pointer("delta_bias", a.delta_bias, 4, false);
    c.pointer("lengths", a.lengths, 4, false);
    c.input("x", a.x, a.dtype);
    c.input("delta", a.delta, a.dtype);
    c.input("gate", a.gate, a.dtype, false);
    c.input("B", a.B, a.dtype);
    c.input("C", a.C, a.dtype);
    c.pointer("held", a.held, 4, grad && a.batch && a.steps);
    if (grad) {
        c.input("grad_out", a.grad_out, a.dtype);
        c.result("grad_x", a.grad_x, a.dtype, a.channels);
        c.result("grad_delta", a.grad_delta, a.dtype, a.channels);
        if (a.gate.at) c.result("grad_gate", a.grad_gate, a.dtype, a.channels);
        c.result("grad_B", a.grad_B, a.dtype, shared);
        c.result("grad_C", a.grad_C, a.dtype, shared);
        c.pointer("grad_A", a.grad_A, 4, true);
        c.pointer("grad_D", a.grad_D, 4, a.D);
        c.pointer("grad_delta_bias", a.grad_delta_bias, 4, a.delta_bias);
    } else {
        c.result("out", a.out, a.dtype, a.channels);
        c.state("state", a.state, 4, a.state_stride, kept, false);
        c.state("state_out", a.state_out, 4, a.state_out_stride, kept, true);
        if (a.state_out && a.state_out == a.state && a.state_stride != a.state_out_stride) c.fail("state_out", "has another stride than the state that it is");
    }
    return c.status;
}

bps_status check_norm(const char* what, const bps_norm& a, bool grad) {
    if (!known(a.dtype)) return fail_here(BPS_ERR_INVALID_ARG, "%s: unknown element type %d", what, a.dtype);
    if (a.residual_dtype != a.dtype && a.residual_dtype != BPS_F32) return fail_here(BPS_ERR_INVALID_ARG, "%s: a residual of type %d for blocks of type %d", what, a.residual_dtype, a.dtype);
    if (a.weight_dtype != a.dtype && a.weight_dtype != BPS_F32) return fail_here(BPS_ERR_INVALID_ARG, "%s: weights of type %d for blocks of type %d", what, a.weight_dtype, a.dtype);
    if (a.activation != 0 && a.activation != 1) return fail_here(BPS_ERR_INVALID_ARG, "%s: unknown activation %d", what, a.activation);
    if (a.width == 0 || a.width > bps::kMaxNormWidth) return fail_here(BPS_ERR_INVALID_ARG, "%s: width=%u must be 1 .. %u", what, a.width, bps::kMaxNormWidth);
    if (a.rows >= 1ull << 40) return fail_here(BPS_ERR_INVALID_ARG, "%s: rows must be below 2^40", what);
    // the hardware's root takes what is smaller for nothing, and a row of zeros would be zero times infinity
    if (!(a.eps > 0.0f) || !std::isnormal(a.eps)) return fail_here(BPS_ERR_INVALID_ARG, "%s: eps must be positive, finite and no less than 2^-126", what);
    Checks c{what, 1, 1};
    const uint32_t size = size_of(a.dtype), stream_size = size_of(a.residual_dtype), weight_size = size_of(a.weight_dtype);
    const bool some = a.rows;
    auto rows = [&](const char* name, const void* p, uint32_t bytes, int64_t stride, bool needed, bool written) {
        c.pointer(name, p, bytes, needed && some);
        if (p && written && a.rows > 1 && distance(stride) < a.width) c.fail(name, "has rows that overlap");
    };
    rows("residual", a.residual, stream_size, a.residual_stride, true, false);
    rows("block", a.block, size, a.block_stride, true, false);
    rows("gate", a.gate, size, a.gate_stride, false, false);
    c.pointer("post_weight", a.post_weight, weight_size, false);
    c.pointer("scale", a.scale, weight_size, false);
    c.pointer("pre_weight", a.pre_weight, weight_size, false);
    c.pointer("roots", a.roots, 4, grad && some && (a.post_weight || a.pre_weight));
    if (grad) {
        rows("grad_residual_out", a.grad_residual_out, stream_size, a.grad_residual_out_stride, false, false);
        rows("grad_out", a.grad_out, size, a.grad_out_stride, false, false);
        rows("grad_residual", a.grad_residual, stream_size, a.grad_residual_stride, true, true);
        rows("grad_block", a.grad_block, size, a.grad_block_stride, true, true);
        rows("grad_gate", a.grad_gate, size, a.grad_gate_stride, a.gate, true);
        c.pointer("grad_post_weight", a.grad_post_weight, weight_size, a.post_weight);
        c.pointer("grad_scale", a.grad_scale, weight_size, a.scale);
        c.pointer("grad_pre_weight", a.grad_pre_weight, weight_size, a.pre_weight);
    } else {
        rows("residual_out", a.residual_out, stream_size, a.residual_out_stride, !a.pre_weight, true);
        rows("out", a.out, size, a.out_stride, a.pre_weight, true);
        if (a.residual_out && a.residual_out == a.residual && a.residual_stride != a.residual_out_stride) c.fail("residual_out", "has another stride than the residual that it is");
    }
    return c.status;
}

}  // namespace

extern "C" {

bps_status bps_causal_conv(const bps_conv* args, void* stream) {
    const char* what = "bps_causal_conv";
    if (!args) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (bps_status st = check_conv(what, *args, false)) return st;
    if (args->batch == 0 || (args->steps == 0 && !args->state_out)) return BPS_OK;
    return launched(what, bps::launch_conv(*args, static_cast<hipStream_t>(stream)));
}

size_t bps_causal_conv_backward_workspace(const bps_conv* args) {
    if (!args || !known(args->dtype) || args->taps == 0 || args->taps > bps::kMaxTaps || args->channels == 0 || args->channels >= kMaxChannels || args->steps >= 1u << 31) return 0;
    return bps::conv_grad_workspace(*args);
}

bps_status bps_causal_conv_backward(const bps_conv* args, void* workspace, size_t workspace_bytes, void* stream) {
    const char* what = "bps_causal_conv_backward";
    if (!args) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (bps_status st = check_conv(what, *args, true)) return st;
    if (bps_status st = check_workspace(what, bps::conv_grad_workspace(*args), workspace, workspace_bytes)) return st;
    return launched(what, bps::launch_conv_grad(*args, workspace, static_cast<hipStream_t>(stream)));
}

// Sizes that a plan can be made for; others are refused with a text by the call itself.
static bool scan_sizes(const bps_scan* a) {
    return a && known(a->dtype) && a->states && a->states <= bps::kMaxStates && a->channels && a->channels < kMaxChannels && a->groups && a->channels % a->groups == 0 && a->steps < 1u << 31;
}

size_t bps_selective_scan_workspace(const bps_scan* args) { return scan_sizes(args) ? bps::scan_workspace(*args) : 0; }

bps_status bps_selective_scan(const bps_scan* args, void* workspace, size_t workspace_bytes, void* stream) {
    const char* what = "bps_selective_scan";
    if (!args) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (bps_status st = check_scan(what, *args, false)) return st;
    if (args->batch == 0 || (args->steps == 0 && !args->state_out)) return BPS_OK;
    if (bps_status st = check_workspace(what, bps::scan_workspace(*args), workspace, workspace_bytes)) return st;
    return launched(what, bps::launch_scan(*args, workspace, static_cast<hipStream_t>(stream)));
}

size_t bps_selective_scan_backward_workspace(const bps_scan* args) { return scan_sizes(args) ? bps::scan_grad_workspace(*args) : 0; }

bps_status bps_selective_scan_backward(const bps_scan* args, void* workspace, size_t workspace_bytes, void* stream) {
    const char* what = "bps_selective_scan_backward";
    if (!args) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (bps_status st = check_scan(what, *args, true)) return st;
    if (bps_status st = check_workspace(what, bps::scan_grad_workspace(*args), workspace, workspace_bytes)) return st;
    return launched(what, bps::launch_scan_grad(*args, workspace, static_cast<hipStream_t>(stream)));
}

bps_status bps_residual_norm(const bps_norm* args, void* stream) {
    const char* what = "bps_residual_norm";
    if (!args) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (bps_status st = check_norm(what, *args, false)) return st;
    if (args->rows == 0) return BPS_OK;
    return launched(what, bps::launch_norm(*args, static_cast<hipStream_t>(stream)));
}

size_t bps_residual_norm_backward_workspace(const bps_norm* args) {
    if (!args || !known(args->dtype) || args->width == 0 || args->width > bps::kMaxNormWidth) return 0;
    return bps::norm_grad_workspace(*args);
}

bps_status bps_residual_norm_backward(const bps_norm* args, void* workspace, size_t workspace_bytes, void* stream) {
    const char* what = "bps_residual_norm_backward";
    if (!args) return fail_here(BPS_ERR_INVALID_ARG, "%s: null argument", what);
    if (bps_status st = check_norm(what, *args, true)) return st;
    if (bps_status st = check_workspace(what, bps::norm_grad_workspace(*args), workspace, workspace_bytes)) return st;
    return launched(what, bps::launch_norm_grad(*args, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
