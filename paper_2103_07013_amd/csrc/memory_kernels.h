// Operators of a policy's memory (the recurrent block between a policy's embedding and its scores), written for gfx950: a short
// causal convolution, a selective state space scan, and the norms around a block.
// Launchers only; arguments are checked in memory_api.hip, and every launcher relies on what is said there.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/bps_memory.h"

namespace bps {

bps_status fail_here(bps_status code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

constexpr uint32_t kMaxTaps = 8;
constexpr uint32_t kMaxStates = 32;
constexpr uint32_t kMaxNormWidth = 16384;
constexpr uint32_t kHeldSteps = 16;       // a scan's states are held before each step whose number is a multiple of this

hipError_t launch_conv(const bps_conv& a, hipStream_t stream);
size_t conv_grad_workspace(const bps_conv& a);
hipError_t launch_conv_grad(const bps_conv& a, void* workspace, hipStream_t stream);

size_t scan_workspace(const bps_scan& a);
hipError_t launch_scan(const bps_scan& a, void* workspace, hipStream_t stream);
size_t scan_grad_workspace(const bps_scan& a);
hipError_t launch_scan_grad(const bps_scan& a, void* workspace, hipStream_t stream);

hipError_t launch_norm(const bps_norm& a, hipStream_t stream);
size_t norm_grad_workspace(const bps_norm& a);
hipError_t launch_norm_grad(const bps_norm& a, void* workspace, hipStream_t stream);

// Sums of what work-groups left in parts, `stride` floats apart: out[d * inner + k] = sum over the parts of parts[p][k][d], for d < width
// and k < inner, as `dtype`.
struct JoinJob {
    const float* parts;
    void* out;
    uint32_t width, inner;
    int32_t dtype;
};
struct JoinJobs {
    JoinJob job[3];
    uint32_t count = 0;
    void add(const float* parts, uint32_t width, uint32_t inner, int32_t dtype, void* out) { job[count++] = {parts, out, width, inner, dtype}; }
};
hipError_t launch_join_parts(const JoinJobs& jobs, uint32_t count, size_t stride, hipStream_t stream);

}  // namespace bps
