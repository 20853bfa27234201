/* The stand-in for the HIP runtime (fake_hip.c) with a line for every launch that says how large it is, with what the runtime
 * refuses (a grid of 2^32 threads or more along x, or more than 65535 work-groups along y), and with the last error, which stays until it is read. */
#define hipLaunchKernel fake_plain_launch
#define hipGetLastError fake_no_last_error
#define hipMalloc fake_plain_malloc
#include "fake_hip.c"
#undef hipLaunchKernel
#undef hipGetLastError
#undef hipMalloc

static hipError_t g_last;
hipError_t hipGetLastError(void) {
    const hipError_t e = g_last;
    g_last = hipSuccess;
    return e;
}
static hipError_t kept(hipError_t e) {
    if (e != hipSuccess) g_last = e;
    return e;
}
hipError_t hipMalloc(void** p, size_t n) { return kept(fake_plain_malloc(p, n)); }

static char g_launches[1 << 16];
static size_t g_launches_at;
const char* fake_launches(void) { return g_launches; }
void fake_clear_launches(void) { g_launches[g_launches_at = 0] = 0; }

hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t shared, hipStream_t stream) {
    (void)args; (void)stream;
    const size_t room = sizeof(g_launches) - g_launches_at;
    const int n = snprintf(g_launches + g_launches_at, room, "%s grid=%ux%u threads=%u lds=%zu\n", kernel_name(f), grid.x, grid.y, block.x, shared);
    if (n < 0 || (size_t)n >= room) abort();
    g_launches_at += (size_t)n;
    return kept((uint64_t)grid.x * block.x >> 32 || grid.y > 65535 ? hipErrorInvalidConfiguration : hipSuccess);
}
hipError_t hipGetDevice(int* device) { *device = 0; return hipSuccess; }
