"""MI355X-native batch renderer for large-batch simulation (arXiv 2103.07013, Sec. 3.2), and operators of the policy
that consumes its frames (Sec. 3.3, 3.4).

Thin ctypes binding over libbps.so and libbps_memory.so, the C-ABI libraries declared in include/bps.h and bps_memory.h.  Every
step of rendering, and each operator, runs in the library's HIP kernels; this package only marshals arguments.
PyTorch is used for device memory and streams.  There is no CPU fallback: if the library
is missing or no GPU is present, calls raise.
"""
from .binding import (BpsError, Renderer, bps_create, bps_destroy, bps_last_error, bps_last_kernel_ms, bps_kernel_ms_total, bps_kernel_ms_each, bps_set_diagnostics, bps_read_diagnostics,
                      bps_load_scene, bps_load_scene_async, bps_load_scene_textured, bps_scene_ready, bps_pack_clusters, bps_query, bps_render, bps_render_static, bps_set_profiling, bps_unload_scene, load_library,
                      MODE_DEPTH, MODE_RGBD, FLAG_NO_CLUSTER_CULL, FLAG_NO_OCCLUSION_CULL, FLAG_NO_DISPATCH_ORDER, FLAG_INPUTS_READY, FLAG_BILINEAR, EXPORTS)

__all__ = ["BpsError", "Renderer", "bps_create", "bps_destroy", "bps_last_error", "bps_last_kernel_ms", "bps_kernel_ms_total", "bps_kernel_ms_each", "bps_set_diagnostics", "bps_read_diagnostics",
           "bps_load_scene", "bps_load_scene_async", "bps_load_scene_textured", "bps_scene_ready", "bps_pack_clusters", "bps_query", "bps_render", "bps_render_static", "bps_set_profiling", "bps_unload_scene", "load_library",
           "MODE_DEPTH", "MODE_RGBD", "FLAG_NO_CLUSTER_CULL", "FLAG_NO_OCCLUSION_CULL", "FLAG_NO_DISPATCH_ORDER", "FLAG_INPUTS_READY", "FLAG_BILINEAR", "EXPORTS"]

# The policy's operators need torch from the start, the renderer only where it is given torch's tensors: they are imported when they are
# first asked for, and not by `import *`.
_POLICY = ("log_probs", "log_probs_backward", "LogProbs", "embedding", "embedding_backward", "AdamW")
_MEMORY = ("causal_conv", "causal_conv_backward", "causal_conv_step", "CausalConv", "ConvGrads", "selective_scan", "selective_scan_backward", "selective_scan_step", "SelectiveScan",
           "ScanGrads", "residual_norm", "residual_norm_backward", "ResidualNorm", "NormGrads")


def __dir__():
    return sorted({*globals(), *_POLICY, *_MEMORY})


def __getattr__(name):
    if name in _POLICY or name in _MEMORY:
        from . import memory, policy
        globals().update((n, getattr(module, n)) for module, names in ((policy, _POLICY), (memory, _MEMORY)) for n in names)
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
