"""Builds libbps.so (the C-ABI batch renderer) and libbps_memory.so (operators of a policy's memory, beside it) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbps.so")
MEMORY_LIB = os.path.join(HERE, "libbps_memory.so")
SOURCES = ["bps_api.hip", "raster_kernels.hip", "shade_kernels.hip", "clusters.cpp",
           "policy_api.hip", "score_kernels.hip", "embedding_kernels.hip", "adamw_kernels.hip"]
MEMORY_SOURCES = ["memory_api.hip", "conv_kernels.hip", "scan_kernels.hip", "norm_kernels.hip"]
HEADERS = ["raster_kernels.h", "raster_device.h", "clusters.h", "policy_kernels.h", "policy_device.h", os.path.join("..", "..", "include", "bps.h")]
MEMORY_HEADERS = ["memory_kernels.h", "memory_device.h", "policy_device.h", os.path.join("..", "..", "include", "bps.h"), os.path.join("..", "..", "include", "bps_memory.h")]
# -ffp-contract=off: the numeric rule fixes where fused multiply-adds happen.
# packed FP32 instructions are switched off on purpose (hipcc's host pass does not know the
# feature and says so; that message is harmless).
# -amdgpu-atomic-optimizer-strategy=None: the kernels add up over a wavefront themselves and let one lane
# do the atomic; the compiler's own combining would wrap that lane in a second reduction (a dozen
# instructions around every work counter in LDS).
HIPCC_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-ffp-contract=off", "-fPIC", "-shared",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-mllvm", "-amdgpu-atomic-optimizer-strategy=None"]


def stale() -> bool:
    for lib, files in ((LIB, SOURCES + HEADERS), (MEMORY_LIB, MEMORY_SOURCES + MEMORY_HEADERS)):
        if not os.path.exists(lib) or any(os.path.getmtime(os.path.join(CSRC, f)) > os.path.getmtime(lib) for f in files):
            return True
    return False


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile every HIP source into paper_2103_07013_amd/libbps.so and libbps_memory.so, which finds the former beside it."""
    if not force and not stale():
        return LIB
    _make([(SOURCES, LIB, []), _memory()], verbose)
    return LIB


def build_memory(verbose: bool = False) -> str:
    """Compile libbps_memory.so alone, beside the libbps.so that is there and may be loaded."""
    _make([_memory()], verbose)
    return MEMORY_LIB


def _memory():
    return MEMORY_SOURCES, MEMORY_LIB, ["-L" + HERE, "-lbps", "-Wl,-rpath,$ORIGIN"]


def compile_hip(sources, lib: str, verbose: bool = False) -> str:
    """Compile HIP sources into one shared library with the flags that the numeric rule needs."""
    _make([([os.path.abspath(s) for s in sources], lib, [])], verbose)
    return lib


def _make(libs, verbose):
    """libs: (sources, library, what it is linked with), a library after those that it is linked with.  All sources are compiled by
    themselves, as many at a time as there are processors to give."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(lib, arguments):
        res = subprocess.run([hipcc, *HIPCC_FLAGS, *arguments], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if verbose or res.returncode != 0:
            print(res.stdout)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed building %s:\n" % os.path.basename(lib) + res.stdout)

    with tempfile.TemporaryDirectory() as objects, concurrent.futures.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        made, jobs = [], []
        for sources, lib, link in libs:
            names = [os.path.join(objects, "%d_%d.o" % (len(made), k)) for k in range(len(sources))]
            jobs += [pool.submit(run, lib, ["-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(sources, names)]
            made.append((names, lib, link))
        for job in jobs:
            job.result()
        for names, lib, link in made:
            run(lib, [*names, *link, "-o", lib])


if __name__ == "__main__":
    print(build(force=True, verbose=True))
