"""Which kernels the operators of a policy's memory launch, without a GPU: libbps_memory.so runs on a stand-in for the HIP runtime
(fake_hip_launches.c, with room for both libraries' kernels) that notes every launch and refuses those that the runtime refuses."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PRELUDE = """
import ctypes, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)      # found before the real runtime
fake.fake_launches.restype = ctypes.c_char_p
import paper_2103_07013_amd as bps          # without torch, whose kernels the stand-in has no room for
from paper_2103_07013_amd import build
bps.load_library()
lib = ctypes.CDLL(build.MEMORY_LIB)
p, i, u, l, f, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
P = 1 << 40          # addresses that nothing looks behind

class Seq(ctypes.Structure):
    _fields_ = [("at", p), ("batch", l), ("step", l)]
class Conv(ctypes.Structure):
    _fields_ = [("dtype", i), ("weight_dtype", i), ("batch", u), ("steps", u), ("channels", u), ("taps", u), ("silu", i), ("x", Seq), ("out", Seq), ("weight", p), ("bias", p), ("starts", Seq),
                ("lengths", p), ("state", p), ("state_out", p), ("state_stride", l), ("state_out_stride", l), ("grad_out", Seq), ("grad_x", Seq), ("grad_weight", p), ("grad_bias", p)]
class Scan(ctypes.Structure):
    _fields_ = [("dtype", i), ("softplus", i), ("batch", u), ("steps", u), ("channels", u), ("states", u), ("groups", u), *((n, Seq) for n in ("x", "delta", "gate", "B", "C", "out")), ("A", p), ("D", p),
                ("delta_bias", p), ("starts", Seq), ("lengths", p), ("state", p), ("state_out", p), ("state_stride", l), ("state_out_stride", l), ("held", p),
                *((n, Seq) for n in ("grad_out", "grad_x", "grad_delta", "grad_gate", "grad_B", "grad_C")), ("grad_A", p), ("grad_D", p), ("grad_delta_bias", p)]
for name in ("bps_causal_conv_backward", "bps_selective_scan", "bps_selective_scan_backward"):
    getattr(lib, name + "_workspace").restype = size
    getattr(lib, name).argtypes = [p, p, size, p]
lib.bps_causal_conv.argtypes = [p, p]

def run(name, a):
    fake.fake_clear_launches()
    if name == "bps_causal_conv":
        status, need = lib.bps_causal_conv(ctypes.byref(a), None), 0
    else:
        need = getattr(lib, name + "_workspace")(ctypes.byref(a))
        status = getattr(lib, name)(ctypes.byref(a), P if need else None, need, None)
    print("status=%d workspace=%d %s" % (status, need, bps.bps_last_error() if status else ""))
    print(fake.fake_launches().decode(), end="")

def conv(batch, steps, channels, taps=4, dtype=1):
    s = Seq(P, steps * channels, channels)
    a = Conv(dtype, dtype, batch, steps, channels, taps, 1, s, s, P, P, Seq(), None, None, P, 0, (taps - 1) * channels, s, s, P, P)
    run("bps_causal_conv", a)
    run("bps_causal_conv_backward", a)

def scan(batch, steps, channels, states=16, groups=1, dtype=1, held=True):
    s, b = Seq(P, steps * channels, channels), Seq(P, steps * groups * states, groups * states)
    a = Scan(dtype, 1, batch, steps, channels, states, groups, s, s, s, b, b, s, P, P, P, Seq(), None, None, P, 0, states * channels, P if held else None, s, s, s, s, b, b, P, P, P)
    run("bps_selective_scan", a)
    if held:
        run("bps_selective_scan_backward", a)
"""


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    where = tmp_path_factory.mktemp("fake")
    for name in ("fake_hip.c", "fake_hip_launches.c"):
        with open(os.path.join(ROOT, "tests", name)) as f:
            (where / name).write_text(f.read().replace("g_kernels[256]", "g_kernels[1024]").replace("g_n_kernels == 256", "g_n_kernels == 1024"))
    so = str(where / "fake_hip_launches.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-I/opt/rocm/include", str(where / "fake_hip_launches.c"), "-o", so], check=True)
    return so


def _calls(fake, code):
    """What each call says and launches: (status, workspace, [(kernel, work-groups, threads of each)])."""
    p = subprocess.run([sys.executable, "-c", PRELUDE + code, fake], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout + p.stderr
    calls = []
    for line in p.stdout.splitlines():
        m = re.match(r"_ZN3bps\S*?\d(k_[a-z_]+)I?\S* grid=(\d+)x(\d+) threads=(\d+)", line)
        if m:
            calls[-1][2].append((m[1], int(m[2]) * int(m[3]), int(m[4])))
        else:
            said = re.match(r"status=(-?\d+) workspace=(\d+) (.*)", line)
            calls.append((int(said[1]), int(said[2]), []))
            assert said[1] == "0" or "too many" in said[3], said[3]
    return calls


@pytest.mark.parametrize("batch,steps,channels", [(1, 1, 1), (1, 1 << 24, 1), (1024, 1, 512), (1 << 20, 1, 64), (3, 5003, 1111), (1, 16384, 4096), (1 << 16, 128, 100), (1, 1, (1 << 24) - 1), (1, 0, 5)])
@pytest.mark.parametrize("dtype,taps", [(0, 1), (1, 4), (2, 8)])
def test_every_element_of_a_convolution_has_a_thread(fake, batch, steps, channels, dtype, taps):
    (status, _, forward), (back, _, backward) = _calls(fake, f"conv({batch}, {steps}, {channels}, {taps}, {dtype})")
    assert status == 0 and back == 0
    (name, groups, threads), = forward
    vectors = -(-channels // (8 if dtype else 4))
    runs = groups * threads / (batch * vectors)
    assert name == "k_conv" and runs >= 1 and (steps == 0 or runs * 64 >= steps)
    assert [n for n, _, _ in backward] == (["k_conv_grad"] if steps else []) + ["k_join_parts"]


@pytest.mark.parametrize("batch,steps,channels,states,groups", [(1, 1, 1, 1, 1), (8, 4096, 2048, 16, 1), (1, 16384, 2048, 16, 1), (1024, 32, 512, 16, 1), (7, 1111, 778, 13, 2), (1, 1 << 20, 64, 32, 1),
                                                                (1 << 20, 4, 64, 16, 1), (2, 64, 66, 5, 2), (1, 1, 4096, 4, 64), (3, 0, 12, 4, 1), (1000, 40, 20, 32, 4), (2, 4096, 40, 20, 1), (1, 300, 17, 1, 1), (1, 1, (1 << 24) - 1, 32, 1),
                                                                (1, 2, (1 << 22) - 1, 1, (1 << 22) - 1), ((1 << 23) - 1, 2, 64, 1, 1)])
def test_every_step_of_a_scan_is_in_a_chunk(fake, batch, steps, channels, states, groups):
    (status, space, forward), (back, back_space, backward) = _calls(fake, f"scan({batch}, {steps}, {channels}, {states}, {groups})")
    assert status == 0 and back == 0

    def tiles(threads, lanes):
        """Work-groups for all sequences' channels: a wavefront has 64 / lanes of them."""
        return batch * groups * -(-(channels // groups) // (threads // lanes))

    def cut(first, last, lanes):
        """A pass over all chunks but one, and the one over all of them."""
        chunks = last[1] // tiles(last[2], lanes)
        assert last[1] == chunks * tiles(last[2], lanes) and first[1] == (chunks - 1) * tiles(first[2], lanes) and first[2] == last[2]
        assert chunks > 1 and steps // chunks >= 32 and last[1] * last[2] <= 1024 * 64 * lanes

    names = [n for n, _, _ in forward]
    if len(names) == 3:
        assert names == ["k_scan", "k_scan_join", "k_scan"] and space > 0
        cut(forward[0], forward[2], 4)
    else:
        assert names == ["k_scan"] and space == 0 and forward[0][1] == tiles(forward[0][2], 4)
    names = [n for n, _, _ in backward]
    last = (["k_scan_grad", "k_scan_grad_shared"] if steps else []) + ["k_join_parts"]
    assert names in (last, ["k_scan_grad_first", "k_scan_join", *last]) and back_space > 0


def test_a_step_is_one_launch_without_a_workspace(fake):
    for batch, channels, groups in ((1, 1, 1), (1024, 512, 1), (3, 1030, 2), (100000, 8, 1)):
        (status, space, launches), = _calls(fake, f"scan({batch}, 1, {channels}, 16, {groups}, held=False)")
        assert status == 0 and space == 0 and launches == [("k_scan_step", batch * groups * -(-(channels // groups) // 256), 256)]


def test_calls_that_are_too_large_are_refused(fake):
    """They launch nothing; the largest that are not refused launch no more than the runtime takes."""
    for code in ("conv(1 << 22, 1 << 14, 64)", "scan(1 << 26, 2, 64)", "scan(1 << 23, 1, 64)", "scan(1 << 20, 4096, 64, 16, 64)"):
        for status, _, launches in _calls(fake, code):
            assert status != 0 and not launches
