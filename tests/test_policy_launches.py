"""Which kernels the policy's operators launch, without a GPU: libbps.so runs on a stand-in for the HIP runtime
(fake_hip_launches.c) that notes every launch, and no kernel runs."""
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
lib = bps.load_library()
p, i, u, l, f = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float
lib.bps_log_probs_workspace.restype, lib.bps_log_probs_workspace.argtypes = ctypes.c_size_t, [i, l, u, u]
lib.bps_log_probs.argtypes = [p, i, l, u, l, p, i, p, l, f, u, p, p, p, p, p, p, p, l, p]
P = 4096          # an address that nothing looks behind

def scores(rows, entries, k=0, dtype=1):
    size = lib.bps_log_probs_workspace(dtype, rows, entries, k)
    top = P if k else None
    fake.fake_clear_launches()
    status = lib.bps_log_probs(P, dtype, rows, entries, 0, P, 64, None, 0, 1.0, k, P, P, P, P, top, top, P if size else None, size, None)
    assert status == 0, bps.bps_last_error()
    print("workspace=%d" % size)
    print(fake.fake_launches().decode(), end="")
"""


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("fake") / "fake_hip_launches.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "fake_hip_launches.c"), "-o", so], check=True)
    return so


def _calls(fake, code):
    """What the calls in `code` print and launch: (what was printed before, [(kernel, work-groups, threads of each)]) of each call."""
    p = subprocess.run([sys.executable, "-c", PRELUDE + code, fake], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout + p.stderr
    calls = []
    for line in p.stdout.splitlines():
        m = re.match(r"_ZN3bps\S*?\d(k_[a-z_]+)I?\S* grid=(\d+)x(\d+) threads=(\d+)", line)
        if m:
            calls[-1][1].append((m[1], int(m[2]) * int(m[3]), int(m[4])))
        else:
            calls.append((line, []))
    return calls


@pytest.mark.parametrize("k", [0, 20])
@pytest.mark.parametrize("parts,left", [(1, 1), (1, 10), (1, 64), (2, 3), (1, 65), (1, 5000)])
def test_rows_behind_a_launch_are_cut_into_pieces_only_with_a_workspace(fake, parts, left, k):
    """A call of more rows than a launch takes has many rows, however few the last launch is left with: no row is cut into pieces, whose sums would
    need the workspace that such a call does not have, and all launches run the same kernel."""
    (said, launches), = _calls(fake, f"scores({parts} * 2 ** 21 + {left}, 40000, {k})")
    assert said == "workspace=0"
    assert [name for name, _, _ in launches] == ["k_score"] * (parts + 1)
    assert launches[-1][1:] == (left, launches[0][2])


def test_few_long_rows_are_cut_into_pieces(fake):
    (said, launches), = _calls(fake, "scores(10, 40000, 3)")
    assert int(said.split("=")[1]) > 0 and [name for name, _, _ in launches] == ["k_score_piece", "k_score_join"]


ADAMW = """
class Tensor(ctypes.Structure):
    _fields_ = [("param", p), ("master", p), ("count", l), ("start", l), ("weight_decay", f), ("lr_scale", f)]

class Config(ctypes.Structure):
    _fields_ = [("param_dtype", i), ("state_bits", i), ("tensors", u), ("seed", u), ("total", l), ("tensor", ctypes.POINTER(Tensor)), ("exp_avg", p), ("exp_avg_sq", p),
                ("exp_avg_exponent", p), ("exp_avg_sq_exponent", p)]

def create(*tensors, dtype=0):
    '''tensors: (address, master's address, elements)'''
    rows, start = [], 0
    for at, master, n in tensors:
        rows.append(Tensor(at, master, n, start, 0.0, 1.0))
        start += -(-n // 256) * 256
    out = p()
    status = lib.bps_adamw_create(ctypes.byref(Config(dtype, 32, len(rows), 0, start, (Tensor * len(rows))(*rows), P, P, None, None)), ctypes.byref(out))
    print(status, bps.bps_last_error() if status else "")
    lib.bps_adamw_destroy(out)
"""


@pytest.mark.parametrize("tensors,dtype,fits", [("(P, None, 10), (P + 40, None, 10)", 0, True), ("(P + 40, None, 300), (P, None, 10)", 0, True), ("(P, None, 10), (P, None, 10)", 0, False),
                                                ("(P, None, 10), (P + 36, None, 10)", 0, False), ("(P + 4000, None, 1), (P, None, 1001), (P + 8000, None, 9)", 0, False),
                                                ("(P, 2 * P, 10), (P + 20, 2 * P + 40, 10)", 1, True), ("(P, 2 * P, 10), (P + 18, 2 * P + 40, 10)", 1, False),
                                                ("(P, 2 * P, 10), (P + 20, 2 * P + 36, 10)", 1, False), ("(P, P + 4, 10),", 1, False)])
def test_tensors_that_share_memory_are_refused(fake, tensors, dtype, fits):
    """A step would write to shared elements from two work-groups, in no order."""
    (said, _), = _calls(fake, ADAMW + f"create({tensors} dtype={dtype})" if tensors.endswith(",") else ADAMW + f"create({tensors}, dtype={dtype})")
    assert said.startswith("0" if fits else "-1") and ("overlap" in said) == (not fits)


def test_a_plan_that_does_not_fit_leaves_no_error_behind(fake):
    """The runtime keeps the last error until it is read: the next launch, the library's or torch's, would be taken for a failure."""
    (failed, _), (said, launches) = _calls(fake, ADAMW + """
fake.fake_largest(0, ctypes.c_size_t(0))
create((P, None, 10))
scores(10, 100)
""")
    assert failed.startswith("-3") and "hipMalloc" in failed and said == "workspace=0" and len(launches) == 1


EMBEDDING = """
lib.bps_embedding_backward_workspace.restype, lib.bps_embedding_backward_workspace.argtypes = ctypes.c_size_t, [l, u, u]
lib.bps_embedding_backward.argtypes = [p, i, l, p, i, u, u, l, f, p, i, l, i, p, l, p]

def gradient(count, rows, width, dtype=0, accumulate=0):
    size = lib.bps_embedding_backward_workspace(count, rows, width)
    fake.fake_clear_launches()
    status = lib.bps_embedding_backward(P, 32, count, P, dtype, rows, width, width, 1.0, P, 0, width, accumulate, P if size else None, size, None)
    assert status == 0, bps.bps_last_error()
    print("workspace=%d" % size)
    print(fake.fake_launches().decode(), end="")
"""


@pytest.mark.parametrize("dtype,rows", [(0, 1), (0, 16), (1, 8)])
@pytest.mark.parametrize("count", [5, 16384])
@pytest.mark.parametrize("width", [1 << 20, 20_000_000, 300_000_000, (1 << 30) - 1])
def test_tables_of_few_rows_of_any_width(fake, width, count, rows, dtype):
    """No launch is larger than the runtime takes, however wide the rows are, and the workspace does not grow without end."""
    (said, launches), = _calls(fake, EMBEDDING + f"gradient({count}, {rows}, {width}, {dtype})")
    assert {name for name, _, _ in launches} == {"k_embed_few", "k_embed_few_join"}
    # a work-group takes 64 lanes of columns of a part of the tokens, or 16 sums of the result: all of them are there
    lanes = 64 * (8 if dtype else 4)
    assert sum(n for name, n, _ in launches if name == "k_embed_few") >= -(-width // lanes) * (1 if count == 5 else 256)
    assert sum(n for name, n, _ in launches if name == "k_embed_few_join") >= -(-rows * width // 16)


@pytest.mark.parametrize("count,rows,width", [(1, 1, 1), (33, 1000, 1), (9000, 17, 3), (1 << 20, (1 << 30) - 1, 1), ((1 << 31) - 1, 40, 1), (20000, 100, 1 << 20), (0, (1 << 30) - 1, 8)])
def test_sorted_gradients_of_any_size(fake, count, rows, width):
    _calls(fake, EMBEDDING + f"gradient({count}, {rows}, {width})\ngradient({count}, {rows}, {width}, accumulate=1)")
