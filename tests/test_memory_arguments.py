"""Refusals of the operators of a policy's memory: the C interface checks its arguments before it touches a device, with a status and a
text; the Python layer refuses tensors that do not fit before anything is read."""
import ctypes

import pytest

P = 4096          # an address that no check may look behind


def _memory():
    from paper_2103_07013_amd import memory
    memory._library()
    return memory


def _text():
    import paper_2103_07013_amd as bps
    return bps.bps_last_error()


def _sequences(a, names, batch, step):
    for n in names:
        if getattr(a, n) is None:
            setattr(a, n, P)
        setattr(a, n + "_batch_stride", batch)
        setattr(a, n + "_step_stride", step)


def _set(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _conv(backward=False, space=P, **kw):
    m = _memory()
    a = m._Conv(dtype=0, weight_dtype=0, batch=2, steps=3, channels=5, taps=4, silu=1, weight=P, bias=P, state=P, state_out=2 * P, state_stride=15, state_out_stride=15, grad_weight=P, grad_bias=P)
    _sequences(a, ("x", "out", "grad_out", "grad_x"), 15, 5)
    _set(a, kw)
    if backward:
        return m._library().bps_causal_conv_backward(a, space, 0 if space is None else 1 << 30, None)
    return m._library().bps_causal_conv(a, None)


@pytest.mark.parametrize("wrong,text", [(dict(dtype=3), "element type"), (dict(dtype=-1), "element type"), (dict(weight_dtype=1), "weights of type"), (dict(dtype=1, weight_dtype=2), "weights of type"),
                                        (dict(taps=0), "taps"), (dict(taps=9), "taps"), (dict(channels=0), "channels"), (dict(channels=1 << 24), "channels"), (dict(steps=1 << 31), "steps"),
                                        (dict(weight=None), "weight is null"), (dict(weight=P + 2), "weight is misaligned"), (dict(bias=P + 1), "bias is misaligned"), (dict(x=None), "x is null"),
                                        (dict(x=P + 2), "x is misaligned"), (dict(lengths=P + 2), "lengths is misaligned"), (dict(state=P + 1), "state is misaligned")])
def test_both_convolutions_refuse(wrong, text):
    for backward in (False, True):
        assert _conv(backward, **wrong) == -1 and text in _text()


@pytest.mark.parametrize("wrong,text", [(dict(out=None), "out is null"), (dict(out=P + 3), "out is misaligned"), (dict(out_step_stride=4), "overlap"), (dict(out_step_stride=0), "overlap"),
                                        (dict(out_batch_stride=14), "overlap"), (dict(out_batch_stride=0), "overlap"), (dict(out_step_stride=-4), "overlap"),
                                        (dict(out_step_stride=10, out_batch_stride=4), "overlap"), (dict(state_out_stride=14), "batches that overlap"), (dict(state_out=P), "state_out"),
                                        (dict(state_out=P, steps=1, state_out_stride=30), "state_out")])
def test_the_convolution_refuses(wrong, text):
    assert _conv(**wrong) == -1 and text in _text()


def test_rows_that_do_not_meet_are_no_overlap():
    """Time first, rows in reverse, batches between steps: what is refused is an argument that is checked later."""
    for strides in ((5, 10), (15, 5), (-15, 5), (15, -5), (5, -10), (100, 5), (5, 11)):
        assert _conv(out_batch_stride=strides[0], out_step_stride=strides[1], state_out=P + 1) == -1 and "state_out is misaligned" in _text()


@pytest.mark.parametrize("wrong,text", [(dict(grad_x=None), "grad_x is null"), (dict(grad_out=None), "grad_out is null"), (dict(grad_x_step_stride=4), "overlap"), (dict(grad_weight=None), "grad_weight is null"),
                                        (dict(grad_weight=P + 2), "misaligned"), (dict(grad_bias=P + 2), "misaligned"), (dict(space=None), "workspace"), (dict(space=P + 8), "workspace")])
def test_the_gradient_of_the_convolution_refuses(wrong, text):
    assert _conv(True, **wrong) == -1 and text in _text()


def test_calls_that_have_nothing_to_do():
    assert _conv(batch=0) == 0 and _conv(steps=0, state_out=None) == 0 and _scan(batch=0) == 0 and _scan(steps=0, state_out=None) == 0 and _norm(rows=0, residual=None, block=None) == 0


def test_too_many_elements_for_a_launch():
    assert _conv(batch=1 << 31, steps=1 << 10) not in (0, -1) and "too many" in _text()
    assert _scan(batch=1 << 26, steps=1) not in (0, -1) and "too many" in _text()


def _scan(backward=False, space=P, size=1 << 40, **kw):
    m = _memory()
    a = m._Scan(dtype=0, softplus=1, batch=2, steps=3, channels=6, states=4, groups=1, A=P, D=P, delta_bias=P, state=P, state_out=2 * P, state_stride=24, state_out_stride=24, held=P, grad_A=P,
                grad_D=P, grad_delta_bias=P)
    _sequences(a, ("x", "delta", "gate", "out", "grad_out", "grad_x", "grad_delta", "grad_gate"), 18, 6)
    _sequences(a, ("B", "C", "grad_B", "grad_C"), 12, 4)
    _set(a, kw)
    f = m._library().bps_selective_scan_backward if backward else m._library().bps_selective_scan
    return f(a, space, 0 if space is None else size, None)


@pytest.mark.parametrize("wrong,text", [(dict(dtype=3), "element type"), (dict(states=0), "states"), (dict(states=33), "states"), (dict(channels=0), "channels"), (dict(channels=1 << 24), "channels"),
                                        (dict(groups=0), "groups"), (dict(groups=4), "groups"), (dict(steps=1 << 31), "steps"), (dict(A=None), "A is null"), (dict(A=P + 2), "A is misaligned"),
                                        (dict(D=P + 1), "D is misaligned"), (dict(delta_bias=P + 2), "delta_bias is misaligned"), (dict(x=None), "x is null"), (dict(delta=None), "delta is null"),
                                        (dict(B=None), "B is null"), (dict(C=None), "C is null"), (dict(gate=P + 2), "gate is misaligned"), (dict(held=P + 2), "held is misaligned"),
                                        (dict(lengths=P + 1), "lengths"), (dict(x_step_stride=-6), "step strides"), (dict(C_step_stride=1 << 26), "step strides")])
def test_both_scans_refuse(wrong, text):
    for backward in (False, True):
        assert _scan(backward, **wrong) == -1 and text in _text()


@pytest.mark.parametrize("wrong,text", [(dict(out=None), "out is null"), (dict(out_step_stride=5), "overlap"), (dict(out_batch_stride=17), "overlap"), (dict(state=P + 2), "state is misaligned"),
                                        (dict(state_out_stride=23), "batches that overlap"), (dict(state_out=P, state_out_stride=48), "state_out")])
def test_the_scan_refuses(wrong, text):
    assert _scan(**wrong) == -1 and text in _text()


@pytest.mark.parametrize("wrong,text", [(dict(held=None), "held is null"), (dict(grad_out=None), "grad_out is null"), (dict(grad_x=None), "grad_x is null"), (dict(grad_delta=None), "grad_delta is null"),
                                        (dict(grad_gate=None), "grad_gate is null"), (dict(grad_B=None), "grad_B is null"), (dict(grad_C_step_stride=3), "overlap"), (dict(grad_A=None), "grad_A is null"),
                                        (dict(grad_D=None), "grad_D is null"), (dict(grad_delta_bias=None), "grad_delta_bias is null"), (dict(space=None), "workspace"), (dict(size=64), "workspace")])
def test_the_gradient_of_the_scan_refuses(wrong, text):
    assert _scan(True, **wrong) == -1 and text in _text()


def test_a_scan_in_chunks_needs_its_workspace():
    long = dict(batch=1, steps=4096)
    assert _scan(space=None, **long) == -1 and "workspace" in _text()
    assert _scan(size=1024, **long) == -1 and "workspace" in _text()


def _norm(backward=False, space=P, size=1 << 30, **kw):
    m = _memory()
    a = m._Norm(dtype=1, residual_dtype=0, weight_dtype=0, activation=0, rows=2, width=6, eps=1e-6, residual=P, block=P, gate=P, residual_stride=6, block_stride=6, gate_stride=6, post_weight=P, scale=P,
                pre_weight=P, residual_out=2 * P, out=P, residual_out_stride=6, out_stride=6, roots=P, grad_residual_out=P, grad_out=P, grad_residual_out_stride=6, grad_out_stride=6, grad_residual=P,
                grad_block=P, grad_gate=P, grad_residual_stride=6, grad_block_stride=6, grad_gate_stride=6, grad_post_weight=P, grad_scale=P, grad_pre_weight=P)
    _set(a, kw)
    if backward:
        return m._library().bps_residual_norm_backward(a, space, 0 if space is None else size, None)
    return m._library().bps_residual_norm(a, None)


@pytest.mark.parametrize("wrong,text", [(dict(dtype=5), "element type"), (dict(residual_dtype=2), "residual of type"), (dict(weight_dtype=2), "weights of type"), (dict(activation=2), "activation"),
                                        (dict(width=0), "width"), (dict(width=16385), "width"), (dict(rows=1 << 40), "rows"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"),
                                        (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"), (dict(residual=None), "residual is null"), (dict(block=None), "block is null"),
                                        (dict(residual=P + 2), "residual is misaligned"), (dict(block=P + 1), "block is misaligned"), (dict(gate=P + 1), "gate is misaligned"),
                                        (dict(scale=P + 2), "scale is misaligned"), (dict(roots=P + 2), "roots is misaligned")])
def test_both_norms_refuse(wrong, text):
    for backward in (False, True):
        assert _norm(backward, **wrong) == -1 and text in _text()


@pytest.mark.parametrize("wrong,text", [(dict(out=None), "out is null"), (dict(pre_weight=None, residual_out=None), "residual_out is null"), (dict(out_stride=5), "overlap"),
                                        (dict(residual_out_stride=-5), "overlap"), (dict(residual_out=P, residual_out_stride=7), "residual_out")])
def test_the_norm_refuses(wrong, text):
    assert _norm(**wrong) == -1 and text in _text()


@pytest.mark.parametrize("wrong,text", [(dict(roots=None), "roots is null"), (dict(grad_residual=None), "grad_residual is null"), (dict(grad_block=None), "grad_block is null"),
                                        (dict(grad_gate=None), "grad_gate is null"), (dict(grad_scale=None), "grad_scale is null"), (dict(grad_post_weight=None), "grad_post_weight is null"),
                                        (dict(grad_pre_weight=None), "grad_pre_weight is null"), (dict(grad_block_stride=0), "overlap"), (dict(grad_out=P + 1), "misaligned"), (dict(space=None), "workspace"),
                                        (dict(size=8), "workspace")])
def test_the_gradient_of_the_norm_refuses(wrong, text):
    assert _norm(True, **wrong) == -1 and text in _text()


def test_null_arguments():
    lib = _memory()._library()
    for name in ("bps_causal_conv", "bps_residual_norm"):
        assert getattr(lib, name)(None, None) == -1 and "null" in _text()
    for name in ("bps_causal_conv_backward", "bps_selective_scan", "bps_selective_scan_backward", "bps_residual_norm_backward"):
        assert getattr(lib, name)(None, None, 0, None) == -1 and "null" in _text()
        if name != "bps_selective_scan":
            assert getattr(lib, name + "_workspace")(None) == 0


def test_structures_are_as_large_as_the_header_says(tmp_path):
    """The binding's and the library's layouts of the arguments agree."""
    import os
    import subprocess
    m = _memory()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = {"bps_conv": m._Conv, "bps_scan": m._Scan, "bps_norm": m._Norm}
    last = {"bps_conv": "grad_bias", "bps_scan": "grad_delta_bias", "bps_norm": "grad_pre_weight"}
    (tmp_path / "s.c").write_text('#include "bps_memory.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {' + "".join(
        f'printf("%zu %zu ", sizeof({n}), offsetof({n}, {last[n]}));' for n in names) + "}")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    said = [int(v) for v in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()]
    assert said == [v for n, c in names.items() for v in (ctypes.sizeof(c), getattr(c, last[n]).offset)]


def test_the_library_exports_what_its_header_declares():
    import os
    import re
    m = _memory()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "bps_memory.h")).read(), flags=re.S)
    declared = re.findall(r"^(?:bps_status|size_t)\s+(bps_\w+)\(", text, flags=re.M)
    assert set(declared) == set(m.EXPORTS) and all(hasattr(m._library(), n) for n in declared)


def test_tensors_of_the_processor_are_refused():
    import torch
    import paper_2103_07013_amd as bps
    x, w = torch.zeros(2, 3, 4), torch.zeros(4, 4)
    with pytest.raises(ValueError, match="CUDA"):
        bps.causal_conv(x, w)
    with pytest.raises(ValueError, match="CUDA"):
        bps.causal_conv_step(x[:, 0], torch.zeros(2, 3, 4), w)
    with pytest.raises(ValueError, match="CUDA"):
        bps.selective_scan(x, x, torch.zeros(5, 4), torch.zeros(2, 3, 5), torch.zeros(2, 3, 5))
    with pytest.raises(ValueError, match="CUDA"):
        bps.residual_norm(x, x)
