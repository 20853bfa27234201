"""What the Python layer of the memory's operators refuses before it looks at devices, where a call would lose part of a gradient: tried on the
CPU's tensors, which it refuses for their device otherwise."""
import pytest


def _calls():
    """Both calls that take a state, with what they are given for it and for one other input."""
    import torch
    import paper_2103_07013_amd as bps
    x, b = torch.zeros(2, 5, 8), torch.zeros(2, 5, 4)
    conv = dict(x=x, weight=torch.zeros(8, 4), bias=torch.zeros(8), state=torch.zeros(2, 3, 8))
    scan = dict(x=x, delta=x.clone(), A=-torch.ones(4, 8), B=b, C=b.clone(), D=torch.zeros(8), gate=x.clone(), delta_bias=torch.zeros(8), state=torch.zeros(2, 4, 8))
    return (bps.causal_conv, conv), (bps.selective_scan, scan)


def test_states_that_ask_for_a_gradient_are_refused_beside_any_other_input_that_does():
    """The state's gradient would be left out of an update that goes through the other inputs."""
    import torch
    for call, given in _calls():
        for name in given:
            a = {k: v.clone().requires_grad_(k in (name, "state")) for k, v in given.items()}
            with pytest.raises(ValueError, match="state: no gradient goes through states"):
                call(**a)
            # what computed the state asks for it, not a leaf
            a["state"] = a["state"] * 2.0
            with pytest.raises(ValueError, match="state: no gradient goes through states"):
                call(**a)
            # without a gradient to record, and with a state that was detached, it is the device that does not fit
            with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
                call(**a)
            with pytest.raises(ValueError, match="CUDA"):
                call(**dict(a, state=a["state"].detach()))


@pytest.mark.parametrize("eps", [1e-45, 1e-39, 2.0 ** -127, 1.17e-38])
def test_an_eps_that_is_no_normal_number_is_refused(eps):
    """The root of a row of zeros would be taken of nothing, and be infinite: zero times it is not a number."""
    import ctypes
    import paper_2103_07013_amd as bps
    from paper_2103_07013_amd import memory
    lib, P = memory._library(), 4096
    a = memory._Norm(dtype=0, residual_dtype=0, weight_dtype=0, activation=0, rows=2, width=6, eps=eps, residual=P, block=P, residual_stride=6, block_stride=6, pre_weight=P, residual_out=P, out=P + 2,
                     residual_out_stride=6, out_stride=6, roots=P, grad_residual=P, grad_block=P, grad_residual_stride=6, grad_block_stride=6, grad_pre_weight=P)
    assert 0.0 < a.eps < 2.0 ** -126
    for call, rest in ((lib.bps_residual_norm, ()), (lib.bps_residual_norm_backward, (P, 1 << 30))):
        assert call(ctypes.byref(a), *rest, None) == -1 and "eps" in bps.bps_last_error()
    # the smallest that is taken: what is refused is an argument that is looked at later
    a.eps = 2.0 ** -126
    assert lib.bps_residual_norm(ctypes.byref(a), None) == -1 and "out is misaligned" in bps.bps_last_error()
