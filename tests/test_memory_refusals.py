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
