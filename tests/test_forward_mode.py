"""Forward-mode derivatives: the policy's and the memory's operators compute none, and refuse tensors that carry a tangent instead of losing it.  It is refused
before devices are looked at, so that it is tried on the CPU's tensors, which are refused for their device otherwise."""
import pytest


def _calls():
    """(call, its tensors that could carry a tangent, what else it is given, what it says of tensors of the CPU)"""
    import torch
    import paper_2103_07013_amd as bps
    z = lambda *s: torch.zeros(s)  # noqa: E731
    tokens = torch.zeros(2, dtype=torch.int64)
    scan = dict(x=z(2, 5, 8), delta=z(2, 5, 8), A=z(4, 8), B=z(2, 5, 4), C=z(2, 5, 4), D=z(8), gate=z(2, 5, 8), delta_bias=z(8))
    step = {k: v[:, 0].clone() if v.dim() == 3 else v for k, v in scan.items()}
    norm = dict(residual=z(2, 8), block=z(2, 8), post_weight=z(8), gate=z(2, 8), scale=z(8), pre_weight=z(8))
    conv = dict(x=z(2, 5, 8), weight=z(8, 4), bias=z(8))
    return [(bps.log_probs, dict(logits=z(2, 6)), dict(tokens=tokens)),
            (bps.log_probs_backward, dict(logits=z(2, 6), grad_logp=z(2), grad_entropy=z(2)), dict(tokens=tokens, result=z(5, 2))),
            (bps.embedding, dict(weight=z(4, 8)), dict(tokens=tokens)),
            (bps.embedding_backward, dict(grad_out=z(2, 8)), dict(tokens=tokens, rows=4)),
            (bps.causal_conv, conv | dict(state=z(2, 3, 8)), {}),
            (bps.causal_conv_backward, conv | dict(grad_out=z(2, 5, 8), state=z(2, 3, 8)), {}),
            (bps.causal_conv_step, dict(conv, x=z(2, 8), state=z(2, 3, 8)), {}),
            (bps.selective_scan, scan | dict(state=z(2, 4, 8)), {}),
            (bps.selective_scan_backward, scan | dict(grad_out=z(2, 5, 8)), dict(result=z(2, 1, 4, 8))),
            (bps.selective_scan_step, step | dict(state=z(2, 4, 8)), {}),
            (bps.residual_norm, norm, {}),
            (bps.residual_norm_backward, norm | dict(grad_residual=z(2, 8), grad_out=z(2, 8)), dict(result=z(2, 2)))]


@pytest.mark.parametrize("k", range(12))
def test_tensors_that_carry_a_tangent_are_refused(k):
    import torch
    from torch.autograd import forward_ad
    call, tensors, rest = _calls()[k]
    with forward_ad.dual_level():
        for recorded in (True, False):
            with torch.set_grad_enabled(recorded):
                for name, t in tensors.items():
                    dual = forward_ad.make_dual(t, torch.ones_like(t))
                    with pytest.raises(ValueError, match="forward-mode"):
                        call(**dict(tensors, **{name: dual}), **rest)
                # none of them: what is refused is the device
                with pytest.raises(ValueError) as said:
                    call(**tensors, **rest)
                assert "forward-mode" not in str(said.value)

