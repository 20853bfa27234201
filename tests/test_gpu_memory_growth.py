"""Scans whose states grow, over chunks of time that are gone through side by side: what no float32 holds is the growth over a chunk, not
what the definition makes of it."""
import pytest

pytestmark = pytest.mark.gpu

T = 256           # four chunks of 64 steps
RATE = 1.5        # e^(1.5 * 64) is over 2^138


def _inputs(width=64, N=4, seed=1):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    # sizes and rates whose product is the same for all, with either sign of the size
    size = torch.where(torch.arange(width, device="cuda") % 2 == 0, 0.5, -0.5).expand(2, T, width).contiguous()
    return dict(x=n(2, T, width), delta=size, A=torch.where(size[0, :N] > 0, RATE / 0.5, -RATE / 0.5).contiguous(), B=n(2, T, N), C=n(2, T, N), D=n(width), gate=n(2, T, width), softplus=False), n(2, T, width)


def _definition(a, grad=None):
    import torch
    from memory_reference import cpu, scan, scan_bounds
    h = {k: cpu(v) for k, v in a.items()}
    h = dict(dict(delta_bias=None, starts=None, lengths=None, state=None), **h)
    h["soft"] = h.pop("softplus")
    bounds = scan_bounds(**h, grad_out=None if grad is None else cpu(grad))
    names = ("x", "delta", "A", "B", "C", "D", "gate")
    leaves = {k: h[k].requires_grad_() for k in names}
    out, state = scan(**h)
    return out, state, bounds, None if grad is None else dict(zip(names, torch.autograd.grad(out, list(leaves.values()), cpu(grad))))


def test_states_of_zero_stay_zero_while_they_would_grow():
    """Padding in front: inputs of zero over the first chunks."""
    import paper_2103_07013_amd as bps
    from memory_reference import check
    a, _ = _inputs()
    a["x"][:, :220] = 0.0
    r = bps.selective_scan(**a, hold=True)
    out, state, bounds, _ = _definition(a)
    assert r.out.isfinite().all() and (r.out[:, :220] == 0).all() and (r.held[:, :13] == 0).all()
    check("out", r.out, out, bounds["out"])
    check("state", r.state, state, bounds["state"])


def test_gradients_of_zero_stay_zero_while_they_would_grow():
    """The way back meets outputs that no gradient comes from first, over whole chunks."""
    import paper_2103_07013_amd as bps
    from memory_reference import check
    a, grad = _inputs(seed=2)
    a["x"][:, :220] = 0.0
    grad[:, 30:] = 0.0
    r = bps.selective_scan(**a, hold=True)
    out, _, bounds, want = _definition(a, grad)
    got = bps.selective_scan_backward(grad, result=r, **a)
    for k, w in want.items():
        check("grad " + k, getattr(got, k), w, bounds[k].reshape(w.shape))
    assert want["x"][:, :30].abs().amax() > 1e6


def test_a_small_state_that_a_chunk_makes_a_large_one():
    """The growth over the first chunk is over 2^128, the state behind it is not."""
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import check
    a, _ = _inputs(seed=3)
    a["x"].zero_()
    a["delta"][:, 64:] *= 2.0 ** -10
    a["state"] = torch.full((2, 4, 64), 1e-30, device="cuda")
    r = bps.selective_scan(**a, hold=True)
    out, state, bounds, _ = _definition(a)
    assert state.min() > 1e11
    check("out", r.out, out, bounds["out"])
    check("state", r.state, state, bounds["state"])
