"""Training through the memory's operators as autograd does it, where its tensors are not the ones that a call would be given by hand."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_gradient_that_arrives_time_first_and_far_apart():
    """Outputs that are used time first send their gradient back in that order: 2^26 elements from step to step here, more than a call takes
    of its own tensors."""
    import torch
    import paper_2103_07013_amd as bps
    g = torch.Generator(device="cuda").manual_seed(1)
    batch, T, width = 1 << 15, 2, 1 << 11
    n = lambda *s, d=torch.bfloat16: torch.randn(s, generator=g, device="cuda").to(d)  # noqa: E731
    x, delta, b, c = n(batch, T, width), n(batch, T, width), n(batch, T, 1), n(batch, T, 1)
    A = -torch.rand((1, width), generator=g, device="cuda")
    grad = n(T, batch, width)
    want = bps.selective_scan_backward(grad.transpose(0, 1).contiguous(), x, delta, A, b, c, bps.selective_scan(x, delta, A, b, c, hold=True))
    leaves = [t.requires_grad_() for t in (x, delta, A, b, c)]
    out = bps.selective_scan(*leaves).out
    got = torch.autograd.grad(out.transpose(0, 1), leaves, grad)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
