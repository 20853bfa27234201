"""Gradients that are sums over very many steps or rows: how exact float32 leaves them.

A sum of n terms that are added one after another is off by U / sqrt(3) of the partial sum at each addition at most on average, 0.42 U for mantissas spread as
they are, so of terms of random signs by 0.42 U sqrt(n / 2), 0.3 U sqrt(n) of the sum, and of positive terms by 0.42 U sqrt(n / 3), 0.24 U sqrt(n), as a 2-norm over many
such sums.  The kernels add up to 256 terms one after another and then what they have of those: 5 U, with 2 U for up to 32 such sums and 2 U for the join; the
terms' own errors are as random and under 4 U as a 2-norm.  7 U in all; tests allow 10."""
import pytest

pytestmark = pytest.mark.gpu

LIMIT = 10 * 2.0 ** -24


def _off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def test_sums_over_the_steps_of_a_scan():
    """512 groups of one channel leave eight work-groups to each, of which every one has eight sequences of 512 steps: 4096 terms of a sum."""
    import torch
    import paper_2103_07013_amd as bps
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    batch, T, width = 64, 512, 512
    x, delta, grad, b, c = n(batch, T, width), n(batch, T, width), n(batch, T, width), n(batch, T, width, 1), n(batch, T, width, 1)
    A, D, bias = -torch.rand((1, width), generator=g, device="cuda") - 0.1, n(width), n(width) * 0.2 - 2.0
    got = bps.selective_scan_backward(grad, x, delta, A, b, c, bps.selective_scan(x, delta, A, b, c, D=D, delta_bias=bias, hold=True), D=D, delta_bias=bias)
    leaves = [t.double().requires_grad_() for t in (A, D, bias)]
    x, delta, grad, b, c = (t.double() for t in (x, delta, grad, b[..., 0], c[..., 0]))
    d = torch.nn.functional.softplus(delta + leaves[2])
    a, added = (d * leaves[0]).exp(), d * x * b
    h, outs = torch.zeros_like(added[:, 0]), []
    for t in range(T):
        h = a[:, t] * h + added[:, t]
        outs.append(h)
    out = torch.stack(outs, 1) * c + leaves[1] * x
    want = torch.autograd.grad(out, leaves, grad)
    for name, p, q in zip(("A", "D", "delta_bias"), (got.A, got.D, got.delta_bias), want):
        assert _off(p, q) < LIMIT, (name, _off(p, q) * 2 ** 24)


def test_sums_over_the_rows_of_norms():
    """Rows of 16 lanes, 2048 of them for each of the 8192 that are worked on at a time."""
    import torch
    import paper_2103_07013_amd as bps
    g = torch.Generator(device="cuda").manual_seed(2)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    rows, width = 1 << 24, 32
    residual, block, grad = n(rows, width), n(rows, width), n(rows, width)
    scale, post = torch.rand(width, generator=g, device="cuda") + 0.5, torch.rand(width, generator=g, device="cuda") + 0.5
    r = bps.residual_norm(residual, block, post_weight=post, scale=scale)
    got = bps.residual_norm_backward(residual, block, r, grad_residual=grad, post_weight=post, scale=scale)
    want = torch.zeros(width, dtype=torch.float64, device="cuda")
    for k in range(0, rows, 1 << 22):
        b = block[k:k + (1 << 22)].double()
        want += (grad[k:k + (1 << 22)].double() * b * (b.square().mean(1, keepdim=True) + 1e-6).rsqrt()).sum(0)
    for name, p, factor in (("scale", got.scale, post), ("post_weight", got.post_weight, scale)):
        assert _off(p, want * factor.double()) < LIMIT, (name, _off(p, want * factor.double()) * 2 ** 24)
