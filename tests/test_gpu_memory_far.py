"""The memory's operators on tensors whose parts lie further apart than 32 bits say: the same bits as close together."""
import pytest

pytestmark = pytest.mark.gpu


def _far(t, buffer, at):
    """t's elements in `buffer`, its first dimension 2^32 + 8 elements apart, from element `at` on."""
    import torch
    v = torch.as_strided(buffer, t.shape, (2 ** 32 + 8, *t.stride()[1:]), at)
    v.copy_(t)
    return v


def test_batches_far_apart():
    import torch
    import paper_2103_07013_amd as bps
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s, d=torch.bfloat16: torch.randn(s, generator=g, device="cuda").to(d)  # noqa: E731
    buffer = torch.empty(2 ** 32 + 2 ** 20, dtype=torch.bfloat16, device="cuda")
    x, delta, z, b, c, grad = n(2, 90, 40), n(2, 90, 40), n(2, 90, 40), n(2, 90, 5), n(2, 90, 5), n(2, 90, 40)
    far, at = [], 3
    for t in (x, delta, z, b, c, grad):
        far.append(_far(t, buffer, at))
        at += t[0].numel() + 7
    w, A, state = n(40, 4), -torch.rand((5, 40), generator=g, device="cuda"), n(2, 3, 40)
    want, got = bps.causal_conv(x, w, state=state), bps.causal_conv(far[0], w, state=_far(state, buffer, at))
    assert torch.equal(got.out, want.out) and torch.equal(got.state, want.state)
    for p, q in zip(bps.causal_conv_backward(far[5], far[0], w), bps.causal_conv_backward(grad, x, w)):
        assert p is q is None or torch.equal(p, q)
    want, got = (bps.selective_scan(v[0], v[1], A, v[3], v[4], gate=v[2], hold=True) for v in ((x, delta, z, b, c), far))
    assert torch.equal(got.out, want.out) and torch.equal(got.state, want.state)
    grads = [bps.selective_scan_backward(v[5], v[0], v[1], A, v[3], v[4], r, gate=v[2]) for v, r in (((x, delta, z, b, c, grad), want), (far, got))]
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(*grads))


def test_rows_and_states_far_apart():
    import torch
    import paper_2103_07013_amd as bps
    g = torch.Generator(device="cuda").manual_seed(2)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    buffer = torch.empty(2 ** 32 + 2 ** 16, dtype=torch.float32, device="cuda")
    r, b, z, grad, w = n(2, 70), n(2, 70), n(2, 70), n(2, 70), n(70)
    far, at = [], 1
    for t in (r, b, z, grad):
        far.append(_far(t, buffer, at))
        at += 77
    want, got = (bps.residual_norm(v[0], v[1], gate=v[2], post_weight=w, pre_weight=w) for v in ((r, b, z), far))
    assert torch.equal(got.residual, want.residual) and torch.equal(got.out, want.out)
    grads = [bps.residual_norm_backward(v[0], v[1], want, v[3], v[3], gate=v[2], post_weight=w, pre_weight=w) for v in ((r, b, z, grad), far)]
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(*grads))
    state, A = n(2, 5, 70), -n(5, 70).abs()
    moved = _far(state, buffer, at)
    v = n(2, 5)
    assert torch.equal(bps.selective_scan_step(b, r, state, A, v, v), bps.selective_scan_step(b, r, moved, A, v, v)) and torch.equal(state, moved)


def test_many_steps_far_apart():
    """Time first, 2^22 elements from step to step: the last steps lie behind 2^32 bytes."""
    import torch
    import paper_2103_07013_amd as bps
    g = torch.Generator(device="cuda").manual_seed(3)
    steps = 1100
    buffer = torch.empty(steps * 2 ** 22, dtype=torch.bfloat16, device="cuda")
    x = torch.randn((1, steps, 33), generator=g, device="cuda").to(torch.bfloat16)
    b = torch.randn((1, steps, 4), generator=g, device="cuda").to(torch.bfloat16)
    far, wide = (torch.as_strided(buffer, t.shape, (8, 2 ** 22, 1), at) for t, at in ((x, 5), (b, 100)))
    far.copy_(x)
    wide.copy_(b)
    A, w = -torch.rand((4, 33), generator=g, device="cuda"), torch.randn((33, 3), generator=g, device="cuda")
    assert torch.equal(bps.causal_conv(far, w).out, bps.causal_conv(x, w).out)
    want, got = bps.selective_scan(x, x, A, b, b, hold=True), bps.selective_scan(far, far, A, wide, wide, hold=True)
    assert torch.equal(got.out, want.out) and torch.equal(got.state, want.state)
    for p, q in zip(bps.selective_scan_backward(far, far, far, A, wide, wide, got), bps.selective_scan_backward(x, x, x, A, b, b, want)):
        assert p is q is None or torch.equal(p, q)
    for p, q in zip(bps.causal_conv_backward(far, far, w), bps.causal_conv_backward(x, x, w)):
        assert p is q is None or torch.equal(p, q)
