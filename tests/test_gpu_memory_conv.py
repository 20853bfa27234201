"""The causal convolution against its definition in 64 bits: types, taps, lengths from none to many, episodes, states, strides, gradients."""
import pytest

pytestmark = pytest.mark.gpu


def _inputs(B, T, D, K, dtype, seed, starts=0.0, ragged=False, state=False, bias=True, wide=False):
    import torch
    from memory_reference import TYPES
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]
    n = lambda *s, d=t: torch.randn(s, generator=g, device="cuda").to(d)  # noqa: E731
    w = torch.float32 if wide else t
    return dict(x=n(B, T, D), weight=n(D, K, d=w), bias=n(D, d=w) if bias else None, starts=torch.rand((B, T), generator=g, device="cuda") < starts if starts else None,
                lengths=torch.randint(-1, T + 2, (B,), generator=g, device="cuda", dtype=torch.int32) if ragged else None, state=n(B, K - 1, D) if state else None), n(B, T, D)


def _check(a, grad, silu=True):
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import U, check, conv, cpu
    r = bps.causal_conv(**a, silu=silu)
    K = a["weight"].shape[1]
    h = {k: cpu(v) for k, v in a.items()}
    leaves = [h[k].requires_grad_() for k in ("x", "weight", "bias") if h[k] is not None]
    out, state, size = conv(h["x"], h["weight"], h["bias"], silu, h["starts"], h["lengths"], h["state"])
    # u: K products and sums.  silu's slope is under 1.1; a sigmoid is off by (2 |u| + 8) U at most, as in memory_reference
    u_off = (K + 1) * U * size
    bound = 1.1 * u_off + out.detach().abs() * (2 * size + 10) * U if silu else u_off
    check("out", r.out, out, bound)
    assert torch.equal(r.state.cpu().double(), state.detach())
    want = torch.autograd.grad(out, leaves, cpu(grad), allow_unused=True)
    want = [torch.zeros_like(leaf) if w is None else w for w, leaf in zip(want, leaves)]
    got = bps.causal_conv_backward(grad, **a, silu=silu)
    assert (got.bias is None) == (a["bias"] is None)
    # the slope s (1 + u (1 - s)) is at most 1.1 and changes by at most 0.5 for each of u; its parts are off as the sigmoid is
    slope_off = 0.5 * u_off + (2 * size + 12) * (1 + size) * U if silu else 0.0 * size
    g = cpu(grad).abs()
    du, du_off = 1.1 * g, g * (slope_off + 3 * U)
    B, T, D = a["x"].shape
    w, x = h["weight"].detach().abs(), h["x"].detach().abs().nan_to_num()
    before = h["state"].detach().abs() if h["state"] is not None else x.new_zeros(B, K - 1, D)
    whole = torch.cat([before, x], 1)
    dx, dw = torch.zeros_like(whole), []
    for k in range(K):
        dx[:, k:k + T] += (du_off + du * (K + 1) * U) * w[:, k]
        tap = whole[:, k:k + T]
        dw.append((tap * (du_off + du * (B * T + 2) * U)).sum((0, 1)))
    check("grad x", got.x, want[0], dx[:, K - 1:])
    check("grad weight", got.weight, want[1], torch.stack(dw, 1))
    if a["bias"] is not None:
        check("grad bias", got.bias, want[2], (du_off + du * (B * T + 2) * U).sum((0, 1)))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 6, 7, 8])
def test_taps_and_types(dtype, K):
    a, g = _inputs(3, 37, 21, K, dtype, 10 * K, starts=0.1, ragged=True, state=True)
    _check(a, g)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 64, 65, 130])
@pytest.mark.parametrize("dtype,D", [("f32", 1), ("f32", 66), ("bf16", 8), ("bf16", 67), ("f16", 129)])
def test_lengths_and_widths(dtype, D, T):
    a, g = _inputs(2, T, D, 4, dtype, T + D, starts=0.05, state=True)
    _check(a, g)


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("bias,wide,state", [(False, False, False), (True, True, True), (False, True, False), (True, False, True)])
def test_what_may_be_left_out(bias, wide, state, silu):
    a, g = _inputs(2, 19, 33, 3, "bf16", 5, starts=0.2, state=state, bias=bias, wide=wide)
    _check(a, g, silu)


def test_every_step_begins_an_episode():
    a, g = _inputs(2, 11, 9, 4, "f32", 6, starts=1.0, state=True)
    assert a["starts"].all()
    _check(a, g)


def test_sequences_that_are_empty():
    """Their state stays, or is zero; all of their outputs and gradients are zero."""
    import torch
    a, g = _inputs(3, 5, 12, 4, "f16", 7, state=True)
    a["lengths"] = torch.zeros(3, dtype=torch.int32, device="cuda")
    _check(a, g)
    a["lengths"][1] = 2
    _check(a, g)


def test_no_steps_and_no_sequences():
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(3, 0, 12, 4, "f32", 8, state=True)
    r = bps.causal_conv(**a)
    assert r.out.shape == (3, 0, 12) and torch.equal(r.state, a["state"])
    d = bps.causal_conv_backward(g, **a)
    assert d.x.shape == (3, 0, 12) and (d.weight == 0).all() and (d.bias == 0).all()
    a, g = _inputs(0, 6, 12, 4, "f32", 8, state=True)
    assert bps.causal_conv(**a).out.shape == (0, 6, 12)
    d = bps.causal_conv_backward(g, **a)
    assert (d.weight == 0).all() and (d.bias == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_lies_behind_the_end_or_before_an_episode_does_not_matter(bad):
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(2, 40, 24, 4, "bf16", 9, state=True)
    a["lengths"] = torch.tensor([17, 33], dtype=torch.int32, device="cuda")
    a["starts"] = torch.zeros((2, 40), dtype=torch.bool, device="cuda")
    a["starts"][:, 5] = True
    a["starts"][0, 20] = True
    want, grads = bps.causal_conv(**a), bps.causal_conv_backward(g, **a)
    b = dict(a, x=a["x"].clone())
    other = g.clone()
    for k, end in enumerate((17, 33)):
        b["x"][k, end:] = bad
        other[k, end:] = bad
    b["x"][:, 4] = bad
    got, new = bps.causal_conv(**b), bps.causal_conv_backward(other, **b)
    keep = [t for t in range(40) if t != 4]
    assert torch.equal(got.out[:, keep], want.out[:, keep]) and torch.equal(got.state, want.state)
    assert torch.equal(new.x[:, [t for t in keep if t > 4]], grads.x[:, [t for t in keep if t > 4]])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    """Time first, parts of wider rows, one row for all: the same bits as contiguous tensors give."""
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(5, 23, 17, 4, dtype, 11, starts=0.1, ragged=True, state=True)
    want, grads = bps.causal_conv(**a), bps.causal_conv_backward(g, **a)
    wide = torch.zeros(23, 5, 60, dtype=a["x"].dtype, device="cuda").transpose(0, 1)
    wide[:, :, 3:20] = a["x"]
    wide[:, :, 31:48] = g
    states = torch.zeros(5, 4, 17, dtype=a["x"].dtype, device="cuda")
    states[:, :3] = a["state"]
    b = dict(a, x=wide[:, :, 3:20], starts=a["starts"].T.contiguous().T, state=states[:, :3])
    got, new = bps.causal_conv(**b), bps.causal_conv_backward(wide[:, :, 31:48], **b)
    assert torch.equal(got.out, want.out) and torch.equal(got.state, want.state)
    assert all(torch.equal(p, q) for p, q in zip(new, grads))
    one = dict(a, x=a["x"][:1, :1].expand(5, 23, 17))
    _check(one, g)


def test_pieces_of_a_sequence_give_the_whole():
    """Any cut, with the state handed on; and step by step."""
    import torch
    import paper_2103_07013_amd as bps
    a, _ = _inputs(3, 26, 20, 5, "f32", 12, starts=0.1, state=True)
    want = bps.causal_conv(**a)
    for cuts in ([0, 1, 3, 26], [0, 13, 26], [0, 8, 16, 24, 25, 26]):
        state, outs = a["state"], []
        for p, q in zip(cuts, cuts[1:]):
            r = bps.causal_conv(a["x"][:, p:q], a["weight"], a["bias"], starts=a["starts"][:, p:q], state=state)
            outs.append(r.out)
            state = r.state
        assert torch.equal(torch.cat(outs, 1), want.out) and torch.equal(state, want.state)
    state = a["state"].clone()
    for t in range(26):
        assert torch.equal(bps.causal_conv_step(a["x"][:, t], state, a["weight"], a["bias"], starts=a["starts"][:, t]), want.out[:, t])
    assert torch.equal(state, want.state)


@pytest.mark.parametrize("dtype,D", [("f32", 3), ("f32", 67), ("bf16", 5), ("bf16", 67), ("f16", 15)])
def test_channels_stay_apart(dtype, D):
    """Where the last channels do not fill a vector: what one channel holds shows in no other, and steps move the same states on."""
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(2, 19, D, 4, dtype, D, starts=0.05, state=True)
    want, grads = bps.causal_conv(**a), bps.causal_conv_backward(g, **a)
    for k in sorted({0, max(D - 8, 0), max(D - 4, 0), D - 2, D - 1}):
        others = [c for c in range(D) if c != k]
        b = dict(a, x=a["x"].clone(), state=a["state"].clone(), weight=a["weight"].clone())
        b["x"][..., k] = float("nan")
        b["state"][..., k] = float("inf")
        b["weight"][k] = float("inf")
        got, new = bps.causal_conv(**b), bps.causal_conv_backward(g, **b)
        assert torch.equal(got.out[..., others], want.out[..., others]) and torch.equal(got.state[..., others], want.state[..., others])
        assert torch.equal(new.x[..., others], grads.x[..., others]) and torch.equal(new.weight[others], grads.weight[others]) and torch.equal(new.bias[others], grads.bias[others])
    state = a["state"].clone()
    for t in range(19):
        assert torch.equal(bps.causal_conv_step(a["x"][:, t], state, a["weight"], a["bias"], starts=a["starts"][:, t]), want.out[:, t])
    assert torch.equal(state, want.state)


def test_autograd():
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(3, 30, 18, 4, "f32", 13, starts=0.1, ragged=True, state=True)
    want = bps.causal_conv_backward(g, **a)
    leaves = [a[k].requires_grad_() for k in ("x", "weight", "bias")]
    r = bps.causal_conv(**a)
    assert not r.state.requires_grad
    got = torch.autograd.grad(r.out, leaves, g)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    # a gradient whose rows are one, as a sum's is
    got = torch.autograd.grad(bps.causal_conv(**a).out.sum(), leaves)
    want = bps.causal_conv_backward(torch.ones_like(g), **{k: v.detach() if v is not None else None for k, v in a.items()})
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_the_gradient_against_differences():
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(2, 12, 6, 4, "f32", 14, starts=0.1, state=True)
    grads = bps.causal_conv_backward(g, **a)
    torch.manual_seed(3)
    for name in ("x", "weight", "bias"):
        way, step = torch.randn_like(a[name]), 2.0 ** -6
        p, q = (bps.causal_conv(**dict(a, **{name: a[name] + s * way})).out.double() for s in (step, -step))
        want = ((p - q) * g.double()).sum() / (2 * step)
        size = ((p - q) * g.double()).abs().sum() / (2 * step) + (p.abs() * g.double().abs()).sum()
        # differences are off by the third derivative times step^2 / 6, under 2^-12 of the sizes here with up to 4 changed inputs, and by
        # rounding over the step, 2^-24 * 20 * 2^6
        assert abs((getattr(grads, name).double() * way.double()).sum() - want) < (2.0 ** -7 + 2.0 ** -13) * size


def test_the_same_bits_every_time():
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(40, 70, 100, 4, "bf16", 15, starts=0.05)
    first = bps.causal_conv_backward(g, **a)
    for _ in range(5):
        assert all(torch.equal(p, q) for p, q in zip(first, bps.causal_conv_backward(g, **a)))
