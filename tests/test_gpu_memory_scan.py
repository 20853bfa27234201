"""The selective scan against its definition in 64 bits: types, states, groups, lengths, episodes, chunks of time, strides, gradients."""
import pytest

pytestmark = pytest.mark.gpu

NAMES = ("x", "delta", "A", "B", "C", "D", "gate", "delta_bias")


def _inputs(batch, T, width, N, dtype, seed, groups=1, starts=0.0, ragged=False, state=False, without=(), softplus=True):
    import torch
    from memory_reference import TYPES
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]
    n = lambda *s, d=t: torch.randn(s, generator=g, device="cuda").to(d)  # noqa: E731
    a = dict(x=n(batch, T, width), delta=n(batch, T, width), gate=n(batch, T, width), B=n(batch, T, groups, N), C=n(batch, T, groups, N),
             A=-torch.rand((N, width), generator=g, device="cuda") * 4 - 0.1, D=n(width, d=torch.float32), delta_bias=n(width, d=torch.float32) - 2.0,
             starts=torch.rand((batch, T), generator=g, device="cuda") < starts if starts else None,
             lengths=torch.randint(-1, T + 2, (batch,), generator=g, device="cuda", dtype=torch.int32) if ragged else None,
             state=n(batch, N, width, d=torch.float32) if state else None, softplus=softplus)
    if groups == 1:
        a["B"], a["C"] = a["B"][:, :, 0], a["C"][:, :, 0]
    if not softplus:
        a["delta"], a["delta_bias"] = (torch.rand((batch, T, width), generator=g, device="cuda") * 0.5 - 0.05).to(t), a["delta_bias"] * 0 + 0.125
    for k in without:
        a[k] = None
    return a, n(batch, T, width)


def _backward(grad, a, r):
    import paper_2103_07013_amd as bps
    return bps.selective_scan_backward(grad, result=r, **{k: v for k, v in a.items() if k != "state"})


def _check(a, grad):
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import check, cpu, scan, scan_bounds
    r = bps.selective_scan(**a, hold=True)
    h = {k: cpu(v) for k, v in a.items()}
    h["soft"] = h.pop("softplus")
    bounds = scan_bounds(**h, grad_out=cpu(grad))
    leaves = {k: h[k].requires_grad_() for k in NAMES if h[k] is not None}
    out, state = scan(**h)
    check("out", r.out, out, bounds["out"])
    check("state", r.state, state, bounds["state"])
    got = _backward(grad, a, r)
    want = dict(zip(leaves, torch.autograd.grad(out, list(leaves.values()), cpu(grad))))
    for k in NAMES:
        if k in want:
            check("grad " + k, getattr(got, k), want[k], bounds[k].reshape(want[k].shape))
        else:
            assert getattr(got, k) is None
    return r, got


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N", [1, 3, 4, 7, 8, 13, 16, 17, 32])
def test_states_and_types(dtype, N):
    a, g = _inputs(3, 21, 37, N, dtype, N, starts=0.1, ragged=True, state=True)
    _check(a, g)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 33])
@pytest.mark.parametrize("width", [1, 63, 64, 65, 130])
def test_lengths_and_widths(T, width):
    a, g = _inputs(2, T, width, 5, "f32", T + width, starts=0.05, state=True)
    _check(a, g)


@pytest.mark.parametrize("groups,width", [(2, 2), (2, 130), (3, 195), (4, 64)])
def test_groups(groups, width):
    a, g = _inputs(2, 18, width, 16, "bf16", groups, groups=groups, starts=0.1, ragged=True, state=True)
    _check(a, g)


@pytest.mark.parametrize("dtype,N", [("f32", 16), ("bf16", 16), ("f16", 14), ("bf16", 32), ("f32", 19), ("bf16", 8), ("f16", 4)])
@pytest.mark.parametrize("width", [64, 200, 256])
@pytest.mark.parametrize("T", [3, 6, 11, 21, 130])
def test_channels_that_fill_work_groups(width, T, dtype, N):
    """As many channels as the wavefronts of most work-groups take, with few steps, a few tiles of them, and chunks."""
    a, g = _inputs(2, T, width, N, dtype, T + width, starts=0.05, ragged=T > 20, state=True)
    _check(a, g)


@pytest.mark.parametrize("without", [(), ("D",), ("gate",), ("delta_bias",), ("D", "gate", "delta_bias")])
@pytest.mark.parametrize("softplus", [True, False])
def test_what_may_be_left_out(without, softplus):
    a, g = _inputs(2, 19, 33, 6, "f32", 5, starts=0.1, without=without, softplus=softplus)
    _check(a, g)


@pytest.mark.parametrize("dtype,N,groups", [("f32", 16, 1), ("bf16", 5, 2), ("f16", 32, 1)])
@pytest.mark.parametrize("T", [64, 65, 200, 333])
@pytest.mark.parametrize("kind", ["whole", "ragged", "episodes"])
def test_time_in_chunks(dtype, N, groups, T, kind):
    """Few sequences of few channels: their time is cut into chunks of 32 steps or more."""
    a, g = _inputs(2, T, 66, N, dtype, T + N, groups=groups, starts=0.02 if kind == "episodes" else 0.0, ragged=kind == "ragged", state=True)
    _check(a, g)


def test_long_decays_over_many_chunks():
    """Steps and rates so small that the first inputs still count at the end."""
    a, g = _inputs(1, 1000, 64, 4, "f32", 8, state=True)
    a["A"] = a["A"] * 0.01
    _check(a, g)


def test_decays_that_leave_nothing():
    """Products of decays that no float32 holds, and steps whose size is none."""
    a, g = _inputs(1, 200, 64, 4, "f32", 9, state=True)
    a["A"] = a["A"] * 1e4
    a["delta"][:, 100:] -= 150.0
    r, got = _check(a, g)
    assert all(t.isfinite().all() for t in (r.out, r.state, *got))


def test_every_step_begins_an_episode():
    a, g = _inputs(2, 75, 9, 4, "f32", 6, starts=1.0, state=True)
    assert a["starts"].all()
    _check(a, g)


@pytest.mark.parametrize("T", [5, 100])
def test_sequences_that_are_empty(T):
    import torch
    a, g = _inputs(3, T, 12, 4, "f16", 7, state=True)
    a["lengths"] = torch.zeros(3, dtype=torch.int32, device="cuda")
    r, _ = _check(a, g)
    assert torch.equal(r.state, a["state"])
    a["lengths"][1] = T - 2
    _check(a, g)


def test_no_steps_and_no_sequences():
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(3, 0, 12, 4, "f32", 8, state=True)
    r = bps.selective_scan(**a, hold=True)
    assert r.out.shape == (3, 0, 12) and torch.equal(r.state, a["state"])
    d = _backward(g, a, r)
    assert d.x.shape == (3, 0, 12) and all((t == 0).all() for t in (d.A, d.D, d.delta_bias))
    a, g = _inputs(0, 6, 12, 4, "f32", 8, state=True)
    r = bps.selective_scan(**a, hold=True)
    d = _backward(g, a, r)
    assert r.out.shape == (0, 6, 12) and all((t == 0).all() for t in (d.A, d.D, d.delta_bias))


@pytest.mark.parametrize("T", [40, 200])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_lies_behind_the_end_or_before_an_episode_does_not_matter(bad, T):
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(2, T, 24, 4, "bf16", 9, state=True)
    ends = (T // 2 - 3, T - 7)
    a["lengths"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    a["starts"] = torch.zeros((2, T), dtype=torch.bool, device="cuda")
    a["starts"][:, 5] = True
    a["starts"][0, T // 2] = True
    want = bps.selective_scan(**a, hold=True)
    grads = _backward(g, a, want)
    b, other = dict(a, **{k: a[k].clone() for k in ("x", "delta", "gate", "B", "C")}), g.clone()
    for k, end in enumerate(ends):
        for n in ("x", "delta", "gate", "B", "C"):
            b[n][k, end:] = bad
        other[k, end:] = bad
    got = bps.selective_scan(**b, hold=True)
    new = _backward(other, b, got)
    assert torch.equal(got.out, want.out) and torch.equal(got.state, want.state) and all(torch.equal(p, q) for p, q in zip(new, grads))
    # the state of an episode that is over
    b = dict(a, state=torch.full_like(a["state"], bad))
    got = bps.selective_scan(**b, hold=True)
    assert torch.equal(got.out[:, 5:], want.out[:, 5:]) and torch.equal(got.state, want.state)
    new = _backward(g, b, got)
    assert torch.equal(new.x, grads.x) and torch.equal(new.delta[:, 5:], grads.delta[:, 5:])


@pytest.mark.parametrize("T", [23, 150])
def test_strides(T):
    """Time first, parts of wider rows: the same bits as contiguous tensors give."""
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(5, T, 17, 6, "bf16", 11, starts=0.1, ragged=True, state=True)
    want = bps.selective_scan(**a, hold=True)
    grads = _backward(g, a, want)
    wide = torch.zeros(T, 5, 5 * 17 + 13, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    b, at = dict(a), 1
    for k in ("x", "delta", "gate", "B", "C"):
        n = a[k].shape[-1]
        wide[:, :, at:at + n] = a[k]
        b[k] = wide[:, :, at:at + n]
        at += n
    wide[:, :, at:at + 17] = g
    states = torch.zeros(5, 7, 17, device="cuda")
    states[:, :6] = a["state"]
    b |= dict(starts=a["starts"].T.contiguous().T, state=states[:, :6])
    got = bps.selective_scan(**b, hold=True)
    new = _backward(wide[:, :, at:at + 17], b, got)
    assert torch.equal(got.out, want.out) and torch.equal(got.state, want.state) and all(torch.equal(p, q) for p, q in zip(new, grads))


def test_pieces_of_a_sequence_give_the_whole():
    """Any cut, with the state handed on; and step by step."""
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import check, cpu, scan, scan_bounds
    a, _ = _inputs(3, 26, 20, 5, "f32", 12, starts=0.1, state=True)
    h = {k: cpu(v) for k, v in a.items()}
    h["soft"] = h.pop("softplus")
    out, state = scan(**h)
    bounds = scan_bounds(**h)
    per_step = ("x", "delta", "B", "C", "gate", "starts")
    for cuts in ([0, 1, 3, 26], [0, 13, 26], list(range(27))):
        at, outs = a["state"], []
        for p, q in zip(cuts, cuts[1:]):
            r = bps.selective_scan(**dict(a, **{k: a[k][:, p:q] for k in per_step}, state=at))
            outs.append(r.out)
            at = r.state
        check("out", torch.cat(outs, 1), out, bounds["out"])
        check("state", at, state, bounds["state"])
    at, outs = a["state"].clone(), []
    for t in range(26):
        outs.append(bps.selective_scan_step(state=at, **dict({k: v for k, v in a.items() if k not in ("state", "lengths")}, **{k: a[k][:, t] for k in per_step})))
    check("out", torch.stack(outs, 1), out, bounds["out"])
    check("state", at, state, bounds["state"])


@pytest.mark.parametrize("dtype,N,groups", [("f32", 16, 1), ("bf16", 16, 2), ("f16", 3, 1), ("f32", 32, 1), ("bf16", 8, 1)])
@pytest.mark.parametrize("batch,width", [(1, 2), (5, 130), (300, 64)])
def test_single_steps(dtype, N, groups, batch, width):
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import check, cpu, scan, scan_bounds
    a, _ = _inputs(batch, 1, width, N, dtype, 3, groups=groups, starts=0.3, state=True)
    h = {k: cpu(v) for k, v in a.items()}
    h["soft"] = h.pop("softplus")
    out, want = scan(**h)
    bounds = scan_bounds(**h)
    pool = torch.zeros(batch, N + 2, width, device="cuda")
    pool[:, 1:-1] = a["state"]
    state = pool[:, 1:-1]
    got = bps.selective_scan_step(state=state, **dict({k: v for k, v in a.items() if k not in ("state", "lengths")}, **{k: a[k][:, 0] for k in ("x", "delta", "B", "C", "gate", "starts")}))
    check("out", got, out[:, 0], bounds["out"][:, 0])
    check("state", state, want, bounds["state"])
    assert (pool[:, 0] == 0).all() and (pool[:, -1] == 0).all()


def test_autograd():
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(3, 70, 18, 5, "f32", 13, groups=2, starts=0.05, ragged=True, state=True)
    r = bps.selective_scan(**a, hold=True)
    want = _backward(g, a, r)
    leaves = [a[k].requires_grad_() for k in NAMES]
    s = bps.selective_scan(**a)
    assert torch.equal(s.out, r.out) and not s.state.requires_grad and not s.held.requires_grad
    got = torch.autograd.grad(s.out, leaves, g)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    # a part of the inputs only, and a gradient that is one row for all
    got, = torch.autograd.grad(bps.selective_scan(**{k: v.detach() if k not in ("A",) and torch.is_tensor(v) else v for k, v in a.items()}).out.sum(), [a["A"]])
    ones = _backward(torch.ones_like(g), {k: v.detach() if torch.is_tensor(v) else v for k, v in a.items()}, r)
    assert torch.equal(got, ones.A)


def test_the_gradient_against_differences():
    import torch
    import paper_2103_07013_amd as bps
    a, g = _inputs(2, 12, 6, 4, "f32", 14, starts=0.1, state=True)
    grads = _backward(g, a, bps.selective_scan(**a, hold=True))
    torch.manual_seed(3)
    for name in NAMES:
        way, step = torch.randn_like(a[name]), 2.0 ** -7
        p, q = (bps.selective_scan(**dict(a, **{name: a[name] + s * way})).out.double() for s in (step, -step))
        want = ((p - q) * g.double()).sum() / (2 * step)
        size = ((p - q) * g.double()).abs().sum() / (2 * step) + (p.abs() * g.double().abs()).sum()
        # the third derivative times step^2 / 6: inputs move by up to 4 steps, and a product of twelve steps' decays by its cube; rounding
        # over the step 2^-24 * 30 * 2^7
        assert abs((getattr(grads, name).double() * way.double()).sum() - want) < 2.0 ** -8 * size, name


def test_the_same_bits_every_time():
    import torch
    import paper_2103_07013_amd as bps
    for batch, T in ((40, 20), (1, 500)):
        a, g = _inputs(batch, T, 150, 16, "bf16", 15, starts=0.05)
        r = bps.selective_scan(**a, hold=True)
        first = _backward(g, a, r)
        for _ in range(5):
            s = bps.selective_scan(**a, hold=True)
            assert torch.equal(r.out, s.out) and torch.equal(r.state, s.state) and all(torch.equal(p, q) for p, q in zip(first, _backward(g, a, s)))
