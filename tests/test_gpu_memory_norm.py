"""The norms around a block against their definition in 64 bits: types, widths, what may be left out, strides, gradients."""
import pytest

pytestmark = pytest.mark.gpu

NAMES = ("residual", "block", "post_weight", "gate", "scale", "pre_weight")


def _inputs(rows, width, dtype, seed, stream=None, weights=None, without=()):
    import torch
    from memory_reference import TYPES
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]
    n = lambda *s, d=t: torch.randn(s, generator=g, device="cuda").to(d)  # noqa: E731
    w, stream = TYPES[weights or dtype], TYPES[stream or dtype]
    a = dict(residual=n(*rows, width, d=stream), block=n(*rows, width), post_weight=n(width, d=w), gate=n(*rows, width), scale=n(width, d=w), pre_weight=n(width, d=w))
    for k in without:
        a[k] = None
    return a, n(*rows, width, d=stream), n(*rows, width)


def _bounds(h, gr, go, eps, activation, r):
    """Bounds of the errors of sum, out and gradients (memory_reference says how they are counted).

    A root: W products and sums, a product, a sum, 3 U of the root itself, half of it through the root: (W / 2 + 4) U relative.  Hat, the sum over
    its root, is off by what the sum is and by that."""
    import torch
    from memory_reference import U
    W = r.shape[-1]
    root = (W / 2 + 4) * U
    one = torch.ones_like(h["block"])
    b = h["block"].abs()
    first = (h["block"].square().mean(-1, keepdim=True) + eps).rsqrt() if h["post_weight"] is not None else torch.ones_like(b[..., :1])
    hat1, hat1_rel = b * first, root + U if h["post_weight"] is not None else 0.0
    post = h["post_weight"].abs() if h["post_weight"] is not None else one
    if h["gate"] is not None:
        z, s = h["gate"], torch.sigmoid(h["gate"])
        rel_s = (2 * z.abs() + 8) * U
        f, f_rel = (z.abs() * s, rel_s + U) if activation == "silu" else (s, rel_s)
        if activation == "silu":
            steep, steep_off = s * (1 + z.abs() * (1 - s)), s * (1 + z.abs()) * (2 * rel_s + 4 * U)
        else:
            steep, steep_off = s * (1 - s), s * (2 * rel_s + 3 * U)
    else:
        f, f_rel = one, 0.0
    scale = h["scale"].abs() if h["scale"] is not None else one
    n, n_rel = hat1 * post, hat1_rel + U
    m, m_rel = n * f * scale, n_rel + f_rel + 2 * U
    total_off = m * m_rel + (h["residual"].abs() + m) * U
    out = dict(residual=total_off)
    d, d_off = gr.abs(), torch.zeros_like(b)
    if h["pre_weight"] is not None:
        pre = h["pre_weight"].abs()
        last = (r.square().mean(-1, keepdim=True) + eps).rsqrt()
        # the root of a sum whose entries are off: by the mean of r off over the mean of r^2
        last_rel = root + (r.abs() * total_off).mean(-1, keepdim=True) * last * last
        hat, hat_off = r.abs() * last, total_off * last + r.abs() * last * (last_rel + U)
        out["out"] = (hat_off + hat * U) * pre
        w, w_off = go.abs() * pre, go.abs() * pre * U
        dot = (w * hat).mean(-1, keepdim=True)
        dot_off = (w * hat_off + w_off * hat).mean(-1, keepdim=True) + dot * (W + 3) * U
        inner = w + hat * dot
        d = d + last * inner
        d_off = last * (w_off + hat_off * dot + hat * dot_off + inner * (last_rel + 3 * U)) + d * U
        R = r[..., 0].numel()
        out["grad pre_weight"] = (go.abs() * (hat_off + hat * (R + 2) * U)).flatten(0, -2).sum(0)
    out["grad residual"] = d_off
    R = r[..., 0].numel()
    if h["scale"] is not None:
        out["grad scale"] = ((d_off + d * (n_rel + f_rel + (R + 3) * U)) * f * n).flatten(0, -2).sum(0)
    d, d_off = d * scale, scale * (d_off + d * U)
    if h["gate"] is not None:
        out["grad gate"] = n * (d_off * steep + d * steep_off + d * steep * (n_rel + 3 * U))
    d, d_off = d * f, f * (d_off + d * (f_rel + U))
    if h["post_weight"] is not None:
        out["grad post_weight"] = (hat1 * (d_off + d * (hat1_rel + (R + 2) * U))).flatten(0, -2).sum(0)
        w, w_off = d * post, post * (d_off + d * U)
        dot = (w * hat1).mean(-1, keepdim=True)
        dot_off = (hat1 * (w_off + w * (hat1_rel + U))).mean(-1, keepdim=True) + dot * (W + 3) * U
        inner = w + hat1 * dot
        d, d_off = first * inner, first * (w_off + hat1 * dot_off + hat1 * dot * hat1_rel + inner * (root + 4 * U))
    out["grad block"] = d_off
    return out


def _check(a, gr, go, eps=1e-6, activation="sigmoid"):
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import check, cpu, norm
    r = bps.residual_norm(**a, eps=eps, activation=activation)
    h = {k: cpu(v) for k, v in a.items()}
    with torch.no_grad():
        total, _ = norm(**h, eps=eps, activation=activation)
        bounds = _bounds(h, cpu(gr), cpu(go), eps, activation, total)
    leaves = {k: h[k].requires_grad_() for k in NAMES if h[k] is not None}
    total, out = norm(**h, eps=eps, activation=activation)
    check("residual", r.residual, total, bounds["residual"])
    outs, grads = [total], [cpu(gr)]
    if out is not None:
        check("out", r.out, out, bounds["out"])
        outs.append(out)
        grads.append(cpu(go))
    got = bps.residual_norm_backward(result=r, grad_residual=gr, grad_out=go if out is not None else None, **a, eps=eps, activation=activation)
    want = dict(zip(leaves, torch.autograd.grad(outs, list(leaves.values()), grads)))
    for k in NAMES:
        if k in want:
            check("grad " + k, getattr(got, k), want[k], bounds["grad " + k])
        else:
            assert getattr(got, k) is None
    return r, got


@pytest.mark.parametrize("dtype,stream,weights", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("bf16", "bf16", "f32"), ("f16", "f16", "f16"),
                                                  ("f16", "f32", "f16"), ("f16", "f16", "f32")])
@pytest.mark.parametrize("width", [1, 7, 8, 64, 255, 256, 257, 769, 1100, 2100])
def test_types_and_widths(dtype, stream, weights, width):
    a, gr, go = _inputs((5,), width, dtype, width, stream, weights)
    _check(a, gr, go)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [4095, 4097, 8191, 9000, 16383, 16384])
def test_wide_rows(dtype, width):
    a, gr, go = _inputs((3,), width, dtype, width, "f32", "f32")
    _check(a, gr, go, activation="silu")


@pytest.mark.parametrize("without", [("post_weight",), ("gate",), ("scale",), ("pre_weight",), ("post_weight", "gate", "scale"), ("post_weight", "gate", "scale", "pre_weight"),
                                     ("gate", "pre_weight"), ("post_weight", "scale")])
@pytest.mark.parametrize("activation", ["sigmoid", "silu"])
def test_what_may_be_left_out(without, activation):
    a, gr, go = _inputs((4, 3), 100, "bf16", 5, "f32", "f32", without)
    _check(a, gr, go, activation=activation)


@pytest.mark.parametrize("rows", [1, 2, 5000])
def test_many_rows(rows):
    a, gr, go = _inputs((rows,), 33, "f32", rows)
    _check(a, gr, go)


@pytest.mark.parametrize("dtype,stream,rows,width", [("f32", "f32", 8500, 17), ("f32", "f32", 8200, 3), ("bf16", "f32", 2200, 500), ("f16", "f16", 2500, 769), ("bf16", "f32", 600, 2049), ("f32", "f32", 530, 4098)])
def test_more_rows_than_are_worked_on_at_once(dtype, stream, rows, width):
    a, gr, go = _inputs((rows,), width, dtype, rows, stream)
    _check(a, gr, go, activation="silu")


def test_rows_of_zeros_and_of_large_values():
    import torch
    a, gr, go = _inputs((6,), 96, "f32", 8)
    a["block"][1] = 0.0
    a["residual"][1] = 0.0
    a["residual"][2] = 0.0
    a["block"][3] *= 1e12
    a["residual"][4] *= 1e15
    a["gate"][5] = torch.linspace(-200, 200, 96, device="cuda")
    _check(a, gr, go, activation="silu")
    _check(a, gr, go)
    a, gr, go = _inputs((6,), 96, "f32", 9)
    a["block"][0] = 0.0
    a["residual"][0] = 0.0
    _check(a, gr, go, eps=0.25)


def test_gradients_of_one_output():
    """The other one's counts as zero."""
    import torch
    import paper_2103_07013_amd as bps
    a, gr, go = _inputs((7,), 130, "bf16", 10, "f32", "f32")
    r = bps.residual_norm(**a)
    for p, q in ((gr, None), (None, go)):
        got = bps.residual_norm_backward(result=r, grad_residual=p, grad_out=q, **a)
        want = bps.residual_norm_backward(result=r, grad_residual=torch.zeros_like(gr) if p is None else p, grad_out=torch.zeros_like(go) if q is None else q, **a)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype,width", [("f32", 33), ("bf16", 1030)])
def test_strides(dtype, width):
    import torch
    import paper_2103_07013_amd as bps
    a, gr, go = _inputs((9,), width, dtype, 11)
    want = bps.residual_norm(**a)
    grads = bps.residual_norm_backward(result=want, grad_residual=gr, grad_out=go, **a)
    wide = torch.zeros(9, 6 * width, dtype=a["block"].dtype, device="cuda")
    parts = [wide[:, k * width + 1:(k + 1) * width + 1] for k in range(5)]
    for p, t in zip(parts, (a["residual"], a["block"], a["gate"], gr, go)):
        p.copy_(t)
    b = dict(a, residual=parts[0], block=parts[1], gate=parts[2])
    got = bps.residual_norm(**b)
    new = bps.residual_norm_backward(result=got, grad_residual=parts[3], grad_out=parts[4], **b)
    assert torch.equal(got.residual, want.residual) and torch.equal(got.out, want.out) and all(torch.equal(p, q) for p, q in zip(new, grads))
    # one gate for all rows
    one = dict(a, gate=a["gate"][:1].expand(9, width))
    _check(one, gr, go)


def test_no_rows():
    import torch
    import paper_2103_07013_amd as bps
    a, gr, go = _inputs((0,), 40, "f32", 12)
    r = bps.residual_norm(**a)
    assert r.residual.shape == r.out.shape == (0, 40)
    d = bps.residual_norm_backward(result=r, grad_residual=gr, grad_out=go, **a)
    assert all((t == 0).all() for t in (d.post_weight, d.scale, d.pre_weight)) and d.block.shape == (0, 40)


def test_autograd():
    import torch
    import paper_2103_07013_amd as bps
    a, gr, go = _inputs((3, 5), 70, "bf16", 13, "f32", "f32")
    r = bps.residual_norm(**a)
    want = bps.residual_norm_backward(result=r, grad_residual=gr, grad_out=go, **a)
    leaves = [a[k].requires_grad_() for k in NAMES]
    s = bps.residual_norm(**a)
    assert not s.held.requires_grad
    got = torch.autograd.grad([s.residual, s.out], leaves, [gr, go])
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    # one output only, and a gate that is one row for all
    gate = a["gate"].detach()[:1, :1].clone().requires_grad_()
    s = bps.residual_norm(**dict(a, gate=gate.expand(3, 5, 70)))
    got, = torch.autograd.grad(s.out, [gate], go)
    whole = bps.residual_norm_backward(result=s, grad_out=go, **{k: (gate.expand(3, 5, 70) if k == "gate" else v).detach() for k, v in a.items()})
    assert torch.equal(got, whole.gate.sum((0, 1), keepdim=True))


def test_the_gradient_against_differences():
    import torch
    import paper_2103_07013_amd as bps
    a, gr, go = _inputs((4,), 24, "f32", 14)
    grads = bps.residual_norm_backward(result=bps.residual_norm(**a), grad_residual=gr, grad_out=go, **a)
    torch.manual_seed(3)
    for name in NAMES:
        way, step = torch.randn_like(a[name]), 2.0 ** -8
        p, q = (bps.residual_norm(**dict(a, **{name: a[name] + s * way})) for s in (step, -step))
        change = (p.residual.double() - q.residual.double()) * gr.double() + (p.out.double() - q.out.double()) * go.double()
        size = change.abs().sum() / (2 * step) + (p.residual.double() * gr.double()).abs().sum() + (p.out.double() * go.double()).abs().sum()
        # the third derivative times step^2 / 6 with inputs that move by up to 4 steps, and rounding over the step, 2^-24 * 30 * 2^8
        assert abs((getattr(grads, name).double() * way.double()).sum() - change.sum() / (2 * step)) < 2.0 ** -8 * size, name


def test_the_same_bits_every_time():
    import torch
    import paper_2103_07013_amd as bps
    a, gr, go = _inputs((3000,), 100, "bf16", 15, "f32", "f32")
    r = bps.residual_norm(**a)
    first = bps.residual_norm_backward(result=r, grad_residual=gr, grad_out=go, **a)
    for _ in range(5):
        assert all(torch.equal(p, q) for p, q in zip(first, bps.residual_norm_backward(result=r, grad_residual=gr, grad_out=go, **a)))
