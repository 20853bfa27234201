"""Definitions of the operators of a policy's memory in 64 bits, step by step, with bounds for what float32 and one rounding to
the outputs' type can add.

U is half a step of float32.  A result that is a sum of products has an error of at most (roundings along the longest way through it) U
times the sum of its products' magnitudes, to first order; the magnitudes come from the same formulas with all factors positive."""
import torch

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(t, dtype):
    """One rounding of t to dtype: half a step relative to the value, or half the smallest step there is (2^-24 in float16's subnormals)."""
    return t.abs() * (torch.finfo(dtype).eps / 2) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def check(name, got, want, bound):
    """bound: absolute, before the rounding to got's type"""
    got, want = got.detach().cpu(), want.detach()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    off = (got.double() - want).abs()
    # the rounding is of the value that was computed, which is up to `bound` larger; products of errors are under a hundredth of their sum
    limit = 1.01 * (bound + half_step(want.abs() + bound, got.dtype)) + 1e-30
    worst = (off / limit).max().item() if off.numel() else 0.0
    assert bool((off <= limit).all()), (name, "is", worst, "times its bound off at", (off / limit).argmax().item())


def cpu(v):
    return v.detach().cpu().double() if torch.is_tensor(v) and v.is_floating_point() else v.cpu() if torch.is_tensor(v) else v


def _ends(lengths, batch, steps):
    return [steps] * batch if lengths is None else [min(max(int(n), 0), steps) for n in lengths]


def conv(x, weight, bias, silu, starts, lengths, state):
    """(out, state, sum of magnitudes in front of silu), differentiable"""
    B, T, D = x.shape
    K = weight.shape[1]
    outs, states, sizes = [], [], []
    for b, end in enumerate(_ends(lengths, B, T)):
        window = list(state[b]) if state is not None else [x.new_zeros(D)] * (K - 1)
        rows, size = [], []
        for t in range(T):
            if t >= end:
                rows.append(x.new_zeros(D))
                size.append(x.new_zeros(D))
                continue
            if starts is not None and starts[b, t]:
                window = [x.new_zeros(D)] * (K - 1)
            window = window + [x[b, t]]
            u = sum(weight[:, k] * window[k] for k in range(K)) + (bias if bias is not None else 0.0)
            size.append(sum((weight[:, k] * window[k]).abs() for k in range(K)).detach() + (bias.abs().detach() if bias is not None else 0.0))
            rows.append(u * torch.sigmoid(u) if silu else u)
            window = window[1:]
        outs.append(torch.stack(rows) if rows else x.new_zeros(0, D))
        sizes.append(torch.stack(size) if size else x.new_zeros(0, D))
        states.append(torch.stack(window) if window else x.new_zeros(0, D))
    # a graph over the weights even where no step is in its sequence
    return torch.stack(outs) + 0.0 * weight.sum(), torch.stack(states), torch.stack(sizes)


def over_channels(b, D):
    """[..., groups, states] -> [..., states, D]"""
    return b.transpose(-1, -2).repeat_interleave(D // b.shape[-2], -1)


def scan(x, delta, A, B, C, D, gate, delta_bias, soft, starts, lengths, state):
    """(out, state), differentiable"""
    batch, T, width = x.shape
    B, C = (over_channels(t if t.dim() == 4 else t[:, :, None], width) for t in (B, C))
    ends = torch.tensor(_ends(lengths, batch, T))
    h = state if state is not None else x.new_zeros(batch, A.shape[0], width)
    outs = []
    for t in range(T):
        on = (t < ends)[:, None]
        v = delta[:, t] + (delta_bias if delta_bias is not None else 0.0)
        d = torch.nn.functional.softplus(v, threshold=700.0) if soft else v
        before = h
        if starts is not None:
            before = torch.where((starts[:, t] & on[:, 0])[:, None, None], 0.0, h)
        new = (d[:, None] * A).exp() * before + (d * torch.where(on, x[:, t], 0.0))[:, None] * B[:, t]
        y = (new * C[:, t]).sum(1) + (D * x[:, t] if D is not None else 0.0)
        if gate is not None:
            y = y * gate[:, t] * torch.sigmoid(gate[:, t])
        outs.append(torch.where(on, y, 0.0))
        h = torch.where(on[..., None], new, h)
    return torch.stack(outs, 1) if outs else x.new_zeros(batch, 0, width), h


def scan_bounds(x, delta, A, B, C, D, gate, delta_bias, soft, starts, lengths, state, grad_out=None):
    """Bounds of the errors of scan's outputs, and of its gradients where there is a grad_out.

    Roundings: a step's size d = softplus(v) is e^-|v| through a power of two, whose argument is off by |v| U twice and which is off by 2 U, a
    quotient of 4 U, a series and two products of 4 U; v itself is off by U |v|: relative to d at most (4 |v| + 16) U in all.  A decay
    2^(d A log2 e) is off by |d A| (d's error and 3 roundings) and 2 U; where the time is in chunks the sum of its d's, T roundings, takes
    their place.  All decays on the way of one term are at most T, each followed by one rounding."""
    batch, T, width = x.shape
    groups = B.shape[2] if B.dim() == 4 else 1
    B, C = (over_channels((t if t.dim() == 4 else t[:, :, None]).abs(), width) for t in (B, C))
    on = (torch.arange(T) < torch.tensor(_ends(lengths, batch, T))[:, None])[..., None]
    v = delta + (delta_bias if delta_bias is not None else 0.0)
    d = torch.nn.functional.softplus(v, threshold=700.0) if soft else v
    rel_d = ((4 * v.abs() + 16) * U if soft else U * (1 + (delta.abs() + (delta_bias.abs() if delta_bias is not None else 0.0)) / v.abs().clamp(min=1e-30)))
    d, x_size = torch.where(on, d.abs(), 0.0), torch.where(on, x.abs(), 0.0)
    rel_d = torch.where(on, rel_d, 0.0)
    N = A.shape[0]
    a = (torch.where(on, torch.nn.functional.softplus(v, threshold=700.0) if soft else v, 0.0)[:, :, None] * A).exp()
    rel_a = (d[:, :, None] * A.abs()) * (rel_d[:, :, None] + (3 + T) * U) + 3 * U
    if starts is not None:
        a = torch.where((starts[..., None] & on)[:, :, None], 0.0, a)
    h = state.abs() if state is not None else x.new_zeros(batch, N, width)
    e = torch.zeros_like(h)
    hs, es = [h], [e]
    for t in range(T):
        added = (d[:, t] * x_size[:, t])[:, None] * B[:, t]
        e = a[:, t] * (e + h * rel_a[:, t]) + added * (rel_d[:, t][:, None] + 3 * U)
        h = a[:, t] * h + added
        e = e + h * U
        hs.append(h)
        es.append(e)
    hs, es = torch.stack(hs, 1), torch.stack(es, 1)
    skip = D.abs() * x_size if D is not None else torch.zeros_like(x)
    y = (hs[:, 1:] * C).sum(2) + skip
    y_off = (es[:, 1:] * C).sum(2) + (N + 3) * U * y
    s = torch.sigmoid(gate) if gate is not None else None
    # a sigmoid: argument |z| U twice, a power of 2 U, a sum and a quotient of 3 U
    rel_s = (2 * gate.abs() + 8) * U if gate is not None else 0.0
    f = gate.abs() * s if gate is not None else torch.ones_like(x)
    bounds = dict(out=torch.where(on, f * (y_off + y * (rel_s + 2 * U)), 0.0), state=es[:, -1])
    if grad_out is None:
        return bounds
    grad = torch.where(on, grad_out.abs(), 0.0)
    dy = grad * f
    rel_dy = rel_s + 3 * U
    g, off = torch.zeros_like(h), torch.zeros_like(h)
    gs, offs = [None] * T, [None] * T
    for t in reversed(range(T)):
        if t + 1 < T:
            off = a[:, t + 1] * (off + g * rel_a[:, t + 1])
            g = a[:, t + 1] * g
        new = C[:, t] * dy[:, t][:, None]
        off = off + new * ((rel_dy[:, t] if torch.is_tensor(rel_dy) else rel_dy) if gate is None else rel_dy[:, t][:, None])
        g = g + new
        off = off + g * 2 * U
        gs[t], offs[t] = g, off
    gs, offs = torch.stack(gs, 1), torch.stack(offs, 1)
    rd = rel_dy if gate is None else rel_dy[:, :, None]
    each = width // groups

    def shared(p, terms):
        """Summed over the channels of a group; `terms` are the terms' own errors"""
        p, terms = (q.reshape(batch, T, N, groups, each).sum(4).transpose(2, 3) for q in (p, terms))
        return terms + p * (each + 2) * U

    c_terms = dy[:, :, None] * hs[:, 1:]
    in_size = (d * x_size)[:, :, None]
    b_terms = gs * in_size
    p = gs * a * hs[:, :-1]
    # h before: its own error; g after its decay
    p_off = a * (offs * hs[:, :-1] + gs * es[:, :-1]) + p * (rel_a + 3 * U)
    gb, gb_off = (gs * B).sum(2), (offs * B).sum(2) + (N + 1) * U * (gs * B).sum(2)
    dd = gb * x_size + (p * A.abs()).sum(2)
    dd_off = gb_off * x_size + (p_off * A.abs()).sum(2) + (N + 3) * U * dd
    slope = torch.sigmoid(v) if soft else torch.ones_like(x)
    rel_v = (3 * v.abs() + 8) * U if soft else 0.0
    dv, dv_off = dd * slope, slope * (dd_off + dd * (rel_v + 2 * U))
    rows = batch * T
    bounds |= dict(x=d * gb_off + d * gb * (rel_d + 2 * U) + (D.abs() * dy * (rel_dy + 3 * U) if D is not None else 0.0),
                   delta=dv_off, A=(p_off * d[:, :, None] + p * d[:, :, None] * (rel_d[:, :, None] + (rows + 2) * U)).sum((0, 1)),
                   B=shared(b_terms, offs * in_size + b_terms * (rel_d[:, :, None] + 3 * U)), C=shared(c_terms, dy[:, :, None] * es[:, 1:] + c_terms * (rd + 2 * U)),
                   D=(dy * x_size * (rel_dy + (rows + 2) * U)).sum((0, 1)), delta_bias=(dv_off + dv * (rows + 2) * U).sum((0, 1)))
    if gate is not None:
        steep = s * (1 + gate.abs() * (1 - s))
        # the slope's terms are off as the sigmoid is, and by 1 - s, which is off by as much as 1
        steep_off = steep * (rel_s + 4 * U) + s * gate.abs() * (s * rel_s + U)
        bounds["gate"] = grad * (y_off * steep + y * steep_off + y * steep * 3 * U)
    return bounds


def norm(residual, block, post_weight, gate, scale, pre_weight, eps, activation):
    """(sum, out), differentiable"""
    m = block
    if post_weight is not None:
        m = m / (m.square().mean(-1, keepdim=True) + eps).sqrt() * post_weight
    if gate is not None:
        m = m * (gate * torch.sigmoid(gate) if activation == "silu" else torch.sigmoid(gate))
    if scale is not None:
        m = m * scale
    r = residual + m
    return r, None if pre_weight is None else r / (r.square().mean(-1, keepdim=True) + eps).sqrt() * pre_weight
