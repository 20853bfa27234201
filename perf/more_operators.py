"""What a recurrent policy asks of its operators between embedding and scores, as a list of cases that can be timed.

A block of such a policy runs a short convolution over time, a selective state space scan, and joins the result to the residual stream:

  "conv", "conv_learn", "conv_step"   causal depthwise convolution with SiLU: whole sequences; the same and its gradient; one step
  "scan", "scan_learn", "scan_step"   the scan, its output gated: whole sequences; the same and its gradient; one step
  "norm", "norm_learn"                norm after a block, gate, scale, residual sum and the norm before the next block; the same and its gradient

Episodes begin in the middle of sequences where `starts` says so, sequences end at their `lengths`.  `run` computes the plain forms
in float32 torch operations, or makes the framework's calls where `own` is true.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-6


def listed():
    return [
        # one rollout step of 1024 environments: the last inputs of each are kept, finished ones begin anew
        dict(name="conv_step_actions", op="conv_step", B=1024, D=512, K=4, dtype="f32", starts=0.01),
        # a few prompts of different lengths, odd sizes
        dict(name="conv_prompts", op="conv", B=3, T=5003, D=1111, K=3, dtype="f16", starts=0.0, ragged=True),
        # an update over long sequences
        dict(name="conv_learn_long", op="conv_learn", B=8, T=4096, D=2048, K=4, dtype="bf16", starts=0.0, ragged=False),
        # the same rollout step: the state is what is read and written
        dict(name="scan_step_actions", op="scan_step", B=1024, D=512, N=16, G=1, dtype="f32", starts=0.01),
        # one token of every request that is being served
        dict(name="scan_step_requests", op="scan_step", B=192, D=4096, N=16, G=1, dtype="bf16", starts=0.0),
        # one long prompt: few rows, many steps
        dict(name="scan_prompt", op="scan", B=1, T=16384, D=2048, N=16, G=1, dtype="bf16", starts=0.0, ragged=False),
        # a padded batch of prompts of odd sizes, inputs and outputs of the state shared by half of the channels each
        dict(name="scan_prompts", op="scan", B=7, T=1111, D=778, N=13, G=2, dtype="f16", starts=0.002, ragged=True),
        # one update over 32 steps of 1024 environments, episodes that end in between
        dict(name="scan_learn_rollout", op="scan_learn", B=1024, T=32, D=512, N=16, G=1, dtype="f32", starts=0.01, ragged=False),
        # an update over long sequences, the largest that is held at once
        dict(name="scan_learn_long", op="scan_learn", B=8, T=4096, D=2048, N=16, G=1, dtype="bf16", starts=0.0, ragged=False),
        # a rollout step's residual stream
        dict(name="norm_step", op="norm", R=1024, D=256, dtype="f32", stream="f32", post=True, gate="sigmoid", scale=True),
        # an update of odd sizes, no norm after the block
        dict(name="norm_learn_odd", op="norm_learn", R=5003, D=769, dtype="f16", stream="f16", post=False, gate="silu", scale=True),
        # an update over long sequences, 16-bit blocks on a float32 stream
        dict(name="norm_learn_long", op="norm_learn", R=32768, D=4096, dtype="bf16", stream="f32", post=True, gate="sigmoid", scale=True),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["conv", "conv_learn", "conv_step", "scan", "scan_learn", "scan_step", "norm", "norm_learn"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op.startswith("norm"):
        D = _log_int(rng, 16, 8192)
        return dict(op=op, R=_log_int(rng, 1, 100_000_000 // D), D=D, dtype=dtype, stream=rng.choice([dtype, "f32"]), post=rng.random() < 0.5,
                    gate=rng.choice(["none", "sigmoid", "silu"]), scale=rng.random() < 0.5)
    starts = rng.choice([0.0, 0.005, 0.05])
    if op == "conv_step":
        D = _log_int(rng, 8, 8192)
        return dict(op=op, B=_log_int(rng, 1, min(4096, 8_000_000 // D)), D=D, K=rng.randint(2, 8), dtype=dtype, starts=starts)
    if op in ("conv", "conv_learn"):
        D = _log_int(rng, 8, 4096)
        T = _log_int(rng, 1, 16384)
        B = _log_int(rng, 1, max(1, min(2048, 60_000_000 // (D * T))))
        return dict(op=op, B=B, T=T, D=D, K=rng.randint(2, 8), dtype=dtype, starts=starts, ragged=rng.random() < 0.5)
    N = rng.choice([1, 4, 8, 13, 16, 16, 16, 27, 32])
    G = rng.choice([1, 1, 1, 2, 4])
    D = G * _log_int(rng, 4, 4096 // G)
    if op == "scan_step":
        return dict(op=op, B=_log_int(rng, 1, min(4096, 60_000_000 // (D * N))), D=D, N=N, G=G, dtype=dtype, starts=starts)
    T = _log_int(rng, 1, 16384 if op == "scan" else 4096)
    B = _log_int(rng, 1, max(1, min(2048, 500_000_000 // (D * T * N))))
    while B * T * D * N > 1_000_000_000:
        T //= 2
    return dict(op=op, B=B, T=T, D=D, N=N, G=G, dtype=dtype, starts=starts, ragged=rng.random() < 0.5)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)
    op, dtype, D = case["op"], _TYPES[case["dtype"]], case["D"]

    def normal(*shape, size=1.0, dtype=dtype):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * size).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)

    s = dict(op=op)
    if op.startswith("norm"):
        R, stream = case["R"], _TYPES[case["stream"]]
        s["residual"], s["block"] = normal(R, D, size=2.0, dtype=stream), normal(R, D, size=0.7)
        s["post_weight"] = normal(D, size=0.2, dtype=torch.float32).add_(1.0) if case["post"] else None
        s["gate"], s["activation"] = (None, "sigmoid") if case["gate"] == "none" else (normal(R, D), case["gate"])
        s["scale"] = uniform(D) * 0.5 + 0.1 if case["scale"] else None
        s["pre_weight"] = normal(D, size=0.2, dtype=torch.float32).add_(1.0)
        if op == "norm_learn":
            s["grad_residual"], s["grad_out"] = normal(R, D, size=0.1, dtype=stream), normal(R, D, size=0.1)
    else:
        B, T = case["B"], case.get("T")
        step = T is None
        rows = (B,) if step else (B, T)
        s["x"] = normal(*rows, D)
        s["starts"] = uniform(*rows) < case["starts"] if case["starts"] else None
        if not step:
            s["lengths"] = None
            if case["ragged"]:
                s["lengths"] = (uniform(B) * 1.2 * T).clamp(max=T).to(torch.int32)
        if op.startswith("conv"):
            K = case["K"]
            s["weight"], s["bias"] = normal(D, K, size=1.0 / math.sqrt(K)), normal(D, size=0.1)
            s["state"] = normal(B, K - 1, D) if step or op == "conv" else None
        else:
            N, G = case["N"], case["G"]
            s["delta"] = normal(*rows, D, size=0.5)
            s["gate"] = normal(*rows, D)
            # the rates 1 .. N, moved by training; steps of 0.001 .. 0.1
            s["A"] = -(torch.arange(1, N + 1, device="cuda", dtype=torch.float32)[:, None] * (normal(N, D, size=0.1, dtype=torch.float32)).exp())
            s["B"], s["C"] = normal(*rows, G, N), normal(*rows, G, N)
            s["D"] = normal(D, size=0.2, dtype=torch.float32).add_(1.0)
            s["delta_bias"] = torch.expm1(torch.exp(uniform(D) * math.log(100.0) + math.log(0.001))).log()
            s["state"] = normal(B, N, D, dtype=torch.float32) if step or op == "scan" else None
        if op.endswith("learn"):
            s["grad_out"] = normal(*rows, D, size=0.1)
    if own:
        import paper_2103_07013_amd as bps
        s["bps"] = bps
    return s


def run(s):
    return (_own if own else _plain)[s["op"]](s)


# ---------------------------------------------------------------------------------------------- plain forms

def _silu(x):
    return x / (1.0 + (-x).exp())


def _silu_slope(x):
    p = 1.0 / (1.0 + (-x).exp())
    return p * (1.0 + x * (1.0 - p))


def _inside(s):
    """Which steps are in their sequence, [B, T, 1]; and how many steps each sequence has."""
    B, T = s["x"].shape[:2]
    if s["lengths"] is None:
        return None, torch.full((B,), T, device="cuda")
    return (torch.arange(T, device="cuda") < s["lengths"][:, None])[..., None], s["lengths"].long()


def _episodes(s):
    """The number of starts up to each step, [B, T]: two steps are of one episode where it is the same."""
    return None if s["starts"] is None else s["starts"].cumsum(1)


def _padded(s):
    """The inputs behind the state's, with the episode that each belongs to."""
    x, K = s["x"].float(), s["weight"].shape[1]
    before = s["state"].float() if s["state"] is not None else x.new_zeros((x.shape[0], K - 1, x.shape[2]))
    episode = _episodes(s)
    if episode is not None:
        episode = torch.nn.functional.pad(episode, (K - 1, 0))
    return torch.cat([before, x], 1), episode


def _tap(xs, episode, k, K, T):
    """What the k-th weight meets at each step."""
    x = xs[:, k:k + T]
    if episode is not None:
        x = torch.where((episode[:, k:k + T] == episode[:, K - 1:])[..., None], x, 0.0)
    return x


def _conv_sum(s):
    xs, episode = _padded(s)
    w, T, K = s["weight"].float(), s["x"].shape[1], s["weight"].shape[1]
    u = s["bias"].float().expand(s["x"].shape)
    for k in range(K):
        u = u + _tap(xs, episode, k, K, T) * w[:, k]
    return u, xs, episode


def _plain_conv(s):
    u, xs, episode = _conv_sum(s)
    inside, lengths = _inside(s)
    out = _silu(u)
    if inside is not None:
        out = torch.where(inside, out, 0.0)
    at = lengths[:, None] + torch.arange(s["weight"].shape[1] - 1, device="cuda")
    last = xs.gather(1, at[..., None].expand(-1, -1, xs.shape[2]))
    if episode is not None:
        end = (at[:, :1] + s["weight"].shape[1] - 2).clamp(min=0)
        last = torch.where((episode.gather(1, at) == episode.gather(1, end))[..., None], last, 0.0)
    dtype = s["x"].dtype
    return dict(out=out.to(dtype), state=last.to(dtype))


def _plain_conv_learn(s):
    u, xs, episode = _conv_sum(s)
    inside, _ = _inside(s)
    w, T, K, dtype = s["weight"].float(), s["x"].shape[1], s["weight"].shape[1], s["x"].dtype
    du = s["grad_out"].float() * _silu_slope(u)
    if inside is not None:
        du = torch.where(inside, du, 0.0)
    dx, dw = torch.zeros_like(xs), []
    for k in range(K):
        part = du * w[:, k]
        if episode is not None:
            part = torch.where((episode[:, k:k + T] == episode[:, K - 1:])[..., None], part, 0.0)
        dx[:, k:k + T] += part
        dw.append((du * _tap(xs, episode, k, K, T)).sum((0, 1)))
    return dict(_plain_conv(s), grad_x=dx[:, K - 1:].to(dtype), grad_weight=torch.stack(dw, 1).to(dtype), grad_bias=du.sum((0, 1)).to(dtype))


def _plain_conv_step(s):
    state = s["state"].float()
    if s["starts"] is not None:
        state = torch.where(s["starts"][:, None, None], 0.0, state)
    xs = torch.cat([state, s["x"].float()[:, None]], 1)
    u = (xs * s["weight"].float().T).sum(1) + s["bias"].float()
    s["state"].copy_(xs[:, 1:])
    return dict(out=_silu(u).to(s["x"].dtype), state=s["state"])


def _softplus(v):
    return v.clamp(min=0.0) + torch.log1p((-v.abs()).exp())


def _over_channels(b, D):
    """[..., G, N] -> [..., N, D]: each group's for its channels"""
    return b.float().transpose(-1, -2).repeat_interleave(D // b.shape[-2], -1)


def _recurrence(a, b):
    """h[t] = a[t] h[t - 1] + b[t] with h[-1] = 0: pieces of about sqrt(T) steps side by side, then what each piece hands on"""
    T = a.shape[0]
    size = math.isqrt(T - 1) + 1
    count = -(-T // size)
    rest = count * size - T
    if rest:
        a, b = (torch.cat([x, x.new_zeros((rest, *x.shape[1:]))]) for x in (a, b))
    h, c = (x.reshape(count, size, *x.shape[1:]).clone() for x in (b, a))
    for i in range(1, size):
        h[:, i].addcmul_(c[:, i], h[:, i - 1])
        c[:, i] *= c[:, i - 1]
    for k in range(1, count):
        h[k].addcmul_(c[k], h[k - 1, -1])
    return h.flatten(0, 1)[:T]


def _scan_parts(s):
    """Time first: steps, decays [T, B, N, D], what is added to the state, states behind each step and before each."""
    x, D = s["x"].float().transpose(0, 1), s["x"].shape[-1]
    v = s["delta"].float().transpose(0, 1) + s["delta_bias"]
    d = _softplus(v)
    inside, _ = _inside(s)
    if inside is not None:
        inside = inside.transpose(0, 1)
        d = torch.where(inside, d, 0.0)
    a = (d[:, :, None] * s["A"]).exp()
    if s["starts"] is not None:
        begins = s["starts"].T[..., None] if inside is None else s["starts"].T[..., None] & inside
        a = torch.where(begins[:, :, None], 0.0, a)
    b = _over_channels(s["B"], D).transpose(0, 1)
    added = (d * x)[:, :, None] * b
    first = s["state"] if s["state"] is not None else torch.zeros_like(added[0])
    added[0] += a[0] * first
    return x, v, d, a, b, torch.cat([first[None], _recurrence(a, added)]), inside


def _scan_out(s, x, states, inside):
    c = _over_channels(s["C"], x.shape[-1]).transpose(0, 1)
    y = (states[1:] * c).sum(2) + s["D"] * x
    out = y * _silu(s["gate"].float().transpose(0, 1))
    if inside is not None:
        out = torch.where(inside, out, 0.0)
    return c, y, dict(out=out.transpose(0, 1).to(s["x"].dtype).contiguous(), state=states[-1].clone())


def _plain_scan(s):
    x, _, _, _, _, states, inside = _scan_parts(s)
    return _scan_out(s, x, states, inside)[2]


def _plain_scan_learn(s):
    x, v, d, a, b, states, inside = _scan_parts(s)
    c, y, out = _scan_out(s, x, states, inside)
    z, grad = s["gate"].float().transpose(0, 1), s["grad_out"].float().transpose(0, 1)
    if inside is not None:
        grad = torch.where(inside, grad, 0.0)
    dy = grad * _silu(z)
    # the same recurrence from the last step to the first, each step's decay being the next one's
    g = _recurrence(torch.cat([a[1:], torch.zeros_like(a[:1])]).flip(0), (c * dy[:, :, None]).flip(0)).flip(0)
    del c
    T, B, N, D = g.shape
    groups = s["B"].shape[2]

    def shared(p):
        """[T, B, N, D] -> [B, T, G, N], summed over each group's channels"""
        return p.view(T, B, N, groups, D // groups).sum(4).permute(1, 0, 3, 2).to(s["x"].dtype)

    grad_c = shared(states[1:] * dy[:, :, None])
    grad_b = shared(g * (d * x)[:, :, None])
    gb = (g * b).sum(2)
    del b
    p = g * a * states[:-1]
    dd = gb * x + (p * s["A"]).sum(2)
    dv = dd * (1.0 / (1.0 + (-v).exp()))
    if inside is not None:
        dv = torch.where(inside, dv, 0.0)
    dtype = s["x"].dtype
    back = lambda t: t.transpose(0, 1).to(dtype).contiguous()  # noqa: E731
    return dict(out, grad_x=back(d * gb + s["D"] * dy), grad_delta=back(dv), grad_A=(p * d[:, :, None]).sum((0, 1)), grad_B=grad_b, grad_C=grad_c,
                grad_D=(dy * x).sum((0, 1)), grad_gate=back(grad * y * _silu_slope(z)), grad_delta_bias=dv.sum((0, 1)))


def _plain_scan_step(s):
    x, D = s["x"].float(), s["x"].shape[-1]
    d = _softplus(s["delta"].float() + s["delta_bias"])
    state = s["state"]
    if s["starts"] is not None:
        state = torch.where(s["starts"][:, None, None], 0.0, state)
    h = (d[:, None] * s["A"]).exp() * state + (d * x)[:, None] * _over_channels(s["B"], D)
    y = (h * _over_channels(s["C"], D)).sum(1) + s["D"] * x
    s["state"].copy_(h)
    return dict(out=(y * _silu(s["gate"].float())).to(s["x"].dtype), state=s["state"])


def _norm_parts(s):
    """The block's part of the sum and the factors that it is made of, the sum, and both roots."""
    b = s["block"].float()
    n, post = b, None
    if s["post_weight"] is not None:
        post = (b.square().mean(1, keepdim=True) + _EPS).rsqrt()
        n = b * post * s["post_weight"]
    f = torch.ones_like(b)
    if s["gate"] is not None:
        f = _silu(s["gate"].float()) if s["activation"] == "silu" else 1.0 / (1.0 + (-s["gate"].float()).exp())
    m = f * n
    if s["scale"] is not None:
        m = m * s["scale"]
    r = s["residual"].float() + m
    pre = (r.square().mean(1, keepdim=True) + _EPS).rsqrt()
    return n, f, r, post, pre


def _norm_out(s, r, pre):
    return dict(residual=r.to(s["residual"].dtype), out=(r * pre * s["pre_weight"]).to(s["block"].dtype))


def _plain_norm(s):
    _, _, r, _, pre = _norm_parts(s)
    return _norm_out(s, r, pre)


def _plain_norm_learn(s):
    n, f, r, post, pre = _norm_parts(s)
    out = _norm_out(s, r, pre)
    dtype, go = s["block"].dtype, s["grad_out"].float()
    hat = r * pre
    out["grad_pre_weight"] = (go * hat).sum(0)
    w = go * s["pre_weight"]
    dr = s["grad_residual"].float() + pre * (w - hat * (w * hat).mean(1, keepdim=True))
    out["grad_residual"] = dr.to(s["residual"].dtype)
    if s["scale"] is not None:
        out["grad_scale"] = (dr * f * n).sum(0)
        dr = dr * s["scale"]
    if s["gate"] is not None:
        z = s["gate"].float()
        out["grad_gate"] = (dr * n * (_silu_slope(z) if s["activation"] == "silu" else f * (1.0 - f))).to(dtype)
    dn = dr * f
    if post is not None:
        hat = s["block"].float() * post
        out["grad_post_weight"] = (dn * hat).sum(0)
        w = dn * s["post_weight"]
        dn = post * (w - hat * (w * hat).mean(1, keepdim=True))
    out["grad_block"] = dn.to(dtype)
    return out


_plain = dict(conv=_plain_conv, conv_learn=_plain_conv_learn, conv_step=_plain_conv_step, scan=_plain_scan, scan_learn=_plain_scan_learn,
              scan_step=_plain_scan_step, norm=_plain_norm, norm_learn=_plain_norm_learn)


# ---------------------------------------------------------------------------------------------- the framework's operators

def _own_conv(s):
    r = s["bps"].causal_conv(s["x"], s["weight"], s["bias"], starts=s["starts"], lengths=s["lengths"], state=s["state"])
    return dict(out=r.out, state=r.state)


def _own_conv_learn(s):
    g = s["bps"].causal_conv_backward(s["grad_out"], s["x"], s["weight"], s["bias"], starts=s["starts"], lengths=s["lengths"], state=s["state"])
    return dict(_own_conv(s), grad_x=g.x, grad_weight=g.weight, grad_bias=g.bias)


def _own_conv_step(s):
    return dict(out=s["bps"].causal_conv_step(s["x"], s["state"], s["weight"], s["bias"], starts=s["starts"]), state=s["state"])


def _scan_rest(s):
    return dict(D=s["D"], gate=s["gate"], delta_bias=s["delta_bias"], starts=s["starts"])


def _own_scan(s):
    r = s["bps"].selective_scan(s["x"], s["delta"], s["A"], s["B"], s["C"], **_scan_rest(s), lengths=s["lengths"], state=s["state"])
    return dict(out=r.out, state=r.state)


def _own_scan_learn(s):
    inputs = s["x"], s["delta"], s["A"], s["B"], s["C"]
    r = s["bps"].selective_scan(*inputs, **_scan_rest(s), lengths=s["lengths"], state=s["state"], hold=True)
    g = s["bps"].selective_scan_backward(s["grad_out"], *inputs, r, **_scan_rest(s), lengths=s["lengths"])
    return dict(out=r.out, state=r.state, grad_x=g.x, grad_delta=g.delta, grad_A=g.A, grad_B=g.B, grad_C=g.C, grad_D=g.D, grad_gate=g.gate, grad_delta_bias=g.delta_bias)


def _own_scan_step(s):
    return dict(out=s["bps"].selective_scan_step(s["x"], s["delta"], s["state"], s["A"], s["B"], s["C"], **_scan_rest(s)), state=s["state"])


def _norm_rest(s):
    return dict(post_weight=s["post_weight"], gate=s["gate"], scale=s["scale"], pre_weight=s["pre_weight"], eps=_EPS, activation=s["activation"])


def _own_norm(s):
    r = s["bps"].residual_norm(s["residual"], s["block"], **_norm_rest(s))
    return dict(residual=r.residual, out=r.out)


def _own_norm_learn(s):
    r = s["bps"].residual_norm(s["residual"], s["block"], **_norm_rest(s))
    g = s["bps"].residual_norm_backward(s["residual"], s["block"], r, s["grad_residual"], s["grad_out"], **_norm_rest(s))
    out = dict(residual=r.residual, out=r.out, grad_residual=g.residual, grad_block=g.block, grad_pre_weight=g.pre_weight)
    for name in ("post_weight", "gate", "scale"):
        if s[name] is not None:
            out["grad_" + name] = getattr(g, name)
    return out


_own = dict(conv=_own_conv, conv_learn=_own_conv_learn, conv_step=_own_conv_step, scan=_own_scan, scan_learn=_own_scan_learn, scan_step=_own_scan_step,
            norm=_own_norm, norm_learn=_own_norm_learn)


# ---------------------------------------------------------------------------------------------- work and exact values

def work(case):
    op, D, b = case["op"], case["D"], _BYTES[case["dtype"]]
    if op.startswith("norm"):
        n, r = case["R"] * D, _BYTES[case["stream"]]
        gate = b if case["gate"] != "none" else 0
        data = n * (2 * r + 2 * b + gate)
        if op == "norm":
            return dict(bytes=data, flops=12 * n)
        # both gradients in, those of stream, block and gate out
        return dict(bytes=data + n * (2 * r + 2 * b + gate), flops=40 * n)
    n = case["B"] * case.get("T", 1) * D
    if op.startswith("conv"):
        K = case["K"]
        state = case["B"] * (K - 1) * D * b
        if op == "conv_learn":
            return dict(bytes=4 * n * b + state, flops=(6 * K + 16) * n)
        return dict(bytes=2 * n * b + 2 * state, flops=(2 * K + 4) * n)
    N, G = case["N"], case["G"]
    state, shared = case["B"] * N * D * 4, case["B"] * case.get("T", 1) * G * N * 2 * b
    data = 4 * n * b + shared + N * D * 4 + state
    if op != "scan_learn":
        return dict(bytes=data + state, flops=n * (7 * N + 12))
    return dict(bytes=data + 4 * n * b + shared + N * D * 4, flops=n * (22 * N + 40))


def exact(case, seed):
    """run()'s outputs from the definition in 64 bits."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    with torch.enable_grad():
        return dict(conv=_exact_conv, scan=_exact_scan, norm=_exact_norm)[case["op"].split("_")[0]](case, s)


def _exact_conv(case, s):
    """Window by window: the inputs of the last K steps travel along, and are cleared where an episode begins."""
    w, bias, K = s["weight"], s["bias"], case["K"]
    step = "T" not in case
    x = s["x"][:, None] if step else s["x"]
    B, T, D = x.shape
    starts = s["starts"] if s["starts"] is None or not step else s["starts"][:, None]
    lengths = None if step else s["lengths"]
    # how many steps ago the episode began, more than any window where it began before the call
    age = torch.full((B,), K, device="cuda")
    ages = []
    for t in range(T):
        age = (age + 1).clamp(max=K)
        if starts is not None:
            age = torch.where(starts[:, t], 0, age)
        ages.append(age)
    age = torch.stack(ages, 1)
    before = s["state"] if s["state"] is not None else x.new_zeros((B, K - 1, D))
    learn = case["op"] == "conv_learn"
    dx = torch.zeros_like(x)
    dw, db = torch.zeros_like(w), torch.zeros_like(bias)
    out, last = [], []
    for i in range(B):
        xi = x[i].clone().requires_grad_(learn)
        wi, bi = w.clone().requires_grad_(learn), bias.clone().requires_grad_(learn)
        whole = torch.cat([before[i], xi])
        window = whole.unfold(0, K, 1)  # [T, D, K]
        keep = torch.arange(K - 1, -1, -1, device="cuda") <= age[i][:, None]
        u = (window * wi * keep[:, None]).sum(2) + bi
        o = u * torch.sigmoid(u)
        n = T if lengths is None else int(lengths[i])
        o = torch.cat([o[:n], torch.zeros_like(o[n:])])
        if learn:
            gx, gw, gb = torch.autograd.grad(o, (xi, wi, bi), s["grad_out"][i])
            dx[i] = gx
            dw += gw
            db += gb
        out.append(o.detach())
        end = whole[n:n + K - 1].detach().clone()
        if n:
            end[torch.arange(K - 2, -1, -1, device="cuda") > age[i][n - 1]] = 0.0
        last.append(end)
    out, last = torch.stack(out), torch.stack(last)
    if step:
        return dict(out=out[:, 0], state=last)
    return dict(out=out, state=last, grad_x=dx, grad_weight=dw, grad_bias=db) if learn else dict(out=out, state=last)


def _exact_scan(case, s):
    """Step by step; the gradient by differentiation of pieces of the time, from the last to the first."""
    step = "T" not in case
    names = ("x", "delta", "gate", "B", "C")
    if step:
        s = dict(s, lengths=None, **{k: s[k][:, None] for k in (*names, "starts") if s[k] is not None})
    x = s["x"]
    B, T, D = x.shape
    each = D // case["G"]

    def piece(h, part, shared, t0):
        outs = []
        for i in range(part["x"].shape[1]):
            p = {k: v[:, i] for k, v in part.items()}
            if s["starts"] is not None:
                begins = s["starts"][:, t0 + i]
                if s["lengths"] is not None:
                    begins = begins & (t0 + i < s["lengths"])
                h = torch.where(begins[:, None, None], 0.0, h)
            d = torch.nn.functional.softplus(p["delta"] + shared["delta_bias"], threshold=700.0)
            b, c = (p[k].transpose(1, 2).repeat_interleave(each, 2) for k in ("B", "C"))
            new = h * torch.exp(d[:, None] * shared["A"]) + (d * p["x"])[:, None] * b
            y = (new * c).sum(1) + shared["D"] * p["x"]
            o = y * p["gate"] * torch.sigmoid(p["gate"])
            if s["lengths"] is not None:
                on = (t0 + i < s["lengths"])[:, None]
                new, o = torch.where(on[..., None], new, h), torch.where(on, o, 0.0)
            h = new
            outs.append(o)
        return h, torch.stack(outs, 1)

    size = max(1, min(256, 400_000_000 // (B * D * case["N"])))
    pieces = range(0, T, size)
    h = s["state"] if s["state"] is not None else x.new_zeros((B, case["N"], D))
    shared = {k: s[k] for k in ("A", "D", "delta_bias")}
    before, out = [], []
    with torch.no_grad():
        for t in pieces:
            before.append(h)
            h, o = piece(h, {k: s[k][:, t:t + size] for k in names}, shared, t)
            out.append(o)
    out = torch.cat(out, 1)
    if step:
        return dict(out=out[:, 0], state=h)
    result = dict(out=out, state=h)
    if case["op"] == "scan_learn":
        grads = {k: torch.zeros_like(s[k]) for k in (*names, *shared)}
        gh = torch.zeros_like(h)
        for t, h0 in reversed(list(zip(pieces, before))):
            h0 = h0.clone().requires_grad_()
            part = {k: s[k][:, t:t + size].clone().requires_grad_() for k in names}
            own_shared = {k: v.clone().requires_grad_() for k, v in shared.items()}
            h1, o = piece(h0, part, own_shared, t)
            leaves = [h0, *part.values(), *own_shared.values()]
            got = torch.autograd.grad([h1, o], leaves, [gh, s["grad_out"][:, t:t + size]])
            gh = got[0]
            for k, v in zip(names, got[1:]):
                grads[k][:, t:t + size] = v
            for k, v in zip(shared, got[1 + len(names):]):
                grads[k] += v
        result |= {"grad_" + k: v for k, v in grads.items()}
    return result


def _exact_norm(case, s):
    """A part of the rows at a time, differentiated."""
    learn = case["op"] == "norm_learn"
    weights = {k: s[k].clone().requires_grad_(learn) for k in ("post_weight", "scale", "pre_weight") if s[k] is not None}
    parts, sums = [], {k: torch.zeros_like(v) for k, v in weights.items()}
    size = max(1, 30_000_000 // case["D"])
    for i in range(0, case["R"], size):
        rows = {k: s[k][i:i + size].clone().requires_grad_(learn) for k in ("residual", "block", "gate") if s[k] is not None}
        m = rows["block"]
        if "post_weight" in weights:
            m = m / torch.sqrt((m * m).mean(1, keepdim=True) + _EPS) * weights["post_weight"]
        if "gate" in rows:
            p = torch.sigmoid(rows["gate"])
            m = m * (p * rows["gate"] if s["activation"] == "silu" else p)
        if "scale" in weights:
            m = m * weights["scale"]
        r = rows["residual"] + m
        o = r / torch.sqrt((r * r).mean(1, keepdim=True) + _EPS) * weights["pre_weight"]
        part = dict(residual=r.detach(), out=o.detach())
        if learn:
            got = torch.autograd.grad([r, o], [*rows.values(), *weights.values()], [s["grad_residual"][i:i + size], s["grad_out"][i:i + size]])
            part |= {"grad_" + k: v for k, v in zip(rows, got)}
            for k, v in zip(weights, got[len(rows):]):
                sums[k] += v
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    return out | {"grad_" + k: v for k, v in sums.items()} if learn else out
