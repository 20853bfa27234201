"""AdamW over many tensors against its definition: in 64 bits, and for 8-bit states bit for bit, by the rule that
include/bps.h states, in numpy's float32."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
BLOCK = 256
SIZES = [1, 255, 256, 257, 5, 4095, 4096, 4097, 20000, 3, 64]
RULE = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-6)


def _torch():
    import torch
    return torch


def _mixed(h):
    h = np.asarray(h, np.uint64) & np.uint64(0xFFFFFFFF)
    for shift, factor in ((16, 0x6A09E667), (15, 0xBB67AE85)):
        h = ((h ^ (h >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
    return h ^ (h >> np.uint64(16))


def _decode(codes, exponents, top):
    c = codes.reshape(-1, BLOCK).astype(np.int64)
    f, k = c >> 3, c & 7
    e = exponents.astype(np.int64)[:, None]
    value = np.where(f > 0, (1 + k / 8) * 2.0 ** (e - 127 - top + f), k / 8 * 2.0 ** (e - 127 - top + 1))
    return np.where(e == 255, np.nan, value).reshape(-1)


def _encode(x, top, least, u):
    """(codes, exponents) of magnitudes x (float32), in numbers of 64 bits where the rule has exact ones."""
    x = x.astype(np.float64).reshape(-1, BLOCK)
    largest = x.max(1, keepdims=True)
    e = np.full(largest.shape, least, np.int64)
    some = largest > 0
    m, p = np.frexp(largest, where=some, out=(np.zeros_like(largest), np.zeros(largest.shape, np.int32)))
    e[some] = np.maximum(least, (p + 126 + (m > 1.875 / 2))[some])
    field = np.maximum(1, np.where(x > 0, np.frexp(x)[1] + 126, 0) - e + top)
    quantum = 2.0 ** (e - 127 - top + field - 3)
    n = np.floor((x / quantum).astype(np.float32) + u.reshape(-1, BLOCK).astype(np.float32)).astype(np.int64)
    return (8 * (field - 1) + n).astype(np.uint8).reshape(-1), e[:, 0].astype(np.uint8)


class Model:
    """The same step in numpy float32, every operation rounded by itself."""

    def __init__(self, params, sizes, bits, seed, decay, lr_scale, exp_avg=None):
        self.sizes, self.bits, self.seed, self.decay, self.lr_scale, self.t = sizes, bits, seed, decay, lr_scale, 0
        self.starts = np.cumsum([0] + [-(-n // BLOCK) * BLOCK for n in sizes])
        self.total = int(self.starts[-1])
        self.w = [p.copy() for p in params]
        self.m, self.v = (np.zeros(self.total, np.float32) for _ in range(2))
        self.codes = [np.zeros(self.total, np.uint8), np.zeros(self.total // BLOCK, np.uint8), np.zeros(self.total, np.uint8), np.zeros(self.total // BLOCK, np.uint8)]

    def step(self, grads, lr, betas, eps, factor=1.0):
        f = np.float32
        self.t += 1
        b1, b2 = betas
        key = _mixed(self.seed + self.t * 0x9E3779B9)
        u = _mixed(((np.arange(self.total, dtype=np.uint64) * np.uint64(0x9E3779B9)) & np.uint64(0xFFFFFFFF)) ^ key)
        for i, (n, g) in enumerate(zip(self.sizes, grads)):
            if g is None:
                continue
            a, b = int(self.starts[i]), int(self.starts[i + 1])
            x = np.zeros(b - a, np.float32)
            x[:n] = g.astype(np.float32) * f(factor)
            m, v = self.m[a:b], self.v[a:b]
            m = m * f(b1) + x * f(1 - b1)
            v = v * f(b2) + x * f(1 - b2) * x
            step_size = f(lr / (1 - b1 ** self.t) * float(f(self.lr_scale[i])))
            root = f(1 / math.sqrt(1 - b2 ** self.t))
            keep = f(1 - lr * float(f(self.lr_scale[i])) * float(f(self.decay[i])))
            self.w[i] = (self.w[i] * keep - (m / (np.sqrt(v) * root + f(eps)) * step_size)[:n]).astype(np.float32)
            if self.bits == 8:
                cm, em = _encode(np.abs(m), 15, 20, (u[a:b] & np.uint64(0xFFFF)) / 65536.0)
                cv, ev = _encode(v, 31, 36, (u[a:b] >> np.uint64(16)) / 65536.0)
                c, r = self.codes, slice(a // BLOCK, b // BLOCK)
                c[0][a:b], c[1][r], c[2][a:b], c[3][r] = cm | np.where(m < 0, 128, 0).astype(np.uint8), em, cv, ev
                m = (_decode(cm, em, 15) * np.where(m < 0, -1, 1)).astype(np.float32)
                v = _decode(cv, ev, 31).astype(np.float32)
            self.m[a:b], self.v[a:b] = m, v


def _tensors(sizes, dtype, seed, size=1.0):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * size).to(getattr(torch, dtype)).cuda() for n in sizes]


def _same(opt, model, params, dtype):
    """All state and weights, bit for bit (and the rounded weights of 16-bit parameters)."""
    torch = _torch()
    m, v = (s.cpu().numpy() for s in opt.states())
    inside = np.zeros(opt.total, bool)
    for a, n in zip(opt.starts, model.sizes):
        inside[a:a + n] = True
    assert np.array_equal(m[inside], model.m[inside]) and np.array_equal(v[inside], model.v[inside])
    if model.bits == 8:
        for got, ref in zip((opt.exp_avg, opt.exp_avg_sq), (model.codes[0], model.codes[2])):
            assert np.array_equal(got.cpu().numpy()[inside], ref[inside])
        assert np.array_equal(opt.exp_avg_exponent.cpu().numpy(), model.codes[1]) and np.array_equal(opt.exp_avg_sq_exponent.cpu().numpy(), model.codes[3])
    for i, (p, a, n) in enumerate(zip(params, opt.starts, model.sizes)):
        w = p if dtype == "float32" else opt.master[a:a + n]
        assert np.array_equal(w.cpu().numpy(), model.w[i]), f"tensor {i} of {n}"
        if dtype != "float32":
            assert torch.equal(p, w.to(p.dtype))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grads", [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float16", "float16"), ("float16", "float32")])
def test_steps_bit_for_bit(dtype, grads, bits):
    import paper_2103_07013_amd as bps
    params = _tensors(SIZES, dtype, 1)
    decay, lr_scale = [0.1 * (i % 3) for i in range(len(SIZES))], [1.0, 0.5, 2.0] * 3 + [1.0, 0.25]
    with bps.AdamW(params, **RULE, weight_decay=decay, lr_scale=lr_scale, state_bits=bits, seed=77) as opt:
        model = Model([p.float().cpu().numpy() for p in params], SIZES, bits, 77, decay, lr_scale)
        for k in range(6):
            g = _tensors(SIZES, grads, 100 + k, size=10.0 ** (k % 3 - 1))
            g[4] = None if k in (0, 3) else g[4]
            opt.step(g, grad_scale=0.5)
            model.step([None if x is None else x.float().cpu().numpy() for x in g], RULE["lr"], RULE["betas"], RULE["eps"], 0.5)
            _same(opt, model, params, dtype)
        assert opt.steps == 6


def test_against_the_definition_in_64_bits():
    """Ten roundings or fewer lie between the inputs and a state or an update, each at most 2^-24 of its result; what cancels in
    m and w is held to the sizes of its terms."""
    import paper_2103_07013_amd as bps
    torch = _torch()
    params = _tensors(SIZES, "float32", 2)
    before = [p.double() for p in params]
    with bps.AdamW(params, **RULE, weight_decay=0.1) as opt:
        m = [torch.zeros_like(p) for p in before]
        v = [torch.zeros_like(p) for p in before]
        for t in range(1, 5):
            grads = _tensors(SIZES, "float32", 50 + t)
            held = [p.double().clone() for p in params]
            opt.step(grads)
            for i, g in enumerate(grads):
                a, n = opt.starts[i], SIZES[i]
                size = (m[i].abs() * 0.9 + 0.1 * g.double().abs())
                m[i], v[i] = 0.9 * m[i] + 0.1 * g.double(), 0.99 * v[i] + 0.01 * g.double() ** 2
                assert ((opt.exp_avg[a:a + n].double() - m[i]).abs() <= 4 * E * size).all()
                assert ((opt.exp_avg_sq[a:a + n].double() - v[i]).abs() <= 5 * E * v[i]).all()
                m[i], v[i] = opt.exp_avg[a:a + n].double(), opt.exp_avg_sq[a:a + n].double()
                step = RULE["lr"] / (1 - 0.9 ** t) * m[i] / ((v[i] / (1 - 0.99 ** t)).sqrt() + 1e-6)
                ref = held[i] * (1 - RULE["lr"] * 0.1) - step
                assert ((params[i].double() - ref).abs() <= E * (3 * held[i].abs() + 10 * step.abs() + ref.abs())).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_bound_on_the_norm(dtype, bits):
    import paper_2103_07013_amd as bps
    torch = _torch()
    sizes = SIZES + [70001]
    for limit, bound in ((1.0, True), (1e4, False)):
        params = _tensors(sizes, dtype, 3)
        plain = [p.clone() for p in params]
        with bps.AdamW(params, **RULE, state_bits=bits, max_grad_norm=limit, seed=5) as opt, bps.AdamW(plain, **RULE, state_bits=bits, seed=5) as other:
            for k in range(3):
                g = _tensors(sizes, dtype, 20 + k)
                norm = math.sqrt(sum(float(x.double().square().sum()) for x in g)) * 0.25
                assert (norm > limit) == bound
                opt.step(g, grad_scale=0.25)
                # the norm is the root of a sum of 17 squares a lane, joined in float32 and then in 64 bits
                assert abs(float(opt.grad_norm) - norm) <= norm * 32 * E
                factor = np.float32(limit) / np.float32(float(opt.grad_norm)) if bound else np.float32(1)
                # the same products in the same order: gradient times scale, times the bound's factor
                other.step([x.float() * 0.25 * float(factor) if dtype == "float32" else (x.float() * 0.25) * float(factor) for x in g])
                for a, b in zip(params, plain):
                    assert torch.equal(a, b)
                assert torch.equal(opt.exp_avg, other.exp_avg) and torch.equal(opt.exp_avg_sq, other.exp_avg_sq)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_gradient_that_is_not_finite(bits, bad):
    """With a bound on the norm the step changes nothing; without it NaN is kept in sight, in its own element or block."""
    import paper_2103_07013_amd as bps
    torch = _torch()
    for limit in (1.0, 0.0):
        params = _tensors(SIZES, "float32", 3)
        with bps.AdamW(params, **RULE, state_bits=bits, max_grad_norm=limit) as opt:
            opt.step(_tensors(SIZES, "float32", 30))
            held = [p.clone() for p in params] + [s.clone() for s in (opt.exp_avg, opt.exp_avg_sq)]
            g = _tensors(SIZES, "float32", 31)
            g[8][12345] = bad
            opt.step(g)
            if limit:
                assert all(torch.equal(a, b) for a, b in zip(held, [*params, opt.exp_avg, opt.exp_avg_sq])) and not math.isfinite(float(opt.grad_norm))
                opt.step(_tensors(SIZES, "float32", 32))
                assert math.isfinite(float(opt.grad_norm)) and all(torch.isfinite(p).all() for p in params)
            else:
                assert not torch.isfinite(params[8][12345]) and all(int((~torch.isfinite(p)).sum()) == (i == 8) for i, p in enumerate(params))
                m, v = opt.states()
                at = opt.starts[8] + 12345
                wrong = (~torch.isfinite(m)).nonzero().flatten().tolist()
                block = list(range(at // BLOCK * BLOCK, at // BLOCK * BLOCK + BLOCK))
                assert wrong == ([at] if bits == 32 else block) and not torch.isfinite(v[at])


@pytest.mark.parametrize("which", ["tiny", "huge", "zero", "spread"])
def test_8_bit_states_of_any_size(which):
    import paper_2103_07013_amd as bps
    torch = _torch()
    sizes = [1000, 7]
    params = _tensors(sizes, "float32", 4)
    with bps.AdamW(params, **RULE, state_bits=8, seed=3) as opt:
        model = Model([p.cpu().numpy() for p in params], sizes, 8, 3, [0.01] * 2, [1.0] * 2)
        for k in range(4):
            g = _tensors(sizes, "float32", 60 + k)
            if which == "spread":
                g = [x * 10.0 ** (torch.rand(x.shape, generator=torch.Generator().manual_seed(k)).cuda() * 20 - 15) for x in g]
            else:
                g = [x * {"tiny": 1e-25, "huge": 1e17, "zero": 0.0}[which] for x in g]
            opt.step(g)
            model.step([x.cpu().numpy() for x in g], RULE["lr"], RULE["betas"], RULE["eps"])
            _same(opt, model, params, "float32")


def test_8_bit_states_keep_the_mean_of_long_averages():
    """An average that moves by a thousandth a step moves by less than half the distance of two codes (a sixteenth) at a time.
    From v = 1 with gradients of 0.5, v tends to 0.25 as 0.25 + 0.75 * 0.999^t.  Rounding to a neighbour at distance q <= v / 8 adds a variance of
    at most p (1 - p) q^2, p q the change: about 0.001 v^2 / 8 a step, so at most v^2 / 16 in all, a deviation of v / 4; over 65536
    elements their mean is within 5 deviations of v / 4 / 256 (0.5 %)."""
    import paper_2103_07013_amd as bps
    torch = _torch()
    n = 65536
    p = [torch.zeros(n, device="cuda")]
    with bps.AdamW(p, lr=0.0, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, state_bits=8, seed=9) as opt:
        opt.exp_avg_sq.fill_(31 * 8)
        opt.exp_avg_sq_exponent.fill_(127)          # 1.0
        assert (opt.states()[1] == 1).all()
        g = [torch.full((n,), 0.5, device="cuda")]
        for t in range(1, 2001):
            opt.step(g)
            if t % 500 == 0:
                m, v = (float(x.double().mean()) for x in opt.states())
                ref = 0.25 + 0.75 * 0.999 ** t
                assert abs(v / ref - 1) <= 5 * 0.25 / 256 and abs(m / 0.5 - 1) <= 0.01, (t, v, ref, m)


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors_and_views_that_begin_anywhere(bits):
    """More tensors than one launch takes addresses for; odd addresses."""
    import paper_2103_07013_amd as bps
    torch = _torch()
    sizes = [1 + (37 * i) % 611 for i in range(1000)]
    flat, gflat = torch.randn(sum(sizes) + 1, device="cuda"), torch.randn(sum(sizes) + 1, device="cuda")
    params, grads = list(flat[1:].split(sizes)), list(gflat[1:].split(sizes))
    with bps.AdamW(params, **RULE, state_bits=bits, max_grad_norm=3.0, seed=8) as opt:
        model = Model([p.cpu().numpy() for p in params], sizes, bits, 8, [0.01] * 1000, [1.0] * 1000)
        for _ in range(2):
            opt.step(grads)
            norm = float(opt.grad_norm)
            assert abs(norm - float(gflat[1:].double().norm())) <= norm * 32 * E
            model.step([g.cpu().numpy() for g in grads], RULE["lr"], RULE["betas"], RULE["eps"], np.float32(3.0) / np.float32(norm))
            _same(opt, model, params, "float32")


def test_gradients_of_the_parameters_and_what_is_kept_between_steps():
    import paper_2103_07013_amd as bps
    torch = _torch()
    w = [torch.nn.Parameter(t) for t in _tensors([40, 300], "float32", 6)]
    with bps.AdamW(w, **RULE) as opt:
        opt.step()                                    # no gradients: nothing happens
        assert opt.steps == 0
        (w[0].sum() * 2 + w[1].square().sum()).backward()
        held = [t.detach().clone() for t in w]
        opt.step()
        # a first step moves every weight by lr against its gradient's sign, and by the decay
        for t, h in zip(w, held):
            ref = h * (1 - RULE["lr"] * 0.01) - RULE["lr"] * t.grad.sign()
            assert torch.allclose(t.detach(), ref, rtol=0, atol=1e-5)
        w[0].data = w[0].data.clone()
        with pytest.raises(ValueError, match="no longer where it was"):
            opt.step()


@pytest.mark.parametrize("bits", [32, 8])
def test_on_another_stream_and_in_a_graph(bits):
    """A captured step replays with the step number it was captured with, on the gradients as they are then."""
    import paper_2103_07013_amd as bps
    torch = _torch()

    def make():
        p = _tensors(SIZES, "float32", 12)
        return p, bps.AdamW(p, **RULE, state_bits=bits, max_grad_norm=2.0, seed=4)

    gs = [_tensors(SIZES, "float32", 70 + k) for k in range(5)]
    side = torch.cuda.Stream()
    (p1, o1), (p2, o2), (p3, o3) = make(), make(), make()
    torch.cuda.synchronize()
    for g in gs:
        o1.step(g)
        o2.step(g, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(p1, p2)) and torch.equal(o1.exp_avg, o2.exp_avg)
    held = [g.clone() for g in gs[0]]
    (p4, o4) = make()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o3.step(held)
    for g in gs:
        for a, b in zip(held, g):
            a.copy_(b)
        graph.replay()
        o4.steps = 0
        o4.step(g)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p3, p4)) and torch.equal(o3.exp_avg, o4.exp_avg) and torch.equal(o3.exp_avg_sq, o4.exp_avg_sq)
    for o in (o1, o2, o3, o4):
        o.close()


def test_tensors_behind_the_reach_of_32_bits():
    import paper_2103_07013_amd as bps
    torch = _torch()
    n = 2 ** 31 + 5000
    p = [torch.zeros(300, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")]
    with bps.AdamW(p, lr=0.5, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.0, state_bits=8) as opt:
        g = [torch.ones_like(t) for t in p]
        g[1][-4000:] = -1
        opt.step(g)
        assert (p[1][:5000] == -0.5).all() and (p[1][2 ** 31 - 100:2 ** 31 + 1000] == -0.5).all() and (p[1][-4000:] == 0.5).all()
        assert float(p[1][::4097].double().sum()) == -0.5 * (p[1][::4097].numel() - 2 * int((torch.arange(0, n, 4097) >= n - 4000).sum()))
