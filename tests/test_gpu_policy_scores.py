"""Log probabilities of given tokens, with entropy and best alternatives, and their gradient, against the definition in 64 bits.

Tolerances, with e = 2^-24: a difference x - m times the scale's constant carries at most 3 e of itself, a power of two and a
logarithm 2 e each, and a sum of V terms in at least 4 partial sums of float32 at most V e / 4 worst of all, about V e / 128
where 64 lanes and more share it; ln z is at most ln V.  What a log probability may be off is so below
e (8 |value| + 16 ln V + 64 + V / 128), the entropy (two such sums) below twice that."""
import math

import pytest

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
HALF = {"float32": 0.0, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}     # half the distance of two values, relative
TINY = {"float32": 0.0, "bfloat16": 0.0, "float16": 2.0 ** -25}           # and where values are subnormal


def _torch():
    import torch
    return torch


def _slack(ref, V):
    torch = _torch()
    size = torch.where(torch.isfinite(ref), ref.abs(), 0.0)
    return E * (8 * size + 16 * math.log(V) + 64 + V / 128)


def _reference(logits, tokens, mask, scale, k=0):
    """(logp, entropy, lse, ids, values, p, part) in float64 on the CPU; no NaN and no +inf among entries that take part."""
    torch = _torch()
    x = logits.detach().cpu().double().reshape(-1, logits.shape[-1])
    t = tokens.cpu().long().reshape(-1)
    part = x > -math.inf
    if mask is not None:
        part = (mask.cpu() != 0).expand(logits.shape).reshape(x.shape) & ~torch.isnan(x.masked_fill(~(mask.cpu() != 0).expand(logits.shape).reshape(x.shape), 0.0)) & part | (
            (mask.cpu() != 0).expand(logits.shape).reshape(x.shape) & torch.isnan(x))
    y = torch.where(part, x * scale, -math.inf)
    lse = torch.logsumexp(y, 1)
    some = part.any(1)
    lp = torch.where(part, y - torch.where(some, lse, 0.0)[:, None], -math.inf)
    p = lp.exp()
    entropy = -torch.where(part, p * torch.where(part, lp, 0.0), 0.0).nan_to_num(0.0).sum(1)
    logp = torch.where(t < 0, 0.0, lp[torch.arange(len(t)), t.clamp(min=0)])
    ids = values = None
    if k:
        order = torch.where(part, x, -math.inf).sort(dim=1, descending=True, stable=True).indices[:, :k]
        there = part.gather(1, order)
        ids = torch.where(there, order, -1)
        values = torch.where(there, lp.gather(1, order), -math.inf)
        if order.shape[1] < k:
            ids = torch.nn.functional.pad(ids, (0, k - order.shape[1]), value=-1)
            values = torch.nn.functional.pad(values, (0, k - order.shape[1]), value=-math.inf)
    return logp, entropy, lse, ids, values, p, part


def _close(got, ref, slack):
    torch = _torch()
    got = got.detach().cpu().double().reshape(ref.shape)
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got)) and torch.equal(got[~fine], ref[~fine])
    off = (got - ref).abs()[fine]
    assert (off <= slack[fine]).all(), f"off by {float((off / slack[fine]).max())} of what is allowed"


def _check(logits, tokens, mask, scale=1.0, k=0, grads=True):
    import paper_2103_07013_amd as bps
    torch = _torch()
    V = logits.shape[-1]
    r = bps.log_probs(logits, tokens, mask=mask, scale=scale, top_k=k)
    logp, entropy, lse, ids, values, p, part = _reference(logits, tokens, mask, scale, k)
    _close(r.logp, logp, _slack(logp, V))
    _close(r.entropy, entropy, 2 * _slack(entropy, V))
    _close(r.lse, lse, _slack(lse, V))
    if k:
        assert torch.equal(r.top_ids.cpu().long().reshape(ids.shape), ids)
        _close(r.top_logp, values, _slack(values, V))
    if not grads:
        return
    g = torch.Generator().manual_seed(V)
    N = len(logp)
    gl, gh = torch.randn(N, generator=g), torch.randn(N, generator=g) * 0.3
    dx = bps.log_probs_backward(logits, tokens, r, gl.reshape(tokens.shape).cuda(), gh.reshape(tokens.shape).cuda(), mask=mask, scale=scale)
    t = tokens.cpu().long().reshape(-1)
    gl = torch.where((t < 0) | (logp == -math.inf), 0.0, gl.double())
    lp = torch.where(p > 0, p.log(), 0.0)
    ref = -p * (gl[:, None] + gh.double()[:, None] * (lp + entropy[:, None]))
    ref[torch.arange(N), t.clamp(min=0)] += gl
    ref = torch.where(part, ref * scale, 0.0)
    # p carries the error of ln p and lse relative to itself; the sums in brackets that of each of their terms
    weight = gl.abs()[:, None] * (p + (torch.arange(V)[None] == t[:, None])) + gh.double().abs()[:, None] * p * (1 + lp.abs() + entropy[:, None])
    kind = str(logits.dtype).replace("torch.", "")
    slack = scale * weight * (4 + lp.abs() + lse.nan_to_num(neginf=0.0).abs()[:, None]) * _slack(entropy, V)[:, None] + 1e-30
    _close(dx, ref, slack + HALF[kind] * (ref.abs() + slack) + TINY[kind])
    assert dx.dtype == logits.dtype and dx.shape == logits.shape


def _inputs(N, V, dtype, mask, seed=0, spread=3.0):
    torch = _torch()
    g = torch.Generator().manual_seed(seed * 1000 + N * 7 + V)
    logits = (torch.randn((N, V), generator=g) * spread).to(getattr(torch, dtype))
    tokens = torch.randint(-1, V, (N,), generator=g)
    m = None
    if mask == "shared":
        m = torch.rand(V, generator=g) < 0.7
    elif mask == "rows":
        m = (torch.rand((N, V), generator=g) < 0.7) & (torch.rand((N, 1), generator=g) < 0.9)
    return logits.cuda(), tokens.cuda(), None if m is None else m.cuda()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("mask", [None, "shared", "rows"])
@pytest.mark.parametrize("N,V", [(1, 1), (3, 2), (1024, 4), (77, 6), (130, 17), (65, 63), (64, 64), (9, 65), (33, 255), (5, 1000), (7, 2047), (3, 2049), (2, 8191),
                                 (3, 16385), (1, 50257), (2, 131072)])
def test_against_the_definition(N, V, mask, dtype):
    _check(*_inputs(N, V, dtype, mask), k=min(5, V))


@pytest.mark.parametrize("k", [0, 1, 2, 20, 63, 64])
@pytest.mark.parametrize("N,V", [(1, 1), (40, 5), (9, 64), (6, 300), (2, 5000), (1, 70001), (300, 1024), (600, 3000)])
def test_any_number_of_alternatives(N, V, k):
    _check(*_inputs(N, V, "bfloat16", "rows", seed=k), k=k, scale=0.7, grads=False)


@pytest.mark.parametrize("V", [4, 64, 1000, 40000])
@pytest.mark.parametrize("order", ["up", "down", "equal", "two"])
def test_orders_that_are_bad_for_a_running_choice(V, order):
    """Every entry better than all before it, or as good: ties go to the lower index."""
    torch = _torch()
    x = torch.arange(V, dtype=torch.float32) / V * 20
    x = {"up": x, "down": x.flip(0), "equal": torch.zeros(V), "two": (torch.arange(V) % 3 == 1).float()}[order]
    logits = x.expand(3, V).contiguous().cuda()
    _check(logits, torch.tensor([0, V - 1, -1], device="cuda"), None, k=64)
    _check(logits.bfloat16(), torch.tensor([0, V - 1, -1], device="cuda"), None, k=64)


@pytest.mark.parametrize("V", [3, 64, 777, 20000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_masks_that_leave_one_entry_or_none(V, dtype):
    torch = _torch()
    logits, _, _ = _inputs(6, V, dtype, None)
    mask = torch.zeros((6, V), dtype=torch.bool)
    mask[1, V - 1] = mask[2, 0] = mask[3, V // 2] = True
    mask[5] = True
    _check(logits, torch.tensor([0, V - 1, 1, -1, -1, 1], device="cuda"), mask.cuda(), k=3)


@pytest.mark.parametrize("V", [5, 64, 1030, 20001])
def test_what_masked_entries_hold_does_not_matter(V):
    import paper_2103_07013_amd as bps
    torch = _torch()
    logits, tokens, mask = _inputs(20, V, "float32", "rows")
    gl = torch.randn(20, device="cuda")
    results = []
    for fill in (0.0, math.nan, math.inf, -math.inf, 3.4e38, -3.4e38):
        x = logits.masked_fill(~mask, fill)
        r = bps.log_probs(x, tokens, mask=mask, top_k=4)
        results.append((*r, bps.log_probs_backward(x, tokens, r, gl, gl, mask=mask)))
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    assert (results[0][-1][~mask] == 0).all()


@pytest.mark.parametrize("V", [3, 64, 2000, 20000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_entries_of_the_lowest_value_and_minus_infinity(V, dtype):
    """A mask that was added as the type's lowest value: next to others such an entry has no weight, among its like it has all."""
    torch = _torch()
    logits, _, _ = _inputs(4, V, dtype, None)
    low = torch.finfo(logits.dtype).min
    logits[0, : V - 1] = low
    logits[1] = low
    logits[2, 1:] = -math.inf
    logits[3] = -math.inf
    import paper_2103_07013_amd as bps
    tokens = torch.tensor([V - 1, 1, 0, 2], device="cuda")
    r = bps.log_probs(logits, tokens, top_k=2)
    assert r.logp[0] == 0 and r.entropy[0] == 0
    assert abs(float(r.logp[1]) + math.log(V)) <= float(_slack(torch.tensor(math.log(V)), V)) and abs(float(r.entropy[1]) - math.log(V)) <= 2 * float(_slack(torch.tensor(math.log(V)), V))
    assert r.top_ids[1].tolist() == [0, 1]
    assert r.logp[2] == 0 and r.entropy[2] == 0 and r.top_ids[2].tolist() == [0, -1] and r.top_logp[2].tolist() == [0, -math.inf]
    assert r.lse[3] == -math.inf and r.logp[3] == -math.inf and r.entropy[3] == 0 and r.top_ids[3].tolist() == [-1, -1]
    one = torch.ones(4, device="cuda")
    dx = bps.log_probs_backward(logits, tokens, r, one, one).float()
    assert torch.isfinite(dx).all() and (dx[0] == 0).all() and (dx[2:] == 0).all()
    assert abs(float(dx[1].double().sum())) <= V * (E + HALF[dtype]) and float(dx[1, 1]) > 0


@pytest.mark.parametrize("V", [3, 64, 2000, 20000])
def test_nan_and_infinity_that_take_part_are_seen(V):
    import paper_2103_07013_amd as bps
    torch = _torch()
    logits, _, _ = _inputs(3, V, "float32", None)
    logits[0, V - 1] = math.nan
    logits[1, V // 2] = math.inf
    tokens = torch.tensor([0, 0, 0], device="cuda")
    r = bps.log_probs(logits, tokens, top_k=2)
    for t in (r.logp, r.entropy, r.lse):
        assert torch.isnan(t[:2]).all() and torch.isfinite(t[2])
    assert r.top_ids[0, 0] == V - 1 and r.top_ids[1, 0] == V // 2
    one = torch.ones(3, device="cuda")
    dx = bps.log_probs_backward(logits, tokens, r, one, one)
    assert torch.isnan(dx[:2]).all() and torch.isfinite(dx[2]).all()


@pytest.mark.parametrize("V", [6, 900, 30000])
def test_tokens_that_are_no_entry(V):
    """None is asked for by -1; others are answered with NaN, and nothing outside the row is read."""
    import paper_2103_07013_amd as bps
    torch = _torch()
    logits, _, _ = _inputs(6, V, "bfloat16", None)
    for kind in (torch.int32, torch.int64):
        tokens = torch.tensor([-1, V, -2, 2 ** 31 - 1, -2 ** 31, 1], dtype=kind, device="cuda")
        r = bps.log_probs(logits, tokens)
        assert r.logp[0] == 0 and torch.isnan(r.logp[1:5]).all() and torch.isfinite(r.logp[5])
        assert torch.isfinite(r.entropy).all()
        dx = bps.log_probs_backward(logits, tokens, r, torch.ones(6, device="cuda"))
        assert (dx[0] == 0).all() and torch.isnan(dx[1:5]).all() and torch.isfinite(dx[5]).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V,room,first", [(5, 9, 1), (64, 67, 3), (1001, 1004, 1), (5000, 5003, 2), (40001, 40003, 1)])
def test_rows_that_lie_apart_and_begin_anywhere(V, room, first, dtype):
    import paper_2103_07013_amd as bps
    torch = _torch()
    wide, tokens, mask = _inputs(12, room, dtype, "rows")
    tokens = tokens.clamp(max=V - 1)
    view = wide[:, first:first + V]
    mask = mask[:, :V].contiguous()
    r, s = bps.log_probs(view, tokens, mask=mask, top_k=3), bps.log_probs(view.contiguous(), tokens, mask=mask, top_k=3)
    assert all(torch.equal(a, b) for a, b in zip(r, s))
    one = torch.ones(12, device="cuda")
    out = torch.full_like(wide, 7.0)
    a = bps.log_probs_backward(view, tokens, r, one, one, mask=mask, out=out[:, first:first + V])
    b = bps.log_probs_backward(view.contiguous(), tokens, r, one, one, mask=mask)
    assert torch.equal(a, b)
    assert (out[:, :first] == 7).all() and (out[:, first + V:] == 7).all()
    into = wide.clone()
    bps.log_probs_backward(into[:, first:first + V], tokens, r, one, one, mask=mask, out=into[:, first:first + V])
    assert torch.equal(into[:, first:first + V], b) and torch.equal(into[:, first + V:], wide[:, first + V:])
    flipped = bps.log_probs(view[:1].expand(4, V), tokens[:4], top_k=2)
    assert torch.equal(flipped.lse, r.lse[:0].new_tensor(bps.log_probs(view[:1].contiguous(), tokens[:1]).lse.item()).expand(4))


def test_leading_dimensions_and_no_rows():
    import paper_2103_07013_amd as bps
    torch = _torch()
    logits, tokens, mask = _inputs(24, 50, "float32", "rows")
    r = bps.log_probs(logits, tokens, mask=mask, top_k=2)
    s = bps.log_probs(logits.view(2, 3, 4, 50), tokens.view(2, 3, 4), mask=mask.view(2, 3, 4, 50), top_k=2)
    assert s.logp.shape == (2, 3, 4) and s.top_ids.shape == (2, 3, 4, 2)
    assert all(torch.equal(a, b.reshape(a.shape)) for a, b in zip(r, s))
    one = bps.log_probs(logits[0], tokens[0], mask=mask[0])
    assert one.logp.shape == () and one.logp == r.logp[0]
    none = bps.log_probs(logits[:0], tokens[:0], top_k=3)
    assert none.logp.shape == (0,) and none.top_ids.shape == (0, 3)
    assert bps.log_probs_backward(logits[:0], tokens[:0], none, none.logp, none.logp).shape == (0, 50)


@pytest.mark.parametrize("V", [4, 65, 3000])
def test_gradient_against_differences(V):
    """Central differences of the forward values: with steps of 2^-5 the third derivatives (below 4 here) leave h^2 / 6 * 4, and errors of
    the values themselves e (16 ln V + 64 + V / 128 + 8 |value|) / h."""
    import paper_2103_07013_amd as bps
    torch = _torch()
    logits, tokens, mask = _inputs(1, V, "float32", "shared")
    tokens = mask.nonzero()[0].to(torch.int32)
    h = 2.0 ** -5
    r = bps.log_probs(logits, tokens, mask=mask)
    zero, one = torch.zeros(1, device="cuda"), torch.ones(1, device="cuda")
    dl = bps.log_probs_backward(logits, tokens, r, one, None, mask=mask)[0]
    dh = bps.log_probs_backward(logits, tokens, r, zero, one, mask=mask)[0]
    at = torch.arange(0, V, max(1, V // 40), device="cuda")
    shifted = logits.repeat(2 * len(at), 1)
    n = torch.arange(len(at), device="cuda")
    shifted[n, at] += h
    shifted[len(at) + n, at] -= h
    f = bps.log_probs(shifted, tokens.expand(2 * len(at)).contiguous(), mask=mask)
    slack = h * h * 4 / 6 + E * (16 * math.log(V) + 64 + V / 128 + 8 * 12) / h
    for value, grad in ((f.logp, dl), (f.entropy, dh)):
        value = value.double()
        d = (value[:len(at)] - value[len(at):]) / (2 * h)
        assert ((d - grad[at].double()).abs() <= slack).all()


def test_autograd():
    import paper_2103_07013_amd as bps
    torch = _torch()
    logits, tokens, mask = _inputs(64, 30, "float32", "rows")
    tokens[0] = -1
    a = logits.clone().requires_grad_()
    r = bps.log_probs(a, tokens, mask=mask, scale=0.5, top_k=2)
    w = torch.linspace(-1, 1, 64, device="cuda")
    fine = torch.isfinite(r.logp.detach())
    (r.logp[fine] * w[fine] + 0.1 * r.entropy[fine]).sum().backward()
    s = bps.log_probs(logits, tokens, mask=mask, scale=0.5)
    ref = bps.log_probs_backward(logits, tokens, s, torch.where(fine, w, 0.0), torch.where(fine, 0.1, 0.0), mask=mask, scale=0.5)
    assert torch.equal(a.grad, ref)
    assert not r.lse.requires_grad and not r.top_logp.requires_grad
    b = logits.clone().requires_grad_()
    bps.log_probs(b, tokens, mask=mask, scale=0.5).entropy.sum().backward()
    assert torch.equal(b.grad, bps.log_probs_backward(logits, tokens, s, None, torch.ones(64, device="cuda"), mask=mask, scale=0.5))


@pytest.mark.parametrize("N,V,k", [(5000, 4, 0), (300, 50257, 5), (2, 131072, 20), (1000, 900, 3)])
def test_the_same_bits_every_time(N, V, k):
    import paper_2103_07013_amd as bps
    torch = _torch()
    logits, tokens, _ = _inputs(N, V, "bfloat16", None)
    first = bps.log_probs(logits, tokens, top_k=k)
    for _ in range(3):
        assert all(a is None or torch.equal(a, b) for a, b in zip(first, bps.log_probs(logits, tokens, top_k=k)))


@pytest.mark.parametrize("N,V", [(1024, 6), (3, 100000)])
def test_on_another_stream_and_in_a_graph(N, V):
    import paper_2103_07013_amd as bps
    torch = _torch()
    sets = [_inputs(N, V, "float32", "rows", seed=s) for s in range(4)]
    gl, gh = torch.randn(N, device="cuda"), torch.randn(N, device="cuda")

    def both(x, t, m, **kw):
        r = bps.log_probs(x, t, mask=m, top_k=4, **kw)
        return (*r, bps.log_probs_backward(x, t, r, gl, gh, mask=m, **kw))

    ref = [both(*s) for s in sets]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got = both(*sets[1], stream=stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref[1]))
    x, t, m = (v.clone() for v in sets[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both(x, t, m)
    for k in (0, 1, 2, 3, 2):
        for a, b in zip((x, t, m), sets[k]):
            a.copy_(b)
        graph.replay()
        if k % 2:
            assert all(torch.equal(a, b) for a, b in zip(both(*sets[3]), ref[3]))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, ref[k])), f"replay of set {k}"


def test_rows_behind_the_reach_of_32_bits():
    """Elements and bytes whose offsets pass 2^32 / 2 and 2^32."""
    import paper_2103_07013_amd as bps
    torch = _torch()
    N, V = 20011, 131072
    logits = torch.zeros((N, V), dtype=torch.bfloat16, device="cuda")
    few = [0, 1, 8191, 16383, 16385, 20010]
    logits[few] = torch.randn((len(few), V), device="cuda").bfloat16() * 3
    tokens = torch.arange(N, device="cuda")
    r = bps.log_probs(logits, tokens, top_k=2)
    s = bps.log_probs(logits[few].contiguous(), tokens[few], top_k=2)
    assert torch.equal(r.top_ids[few], s.top_ids)
    for a, b in zip(r[:5], s[:5]):           # held has five rows
        assert torch.allclose(a[few].double(), b.double(), rtol=1e-5, atol=1e-5)
    assert torch.allclose(r.entropy[2:8191], torch.full((1,), math.log(V), device="cuda"), rtol=1e-5)
    one = torch.ones(N, device="cuda")
    dx = bps.log_probs_backward(logits, tokens, r, one, one, out=logits)
    assert dx.data_ptr() == logits.data_ptr()
    row = torch.full((V,), -1.0 / V, device="cuda").bfloat16()
    row[20009] = 1.0
    assert torch.allclose(dx[20009].float(), row.float(), rtol=2.0 ** -7, atol=1e-9)
