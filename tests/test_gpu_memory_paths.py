"""The memory's operators where their sizes choose other ways through the kernels: wide convolutions and long runs, threads and work-groups that go on to further
sequences, one step as a sequence, the shortest chunks, wide rows that share their sums."""
import pytest

pytestmark = pytest.mark.gpu

# ---------------------------------------------------------------------------------------------- convolution

# Additions that a term of a weight's gradient goes through, at most: two runs of 64 steps in a thread, up to 128 threads of a work-group in LDS (their
# runs have 8 steps) or a sixteenth of 2^17 / 65 parts in the join, and its 16 slices.
ADDITIONS = 2 * 64 + 128 + 16


def _near(name, got, want, bound):
    """memory_reference.check on the GPU"""
    from memory_reference import half_step
    off = (got.double() - want).abs()
    limit = 1.01 * (bound + half_step(want.abs() + bound, got.dtype)) + 1e-30
    assert bool((off <= limit).all()), (name, "is", (off / limit).max().item(), "times its bound off at", (off / limit).argmax().item())


def _convolution(x, weight, bias, starts, lengths, state, grad):
    """(out, sizes of the sums in front of silu, gradients' bounds as weights of |du|, gradients) in 64 bits, all windows at once."""
    import torch
    from memory_reference import U
    B, T, D = x.shape
    K = weight.shape[1]
    at = torch.arange(T, device=x.device)
    begun = torch.where(starts, at, -K).cummax(1).values
    inside = (at < lengths.clamp(0, T)[:, None])[..., None]
    seen = [(at - begun >= i)[..., None] for i in range(K)]
    x, weight, bias = (t.double().requires_grad_() for t in (x, weight, bias))
    whole = torch.cat([state.double(), x], 1)
    u, size = bias, bias.detach().abs()
    for i in range(K):
        part = torch.where(seen[i], whole[:, K - 1 - i:K - 1 - i + T], 0.0) * weight[:, K - 1 - i]
        u, size = u + part, size + part.detach().abs()
    out = torch.where(inside, u * torch.sigmoid(u), 0.0)
    grads = torch.autograd.grad(out, (x, weight, bias), grad.double())
    # the bounds of test_gpu_memory_conv.py, with the additions that there are
    u_off = (K + 1) * U * size
    g = torch.where(inside, grad.double().abs(), 0.0)
    du, du_off = 1.1 * g, g * (0.5 * u_off + (2 * size + 12) * (1 + size) * U + 3 * U)
    whole, w = whole.detach().abs(), weight.detach().abs()
    dx, dw = torch.zeros_like(whole), []
    for i in range(K):
        k = K - 1 - i
        dx[:, k:k + T] += torch.where(seen[i], du_off + du * (K + 1) * U, 0.0) * w[:, k]
        dw.append((torch.where(seen[i], whole[:, k:k + T], 0.0) * (du_off + du * (ADDITIONS + 2) * U)).sum((0, 1)))
    bounds = dx[:, K - 1:], torch.stack(dw[::-1], 1), (du_off + du * (ADDITIONS + 2) * U).sum((0, 1))
    out = out.detach()
    return out, 1.1 * u_off + out.abs() * (2 * size + 10) * U, grads, bounds


def _check_convolution(B, T, D, K, dtype, seed):
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import TYPES
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
    a = dict(x=n(B, T, D), weight=n(D, K), bias=n(D), starts=torch.rand((B, T), generator=g, device="cuda") < 0.02, state=n(B, K - 1, D),
             lengths=torch.randint(T // 2, T + 2, (B,), generator=g, device="cuda", dtype=torch.int32))
    grad = n(B, T, D)
    out, off, grads, bounds = _convolution(**a, grad=grad)
    _near("out", bps.causal_conv(**a).out, out, off)
    for name, got, want, bound in zip(("x", "weight", "bias"), bps.causal_conv_backward(grad, **a), grads, bounds):
        _near("grad " + name, got, want, bound)


@pytest.mark.parametrize("dtype,D,K", [("f32", 257, 4), ("f32", 261, 1), ("f32", 700, 8), ("bf16", 519, 4), ("f16", 1111, 3), ("bf16", 513, 5), ("bf16", 261, 6), ("f16", 300, 7), ("bf16", 1111, 8)])
@pytest.mark.parametrize("T", [3, 37])
def test_convolutions_of_more_channels_than_a_work_group_has(dtype, D, K, T):
    """Each thread has a part of its own; the last vectors begin inside the ones before."""
    _check_convolution(3, T, D, K, dtype, D + K)


@pytest.mark.parametrize("B,T,D,K,dtype", [(4, 4001, 1111, 4, "bf16"), (4, 4001, 1111, 7, "f16"), (3, 3307, 2051, 4, "f32"), (2, 16411, 2051, 4, "bf16"), (228, 3234, 14, 3, "bf16"), (1200, 515, 20, 4, "f32")])
def test_convolutions_in_long_runs_of_which_threads_have_several(B, T, D, K, dtype):
    """Runs of 16, 32, 32, 64, 8 and 16 steps, and more of them than there are threads for in the gradient."""
    _check_convolution(B, T, D, K, dtype, T)


# ---------------------------------------------------------------------------------------------- scan

def _sliced(a, grad, each):
    """Outputs, gradients and bounds by the definition, `each` sequences at a time: so many of them are as many additions of a sum as its
    bound allows."""
    import torch
    from memory_reference import cpu, scan, scan_bounds
    h = {k: cpu(v) for k, v in a.items()}
    h["soft"] = h.pop("softplus")
    joint = ("A", "D", "delta_bias")
    names = [k for k in ("x", "delta", "A", "B", "C", "D", "gate", "delta_bias") if h[k] is not None]
    parts, sums = [], {}
    for s in range(0, len(h["x"]), each):
        p = {k: v[s:s + each] if torch.is_tensor(v) and k not in joint else v for k, v in h.items()}
        g = cpu(grad)[s:s + each]
        bounds = scan_bounds(**p, grad_out=g)
        leaves = [p[k].clone().requires_grad_() for k in names]
        out, state = scan(**(p | dict(zip(names, leaves))))
        got = dict(zip(names, zip(torch.autograd.grad(out, leaves, g), (bounds[k].reshape(p[k].shape) for k in names))))
        parts.append(dict(out=(out.detach(), bounds["out"]), state=(state.detach(), bounds["state"])) | {"grad " + k: v for k, v in got.items() if k not in joint})
        for k in joint:
            if k in got:
                sums["grad " + k] = tuple(p + q for p, q in zip(sums["grad " + k], got[k])) if "grad " + k in sums else got[k]
    return {k: tuple(torch.cat(v) for v in zip(*(p[k] for p in parts))) for k in parts[0]} | sums


# work-groups of a tile of channels in the gradient: 256, 256, 2048, 256 and 341 -- sequences that each has: up to three, two, ...  Additions: of its
# sequences' steps, of a sixteenth of the work-groups and of 16 slices, under `each` times T
@pytest.mark.parametrize("batch,T,width,N,groups,dtype,each", [(600, 20, 200, 16, 1, "bf16", 8), (600, 17, 200, 32, 1, "f32", 8), (2500, 20, 20, 16, 1, "f16", 10), (700, 9, 256, 8, 2, "f32", 10),
                                                               (900, 5, 192, 3, 1, "bf16", 20)])
def test_scans_of_more_sequences_than_work_groups(batch, T, width, N, groups, dtype, each):
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import check
    from test_gpu_memory_scan import _backward, _inputs
    a, grad = _inputs(batch, T, width, N, dtype, batch + N, groups=groups, starts=0.05, ragged=True, state=True)
    assert (a["lengths"] <= 0).any() and (a["lengths"] >= T).any()
    r = bps.selective_scan(**a, hold=True)
    got = dict(out=r.out, state=r.state) | {"grad " + k: v for k, v in _backward(grad, a, r)._asdict().items()}
    for k, (want, bound) in _sliced(a, grad, each).items():
        check(k, got[k], want, bound)


@pytest.mark.parametrize("without", [(), ("D",), ("gate",), ("delta_bias",), ("state",), ("starts",), ("lengths",), ("D", "gate", "delta_bias", "state", "starts", "lengths")])
@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("dtype,N,groups,width", [("f32", 6, 1, 33), ("bf16", 16, 2, 300), ("f16", 32, 1, 257)])
def test_one_step_as_a_sequence(dtype, N, groups, width, softplus, without):
    """Without held states it is the kernel of single steps: sequences that have ended keep their states and give zero."""
    import torch
    import paper_2103_07013_amd as bps
    from memory_reference import check, cpu, scan, scan_bounds
    from test_gpu_memory_scan import _inputs
    a, _ = _inputs(7, 1, width, N, dtype, N, groups=groups, starts=0.4, state=True, softplus=softplus)
    a["lengths"] = torch.tensor([0, 1, 2, -1, 1, 0, 1], dtype=torch.int32, device="cuda")
    a["starts"][:3] = True
    for k in without:
        a[k] = None
    r = bps.selective_scan(**a)
    h = {k: cpu(v) for k, v in a.items()}
    h["soft"] = h.pop("softplus")
    out, state = scan(**h)
    bounds = scan_bounds(**h)
    check("out", r.out, out, bounds["out"])
    check("state", r.state, state, bounds["state"])
    if a["lengths"] is not None:
        assert (r.out[[0, 3, 5]] == 0).all()
        assert a["state"] is None or torch.equal(r.state[[0, 3, 5]], a["state"][[0, 3, 5]])


@pytest.mark.parametrize("dtype,N,groups", [("f32", 16, 1), ("bf16", 5, 2), ("f16", 32, 1)])
@pytest.mark.parametrize("T", [127, 128, 129, 191, 192, 193])
@pytest.mark.parametrize("kind", ["whole", "ragged", "episodes"])
def test_the_shortest_chunks(dtype, N, groups, T, kind):
    """A chunk has 64 steps at least: time is cut from 128 steps on."""
    from test_gpu_memory_scan import _check, _inputs
    a, g = _inputs(2, T, 66, N, dtype, T + N, groups=groups, starts=0.02 if kind == "episodes" else 0.0, ragged=kind == "ragged", state=True)
    _check(a, g)


# ---------------------------------------------------------------------------------------------- norms

@pytest.mark.parametrize("dtype,stream,rows,width", [("bf16", "f32", 600, 4104), ("f16", "f16", 530, 8192), ("f32", "f32", 300, 8193), ("bf16", "bf16", 300, 8201), ("f16", "f32", 270, 16384), ("f32", "f32", 270, 16384)])
def test_wide_rows_of_which_a_work_group_has_several(dtype, stream, rows, width):
    """256 work-groups share their gradient."""
    from test_gpu_memory_norm import _check, _inputs
    a, gr, go = _inputs((rows,), width, dtype, rows, stream)
    _check(a, gr, go, activation="silu")
