"""Gradients of tables of few rows that are wider than one launch's columns."""
import pytest

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.mark.parametrize("dtype,rows,extra", [("float32", 3, 5), ("bfloat16", 8, 1), ("float32", 1, 2 ** 22)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(rows, extra, dtype, accumulate):
    import torch
    import paper_2103_07013_amd as bps
    width, count = 2 ** 22 + extra, 20
    g = torch.Generator(device="cuda").manual_seed(rows)
    grad = torch.randn((count, width), generator=g, device="cuda").to(getattr(torch, dtype))
    tokens = torch.randint(-1, rows, (count,), generator=g, device="cuda")
    out = torch.randn((rows, width), generator=g, device="cuda")
    before = out.double() if accumulate else torch.zeros((rows, width), dtype=torch.float64, device="cuda")
    got = bps.embedding_backward(tokens, grad, rows, scale=0.5, out=out, accumulate=accumulate)
    ref, size = before, torch.zeros_like(before)
    for n, t in enumerate(tokens.tolist()):
        if t >= 0:
            ref[t] += 0.5 * grad[n].double()
            size[t] += 0.5 * grad[n].double().abs()
    assert ((got.double() - ref).abs() <= (count + 2) * E * size + E * ref.abs()).all()
