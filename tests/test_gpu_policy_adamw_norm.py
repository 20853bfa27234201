"""The bound on the gradient's norm where its square is no float32: a norm that is finite is used, and one that is not zero is found."""
import math

import pytest

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.mark.parametrize("size", [1e-36, 1e-30, 1e-21, 1e19, 1e25, 1e36])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_norms_of_any_size(size, dtype):
    """grad_norm within 4 e of the norm (squares and sums in 64 bits, rounded once), and a first step that goes by lr against each gradient's sign,
    bounded or not: m / sqrt(v) is 1 for any size of a gradient whose square is a float32, here 1e-6 after the bound."""
    import torch
    import paper_2103_07013_amd as bps
    kind = getattr(torch, dtype)
    p = [torch.zeros(n, dtype=kind, device="cuda") for n in (3, 5000, 70000)]
    g = [(torch.randint(0, 2, (len(q),), generator=torch.Generator().manual_seed(len(q))) * 2.0 - 1).mul(size).to(kind).cuda() for q in p]
    norm = math.sqrt(sum(float(x.double().square().sum()) for x in g))
    bound = 1e-6 * math.sqrt(75003) if size > 1e-6 else size / 4
    with bps.AdamW(p, lr=0.5, betas=(0.9, 0.99), eps=0.0, weight_decay=0.0, max_grad_norm=bound) as opt:
        opt.step(g)
        assert abs(float(opt.grad_norm) - norm) <= 4 * E * norm
        m = opt.exp_avg.double()
        taken = math.sqrt(float((m * 10).square().sum()))          # m = (1 - 0.9) g
        assert abs(taken - bound) <= 2.0 ** -10 * bound or bound < 1e-33      # (smaller ones lose bits as subnormal numbers)
        if size > 1e-6:
            for q, x in zip(p, g):
                assert torch.allclose(q.float(), -0.5 * x.float().sign(), rtol=1e-3)


def test_a_norm_that_no_float_holds_changes_nothing():
    """Gradients that are finite each, but not their norm."""
    import torch
    import paper_2103_07013_amd as bps
    p, g = [torch.ones(100, device="cuda")], [torch.full((100,), 3e38, device="cuda")]
    with bps.AdamW(p, max_grad_norm=1.0) as opt:
        opt.step(g)
        assert float(opt.grad_norm) == math.inf and (p[0] == 1).all() and int(torch.count_nonzero(opt.exp_avg)) == 0
