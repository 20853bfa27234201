"""Calls of more rows than one launch takes: 2^21 rows of scores, fewer of their gradient where rows are long, 2^22 rows of a lookup."""
import math

import pytest

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.mark.parametrize("left,k", [(1, 0), (37, 3)])
def test_scores_of_long_rows(left, k):
    """The same row for all.  Its tokens' log probabilities are off by at most e (8 |value| + 16 ln V + 64 + V / 128), as other rows' are."""
    import torch
    import paper_2103_07013_amd as bps
    N, V = 2 ** 21 + left, 40000
    row = (torch.randn(V, generator=torch.Generator().manual_seed(left)) * 3).bfloat16()
    tokens = torch.arange(N, device="cuda") % V
    r = bps.log_probs(row.cuda().expand(N, V), tokens, top_k=k)
    y = row.double()
    lp = y - torch.logsumexp(y, 0)
    slack = E * (8 * lp.abs() + 16 * math.log(V) + 64 + V / 128)
    assert ((r.logp.cpu().double() - lp[tokens.cpu()]).abs() <= slack[tokens.cpu()]).all()
    entropy = -(lp.exp() * lp).sum()
    assert ((r.entropy.cpu().double() - entropy).abs() <= 2 * E * (8 * entropy + 16 * math.log(V) + 64 + V / 128)).all()
    if k:
        best = row.float().sort(descending=True, stable=True).indices[:k].to(torch.int32)
        assert (r.top_ids.cpu() == best).all()
        assert ((r.top_logp.cpu().double() - lp[best.long()]).abs() <= slack[best.long()]).all()


@pytest.mark.parametrize("N,V", [(2 ** 21 + 37, 3), (2 ** 21 + 1, 40)])
def test_scores_of_short_rows_and_their_gradient(N, V):
    """Rows on both sides of the split have the bits that they have in a call of their own."""
    import torch
    import paper_2103_07013_amd as bps
    g = torch.Generator(device="cuda").manual_seed(V)
    logits = torch.randn((N, V), generator=g, device="cuda")
    mask = torch.rand((N, V), generator=g, device="cuda") < 0.8
    tokens = torch.randint(-1, V, (N,), generator=g, device="cuda")
    gl, gh = torch.randn((2, N), generator=g, device="cuda").unbind(0)
    r = bps.log_probs(logits, tokens, mask=mask, top_k=2)
    dx = bps.log_probs_backward(logits, tokens, r, gl, gh, mask=mask)
    for first in (0, 2 ** 21 - 500, N - 20):
        at = slice(first, first + 1000)
        s = bps.log_probs(logits[at], tokens[at], mask=mask[at], top_k=2)
        assert all(torch.equal(a[at], b) for a, b in zip(r[:5], s[:5]))
        assert torch.equal(dx[at], bps.log_probs_backward(logits[at], tokens[at], s, gl[at], gh[at], mask=mask[at]))


def test_gradient_of_long_rows():
    """Rows of 8193 entries are split from 2^21 / 3 on."""
    import torch
    import paper_2103_07013_amd as bps
    split, V = 2 ** 21 // 3, 8193
    N = split + 40
    g = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn((1000, V), generator=g, device="cuda").bfloat16().repeat(N // 1000 + 1, 1)[:N]
    tokens = torch.arange(N, device="cuda") % V
    gl, gh = torch.randn((2, N), generator=g, device="cuda").unbind(0)
    r = bps.log_probs(logits, tokens)
    dx = bps.log_probs_backward(logits, tokens, r, gl, gh)
    for first in (0, 20, 39, split - 1, split, N - 1):      # the split is at the front: the last rows come first
        at = slice(first, first + 1)
        assert torch.equal(dx[at], bps.log_probs_backward(logits[at], tokens[at], r.held[:, at].contiguous(), gl[at], gh[at]))


def test_lookup():
    import torch
    import paper_2103_07013_amd as bps
    N = 2 ** 22 + 5
    w = torch.randn((7, 2), generator=torch.Generator().manual_seed(1)).cuda()
    t = torch.arange(N, device="cuda", dtype=torch.int32) % 8 - 1
    assert torch.equal(bps.embedding(t, w, scale=3.0), torch.where((t < 0)[:, None], 0.0, w[t.long().clamp(min=0)] * 3.0))
