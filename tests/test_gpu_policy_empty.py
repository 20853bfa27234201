"""Batches without a row, whatever their other dimensions."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(0,), (2, 0), (0, 3), (3, 0, 5), (4, 2, 0), (0, 0)])
@pytest.mark.parametrize("k", [0, 3])
def test_scores(shape, k):
    import torch
    import paper_2103_07013_amd as bps
    logits, tokens = torch.zeros((*shape, 7), device="cuda"), torch.zeros(shape, dtype=torch.int64, device="cuda")
    mask = torch.ones((*shape, 7), dtype=torch.bool, device="cuda")
    r = bps.log_probs(logits, tokens, mask=mask, top_k=k)
    assert r.logp.shape == r.entropy.shape == r.lse.shape == shape and (not k or r.top_ids.shape == r.top_logp.shape == (*shape, k))
    assert bps.log_probs_backward(logits, tokens, r, r.logp, r.entropy, mask=mask).shape == (*shape, 7)
    assert bps.log_probs_backward(logits, tokens, r, out=logits) is logits
    x = logits.requires_grad_()
    bps.log_probs(x, tokens).logp.sum().backward()
    assert x.grad.shape == (*shape, 7)
    # of strides that no list of rows has
    views = torch.zeros((3, *shape, 7), device="cuda").transpose(0, 1)[:, 0] if len(shape) > 1 else logits.detach()
    assert bps.log_probs(views, torch.zeros(views.shape[:-1], dtype=torch.int64, device="cuda")).logp.numel() == 0


@pytest.mark.parametrize("shape", [(0,), (2, 0), (3, 0, 5)])
def test_embedding(shape):
    import torch
    import paper_2103_07013_amd as bps
    w, tokens = torch.ones((9, 4), device="cuda", requires_grad=True), torch.zeros(shape, dtype=torch.int32, device="cuda")
    out = bps.embedding(tokens, w)
    assert out.shape == (*shape, 4)
    out.sum().backward()
    assert torch.equal(w.grad, torch.zeros((9, 4), device="cuda"))
    given = torch.empty((*shape, 4), device="cuda")
    assert bps.embedding(tokens, w, out=given) is given
    assert (bps.embedding_backward(tokens, given, 9, out=torch.ones((9, 4), device="cuda")) == 0).all()
