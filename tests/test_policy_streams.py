"""Which stream the policy's operators take a `stream` argument for."""
import pytest


def test_handle_zero_is_the_default_stream(monkeypatch):
    """The raw handle of the default stream is 0, which torch's ExternalStream takes for none given (and makes a stream of its own)."""
    import torch
    from paper_2103_07013_amd import policy
    device = torch.device("cuda", 0)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: ("default", device))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: ("external", handle, device))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: s)
    assert policy._stream(0, device) == ("default", device)
    assert policy._stream(4096, device) == ("external", 4096, device)


@pytest.mark.gpu
def test_calls_on_the_default_stream():
    """A call on the default stream by its handle is in order with the default stream's own work before and behind it, from another stream too."""
    import torch
    import paper_2103_07013_amd as bps
    from paper_2103_07013_amd import policy
    handle = torch.cuda.default_stream().cuda_stream
    assert handle == 0
    side = torch.cuda.Stream()
    with torch.cuda.stream(side), policy._stream(handle, torch.device("cuda", 0)):
        assert torch.cuda.current_stream() == torch.cuda.default_stream()
    logits, tokens, w = torch.zeros((2048, 5000), device="cuda"), torch.arange(2048, device="cuda"), torch.zeros((2048, 64), device="cuda")
    g = torch.ones((2048, 64), device="cuda")
    p, grads = [torch.zeros(1000, device="cuda")], [torch.ones(1000, device="cuda")]
    opt = bps.AdamW(p, lr=0.5, weight_decay=0.0)
    torch.cuda.synchronize()
    for k in range(1, 6):
        logits.fill_(0.0)
        logits[:, 0] = float(k)
        w.fill_(float(k))
        g.fill_(float(k))
        with torch.cuda.stream(side):
            r = bps.log_probs(logits, tokens, stream=handle)
            dx = bps.log_probs_backward(logits, tokens, r, r.lse, stream=handle)
            rows = bps.embedding(tokens, w, stream=handle)
            dw = bps.embedding_backward(tokens, g, 2048, stream=handle)
            opt.step(grads, stream=handle)
            opt.states(stream=handle)
        logits.fill_(-7.0)
        w.fill_(-7.0)
        g.fill_(-7.0)
        torch.cuda.synchronize()
        x = torch.zeros((1, 5000), dtype=torch.float64)
        x[0, 0] = k
        assert torch.allclose(r.lse.cpu().double(), torch.logsumexp(x, 1), rtol=1e-5)
        assert torch.isfinite(dx).all() and (rows == k).all() and (dw == k).all()
    opt.close()


def test_a_stream_of_another_device_is_refused(monkeypatch):
    """Made current, it would be another device's stream, and the call would run on this one's, unordered with it."""
    import types
    import torch
    from paper_2103_07013_amd import policy
    monkeypatch.setattr(torch.cuda, "stream", lambda s: s)
    here, there = (types.SimpleNamespace(device=torch.device("cuda", k)) for k in range(2))
    assert policy._stream(here, torch.device("cuda", 0)) is here
    with pytest.raises(ValueError, match="stream"):
        policy._stream(there, torch.device("cuda", 0))
