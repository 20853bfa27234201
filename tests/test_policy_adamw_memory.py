"""What AdamW makes of its public tensors when they are replaced: the plan holds the addresses that it was made with."""
import contextlib
import types

import pytest

NAMES = ["master", "exp_avg", "exp_avg_sq", "exp_avg_exponent", "exp_avg_sq_exponent", "grad_norm"]


@pytest.fixture
def on_host(monkeypatch):
    """AdamW over host tensors that pass for a GPU's, with a library that only counts its calls."""
    import torch
    from paper_2103_07013_amd import policy
    calls = []

    class OnDevice(torch.Tensor):
        is_cuda = True

    def called(name):
        return lambda *a: calls.append(name) or 0

    names = ("bps_adamw_create", "bps_adamw_destroy", "bps_adamw_step", "bps_adamw_read_states")
    monkeypatch.setattr(policy, "_library", lambda: types.SimpleNamespace(**{n: called(n) for n in names}))
    monkeypatch.setattr(policy, "_on", lambda index, call, *a: call(*a, None))
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())

    def make(dtype=torch.bfloat16, **kw):
        p = torch.ones(700, dtype=dtype).as_subclass(OnDevice)
        return policy.AdamW([p], **kw), [torch.ones(700, dtype=dtype).as_subclass(OnDevice)]

    return make, calls


@pytest.mark.parametrize("how", ["another", "none", "data"])
@pytest.mark.parametrize("name", NAMES)
def test_replaced_states_are_refused(on_host, name, how):
    make, calls = on_host
    opt, grads = make(state_bits=8)
    opt.step(grads)
    opt.states()
    assert calls.count("bps_adamw_step") == 1 and calls.count("bps_adamw_read_states") == 1 and opt.steps == 1
    t = getattr(opt, name)
    if how == "data":
        t.data = t.clone()
    else:
        setattr(opt, name, t.clone() if how == "another" else None)
    for call in (lambda: opt.step(grads), opt.states):
        with pytest.raises(ValueError, match=name):
            call()
    assert calls.count("bps_adamw_step") == 1 and calls.count("bps_adamw_read_states") == 1 and opt.steps == 1


def test_values_copied_into_the_states_are_taken(on_host):
    import torch
    make, calls = on_host
    for bits, dtype in ((8, torch.bfloat16), (32, torch.float32)):
        opt, grads = make(dtype, state_bits=bits)
        for name in NAMES:
            if getattr(opt, name) is not None:
                getattr(opt, name).copy_(getattr(opt, name).clone())
        opt.step(grads)
        m, v = opt.states()
        assert bits == 8 or (m is opt.exp_avg and v is opt.exp_avg_sq)
    assert calls.count("bps_adamw_step") == 2


@pytest.mark.gpu
def test_a_step_after_a_refusal():
    """A refused step changes nothing; the states put back, steps go on."""
    import torch
    import paper_2103_07013_amd as bps
    p, g = [torch.ones(1000, device="cuda")], [torch.ones(1000, device="cuda")]
    with bps.AdamW(p, lr=0.25, weight_decay=0.0) as opt:
        opt.step(g)
        kept, after = opt.exp_avg, p[0].clone()
        opt.exp_avg = kept.clone()
        with pytest.raises(ValueError, match="exp_avg"):
            opt.step(g)
        assert torch.equal(p[0], after) and opt.steps == 1
        opt.exp_avg = kept
        opt.step(g)
        # equal gradients: each step goes by lr
        assert torch.allclose(p[0], torch.full_like(p[0], 0.5), atol=1e-5) and opt.steps == 2


@pytest.mark.gpu
def test_parameters_that_share_memory():
    import torch
    import paper_2103_07013_amd as bps
    flat = torch.zeros(1000, device="cuda")
    for params in ([flat, flat], [flat[:600], flat[500:]], [flat[500:], flat, flat.clone()]):
        with pytest.raises(bps.BpsError, match="overlap"):
            bps.AdamW(params)
    with bps.AdamW([flat[500:], flat[:500]], lr=0.5, weight_decay=0.0) as opt:
        opt.step([torch.ones(500, device="cuda")] * 2)
        assert torch.allclose(flat, torch.full_like(flat, -0.5), atol=1e-5)


@pytest.mark.parametrize("failure", [TypeError, KeyboardInterrupt, "status"])
def test_a_step_that_fails_does_not_count(on_host, monkeypatch, failure):
    """Whatever ends the call: an argument of another kind (an lr that is no number, say), or the library's status."""
    import paper_2103_07013_amd as bps
    from paper_2103_07013_amd import policy
    make, calls = on_host
    opt, grads = make()
    opt.step(grads)
    working = policy._on

    def failing(*a):
        if failure == "status":
            return -1
        raise failure()

    monkeypatch.setattr(policy, "_on", failing)
    monkeypatch.setattr(policy, "bps_last_error", lambda: "")
    with pytest.raises(bps.BpsError if failure == "status" else failure):
        opt.step(grads)
    assert opt.steps == 1
    monkeypatch.setattr(policy, "_on", working)
    opt.step(grads)
    assert opt.steps == 2
