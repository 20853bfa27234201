"""Refusals of the policy's operators: the C interface checks its arguments before it touches a device, with a status and a
text; the Python layer refuses tensors that do not fit before anything is read."""
import ctypes

import pytest


def _lib():
    from paper_2103_07013_amd import policy
    return policy._library()


def _text():
    import paper_2103_07013_amd as bps
    return bps.bps_last_error()


P = 4096          # an address that no check may look behind


def _scores(**kw):
    a = dict(logits=P, dtype=0, rows=2, entries=5, stride=5, tokens=P, bits=32, mask=None, mask_stride=0, scale=1.0, k=0, logp=P, entropy=P, lse=P, norm=P, ids=None, top=None, space=None,
             size=0, stream=None)
    a.update(kw)
    return _lib().bps_log_probs(*a.values())


@pytest.mark.parametrize("wrong,text", [(dict(logits=None), "null"), (dict(tokens=None), "null"), (dict(logp=None), "null"), (dict(entropy=None), "null"), (dict(lse=None), "null"), (dict(norm=None), "null"),
                                        (dict(dtype=3), "element type"), (dict(dtype=-1), "element type"), (dict(bits=16), "tokens of 16 bits"), (dict(entries=0), "entries"),
                                        (dict(entries=1 << 30), "entries"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"),
                                        (dict(scale=float("inf")), "scale"), (dict(k=65, ids=P, top=P), "top_k"), (dict(k=2), "top_ids"), (dict(k=2, ids=P), "top_ids"),
                                        (dict(logits=P + 2), "misaligned"), (dict(tokens=P + 4, bits=64), "misaligned"), (dict(logits=P + 1, dtype=1), "misaligned")])
def test_scores_refuse(wrong, text):
    assert _scores(**wrong) == -1 and text in _text()


def test_scores_of_no_rows_do_nothing():
    assert _scores(rows=0, logits=None, tokens=None, logp=None) == 0


def test_scores_refuse_too_little_workspace():
    lib = _lib()
    need = lib.bps_log_probs_workspace(1, 1, 131072, 20)
    if need:
        for kw in (dict(space=None, size=need), dict(space=P, size=need - 1), dict(space=P + 8, size=need)):
            assert _scores(dtype=1, rows=1, entries=131072, stride=131072, k=20, ids=P, top=P, **kw) == -1 and "workspace" in _text()
    assert lib.bps_log_probs_workspace(9, 1, 5, 0) == 0


def _scores_back(**kw):
    a = dict(logits=P, dtype=0, rows=2, entries=5, stride=5, tokens=P, bits=32, mask=None, mask_stride=0, scale=1.0, logp=P, entropy=P, norm=P, gl=None, gh=None, out=P, out_stride=5,
             stream=None)
    a.update(kw)
    return _lib().bps_log_probs_backward(*a.values())


@pytest.mark.parametrize("wrong,text", [(dict(out=None), "null"), (dict(norm=None), "null"), (dict(dtype=7), "element type"), (dict(out_stride=4), "overlap"), (dict(out_stride=0), "overlap"),
                                        (dict(out_stride=-4), "overlap"), (dict(out=P + 2), "misaligned"), (dict(scale=0.0), "scale")])
def test_gradient_of_scores_refuses(wrong, text):
    assert _scores_back(**wrong) == -1 and text in _text()


def _lookup(**kw):
    a = dict(tokens=P, bits=64, count=3, weight=P, dtype=2, rows=4, width=8, stride=8, scale=1.0, out=P, out_stride=8, stream=None)
    a.update(kw)
    return _lib().bps_embedding(*a.values())


@pytest.mark.parametrize("wrong,text", [(dict(tokens=None), "null"), (dict(weight=None), "null"), (dict(out=None), "null"), (dict(dtype=5), "element type"), (dict(bits=8), "tokens of 8 bits"),
                                        (dict(rows=0), "rows"), (dict(width=0), "width"), (dict(out_stride=7), "overlap"), (dict(weight=P + 1), "misaligned"), (dict(count=1 << 41), "count")])
def test_lookup_refuses(wrong, text):
    assert _lookup(**wrong) == -1 and text in _text()


def _lookup_back(**kw):
    a = dict(tokens=P, bits=64, count=3, grad=P, dtype=2, rows=4, width=8, stride=8, scale=1.0, out=P, to=0, out_stride=8, accumulate=0, space=P, size=1 << 20, stream=None)
    a.update(kw)
    return _lib().bps_embedding_backward(*a.values())


@pytest.mark.parametrize("wrong,text", [(dict(tokens=None), "null"), (dict(grad=None), "null"), (dict(out=None), "null"), (dict(dtype=5), "element type"), (dict(to=5), "element type"),
                                        (dict(bits=0), "tokens of 0 bits"), (dict(rows=0), "rows"), (dict(rows=1 << 30), "rows"), (dict(out_stride=7), "overlap"), (dict(out=P + 2), "misaligned"),
                                        (dict(count=1 << 31), "count"), (dict(size=15), "workspace"), (dict(space=None), "workspace"), (dict(space=P + 4), "workspace")])
def test_gradient_of_lookup_refuses(wrong, text):
    assert _lookup_back(**wrong) == -1 and text in _text()


def _plan(table=((P, None, 10, 0), (P, None, 300, 256)), **kw):
    from paper_2103_07013_amd import policy
    n = len(table)
    table = (policy._Tensor * n)(*(policy._Tensor(p, m, n, a, 0.0, 1.0) for p, m, n, a in table))
    a = dict(param_dtype=0, state_bits=32, tensors=n, seed=0, total=768, tensor=table, exp_avg=P, exp_avg_sq=P, exp_avg_exponent=None, exp_avg_sq_exponent=None)
    a.update(kw)
    out = ctypes.c_void_p()
    status = _lib().bps_adamw_create(ctypes.byref(policy._Config(*a.values())), ctypes.byref(out))
    assert status != 0 and out.value is None
    return status


@pytest.mark.parametrize("wrong,text", [(dict(param_dtype=4), "element type"), (dict(state_bits=16), "state_bits"), (dict(tensors=0), "no tensors"), (dict(exp_avg=None), "null state"),
                                        (dict(state_bits=8), "null state"), (dict(exp_avg=P + 4), "16-byte"), (dict(total=700), "multiple"), (dict(total=512), "not inside"),
                                        (dict(param_dtype=1), "master"), (dict(table=((P, P, 10, 0),)), "master"), (dict(table=((P, None, 0, 0),)), "empty"),
                                        (dict(table=((None, None, 5, 0),)), "empty"), (dict(table=((P + 2, None, 5, 0),)), "misaligned"), (dict(table=((P, None, 5, 100),)), "start at 100"),
                                        (dict(table=((P, None, 300, 0), (P, None, 5, 256))), "start at 256"), (dict(table=((P, None, 5, 1 << 40),)), "not inside"),
                                        (dict(table=((P, None, 2 ** 64 - 1, 0),)), "not inside")])
def test_plan_refuses(wrong, text):
    assert _plan(**wrong) == -1 and text in _text()


def test_plan_needs_a_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert _plan() == -4 and "no CPU path" in _text()


def test_null_handles():
    lib = _lib()
    lib.bps_adamw_destroy(None)
    assert lib.bps_adamw_step(None, None, 0, 1, 0.1, 0.9, 0.99, 1e-8, 1.0, 0.0, None, None) == -1 and "null" in _text()
    assert lib.bps_adamw_read_states(None, None, None, None) == -1


def test_python_refuses_tensors_of_the_host():
    import torch
    import paper_2103_07013_amd as bps
    x, t = torch.zeros((2, 3)), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError):
        bps.log_probs(x, t)
    with pytest.raises(ValueError):
        bps.embedding(t, x)
    with pytest.raises(ValueError):
        bps.embedding_backward(t, x, 4)
    with pytest.raises(ValueError):
        bps.AdamW([x])
    with pytest.raises(ValueError):
        bps.AdamW([])


@pytest.mark.gpu
def test_python_refuses_what_does_not_fit():
    import torch
    import paper_2103_07013_amd as bps
    x, t = torch.zeros((4, 6), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    r = bps.log_probs(x, t)
    for call in (lambda: bps.log_probs(x.double(), t), lambda: bps.log_probs(x, t.short()), lambda: bps.log_probs(x, t[:3]), lambda: bps.log_probs(x, t.cpu()),
                 lambda: bps.log_probs(x.t(), torch.zeros(6, dtype=torch.int64, device="cuda")), lambda: bps.log_probs(x, t, mask=torch.ones((4, 5), dtype=torch.bool, device="cuda")),
                 lambda: bps.log_probs(x, t, mask=torch.ones((4, 6), device="cuda")), lambda: bps.log_probs(x, t, mask=torch.ones((6, 4), dtype=torch.bool, device="cuda").t()),
                 lambda: bps.log_probs(x, t, top_k=65), lambda: bps.log_probs(x, t, top_k=-1), lambda: bps.log_probs(x[:, :0], t),
                 lambda: bps.log_probs(torch.zeros((2, 3, 2, 5), device="cuda").transpose(0, 1), torch.zeros((3, 2, 2), dtype=torch.int64, device="cuda")),
                 lambda: bps.log_probs_backward(x, t, r, torch.ones(3, device="cuda")), lambda: bps.log_probs_backward(x, t, r, torch.ones(4, device="cuda").double()),
                 lambda: bps.log_probs_backward(x, t, r, out=x.half()), lambda: bps.log_probs_backward(x, t, r, out=x[:3]),
                 lambda: bps.embedding(t.float(), x), lambda: bps.embedding(t, x[0]), lambda: bps.embedding(t, x, out=torch.zeros((4, 5), device="cuda")),
                 lambda: bps.embedding(torch.zeros((4, 2), dtype=torch.int64, device="cuda")[:, 0], x),
                 lambda: bps.embedding_backward(t[:3], x, 9), lambda: bps.embedding_backward(t, x, 9, accumulate=True), lambda: bps.embedding_backward(t, x, 9, dtype=torch.float64),
                 lambda: bps.embedding_backward(t, x, 9, out=torch.zeros((8, 6), device="cuda")),
                 lambda: bps.AdamW([x, x.half()]), lambda: bps.AdamW([x.t()]), lambda: bps.AdamW([x], state_bits=4), lambda: bps.AdamW([x], weight_decay=[0.1, 0.2])):
        with pytest.raises(ValueError):
            call()
    for scale in (0.0, -1.0, float("nan")):
        with pytest.raises(bps.BpsError) as e:
            bps.log_probs(x, t, scale=scale)
        assert e.value.status == -1
    with bps.AdamW([x], max_grad_norm=1.0) as opt:
        for g in ([x, x], [x.half()], [x[:3]], [torch.zeros((6, 4), device="cuda").t()], [x.cpu()]):
            with pytest.raises(ValueError):
                opt.step(g)
        for name, value in (("lr", float("nan")), ("betas", (1.0, 0.9)), ("betas", (0.9, -0.1)), ("eps", -1.0), ("max_grad_norm", float("inf"))):
            held = getattr(opt, name)
            setattr(opt, name, value)
            with pytest.raises(bps.BpsError) as e:
                opt.step([x])
            assert e.value.status == -1 and opt.steps == 0
            setattr(opt, name, held)
    with pytest.raises(ValueError):
        opt.step([x])
