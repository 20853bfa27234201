"""What a policy trained on the renderer's frames asks of its operators, as a list of cases that can be timed.

A step of such a policy embeds the previous action (or token), scores the one it takes, and learns from both:

  "score"   log probabilities of given tokens with the entropy and the best alternatives (rollout, serving)
  "learn"   the same and the gradient of both with respect to the logits (one update)
  "lookup"  rows of an embedding, scaled (rollout)
  "embed"   the same and the gradient of the table (one update)
  "adamw"   one AdamW step over all tensors of a policy, its states held in 32 or in 8 bits

`run` computes the plain forms in float32 torch operations, or makes the framework's calls where `own` is true.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
#: states of one parameter tensor start at a multiple of this, and so many 8-bit states share an exponent
_BLOCK = 256
#: the dither of 8-bit states: odd integers next to 2^32 times the fractional parts of the golden ratio, sqrt 2 and sqrt 3
_GOLDEN, _ROOT2, _ROOT3 = 0x9E3779B9, 0x6A09E667, 0xBB67AE85
_ADAMW = dict(lr=2.5e-4, betas=(0.9, 0.999), eps=1e-5, weight_decay=0.01)


def listed():
    return [
        # one rollout step: 1024 environments choose among four moves
        dict(name="score_actions", op="score", N=1024, V=4, dtype="f32", mask="none", top_k=0, scale=1.0),
        # one update of that policy: 32 steps of 1024 environments, some moves not allowed, some environments finished
        dict(name="learn_actions", op="learn", N=32768, V=6, dtype="f32", mask="rows", scale=1.0),
        # one token of one answer is scored, with the alternatives shown to a user
        dict(name="score_token", op="score", N=1, V=131072, dtype="bf16", mask="none", top_k=20, scale=1.0),
        # a batch of requests, each at a token of its own, with forbidden tokens and an odd vocabulary
        dict(name="score_batch", op="score", N=192, V=50257, dtype="f16", mask="shared", top_k=5, scale=1.25),
        # an update over whole sequences, the largest logits that are held at once
        dict(name="learn_tokens", op="learn", N=8192, V=131072, dtype="bf16", mask="none", scale=1.0),
        # the previous action of every environment
        dict(name="lookup_actions", op="lookup", N=1024, V=5, D=32, dtype="f32", scale=1.0),
        # its table's gradient over an update: few rows, each used thousands of times
        dict(name="embed_actions", op="embed", N=32768, V=5, D=32, dtype="f32", scale=1.0),
        # a small vocabulary of odd sizes
        dict(name="embed_tokens", op="embed", N=16384, V=50257, D=769, dtype="bf16", scale=27.7),
        # a large vocabulary and a long batch
        dict(name="embed_large", op="embed", N=262144, V=131072, D=2048, dtype="bf16", scale=1.0),
        # the policy of the rollouts above: many small tensors, bounded gradient
        dict(name="adamw_policy", op="adamw", T=38, P=5_300_000, dtype="f32", bits=32, clip=1.0),
        # 16-bit weights with 32-bit masters, states in 8 bits
        dict(name="adamw_8bit", op="adamw", T=30, P=120_000_000, dtype="bf16", bits=8, clip=0.0),
        # a model that fills a good part of a step by itself
        dict(name="adamw_large", op="adamw", T=24, P=400_000_000, dtype="f32", bits=32, clip=0.0),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["score", "learn", "lookup", "embed", "adamw"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op in ("score", "learn"):
        V = _log_int(rng, 2, 150_000)
        N = _log_int(rng, 1, max(1, min(65536, 400_000_000 // V)))
        case = dict(op=op, N=N, V=V, dtype=dtype, mask=rng.choice(["none", "shared", "rows"]), scale=rng.choice([1.0, 1.0, 0.7, 1.25]))
        if op == "score":
            case["top_k"] = rng.choice([0, 1, 5, 20, 64])
        return case
    if op in ("lookup", "embed"):
        V = _log_int(rng, 2, 150_000)
        D = _log_int(rng, 8, 2800)
        N = _log_int(rng, 1, max(1, min(400_000, 500_000_000 // D)))
        while V * D > 300_000_000:
            V //= 2
        return dict(op=op, N=N, V=V, D=D, dtype=dtype, scale=rng.choice([1.0, math.sqrt(D)]))
    T = _log_int(rng, 1, 40)
    return dict(op=op, T=T, P=_log_int(rng, 20_000, 200_000_000), dtype=dtype, bits=rng.choice([32, 8]), clip=0.0)


def _sizes(case):
    """Elements of each of the T tensors of about P elements in all: biases next to matrices, few of them round."""
    rng = np.random.RandomState(case["T"] * 7919 + case["P"] % 104729)
    share = np.exp(rng.uniform(-3.0, 3.0, case["T"]))
    share[rng.rand(case["T"]) < 0.3] *= 1e-3
    share[0] = max(share[0], 1.0)
    return [max(1, int(s)) for s in share / share.sum() * case["P"]]


def _layout(sizes):
    """Where each tensor's states start, and how many there are in all, in whole blocks."""
    ends = np.cumsum([-(-n // _BLOCK) * _BLOCK for n in sizes])
    return [0] + [int(e) for e in ends[:-1]], int(ends[-1])


def _tokens(g, N, V, none):
    """Token numbers as they are used: few of them often, most of them seldom; a share of `none` is -1."""
    t = (float(V) ** torch.rand(N, generator=g, device="cuda", dtype=torch.float64)).long() - 1
    t = (t.clamp(0, V - 1) * 7 + 3) % V if V % 7 else t.clamp(0, V - 1)
    return torch.where(torch.rand(N, generator=g, device="cuda") < none, -1, t).to(torch.int32)


def _normal(g, shape, dtype, size=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * size).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)
    op, dtype = case["op"], _TYPES[case["dtype"]]
    s = dict(op=op)
    if op in ("score", "learn"):
        N, V = case["N"], case["V"]
        s["logits"] = torch.empty((N, V), dtype=dtype, device="cuda")
        step = max(1, 200_000_000 // V)
        for i in range(0, N, step):  # a few standard deviations, as a trained policy's are
            s["logits"][i:i + step] = _normal(g, (min(step, N - i), V), dtype, 3.0)
        s["tokens"] = _tokens(g, N, V, 0.02 if op == "learn" else 0.0)
        s["mask"] = None
        if case["mask"] == "shared":
            s["mask"] = torch.rand(V, generator=g, device="cuda") < 0.9
        elif case["mask"] == "rows":
            s["mask"] = (torch.rand((N, V), generator=g, device="cuda") < 0.8) & (torch.rand((N, 1), generator=g, device="cuda") > 0.01)
        s["scale"] = case["scale"]
        s["top_k"] = min(case.get("top_k", 0), V)
        if op == "learn":
            s["grad_logp"] = _normal(g, (N,), torch.float32)
            s["grad_entropy"] = _normal(g, (N,), torch.float32, 0.1)
    elif op in ("lookup", "embed"):
        N, V, D = case["N"], case["V"], case["D"]
        s["tokens"] = _tokens(g, N, V, 0.01)
        s["weight"] = _normal(g, (V, D), dtype, 0.02)
        s["scale"] = case["scale"]
        if op == "embed":
            s["grad_out"] = _normal(g, (N, D), dtype)
    else:
        sizes = _sizes(case)
        starts, total = _layout(sizes)
        s |= dict(sizes=sizes, starts=starts, total=total, bits=case["bits"], clip=case["clip"], step=1000, seed=int(seed) & 0xFFFF)
        master = [_normal(g, (n,), torch.float32, 0.05) for n in sizes]
        s["params"] = [w.to(dtype) for w in master]
        s["grads"] = [_normal(g, (n,), dtype, 0.01) for n in sizes]
        s["master"] = None if case["dtype"] == "f32" else _flat(master, total)
        del master
        inside = _flat([torch.ones(n, dtype=torch.bool, device="cuda") for n in sizes], total)
        if case["bits"] == 32:
            s["exp_avg"] = _normal(g, (total,), torch.float32, 0.003) * inside
            s["exp_avg_sq"] = _normal(g, (total,), torch.float32, 0.01).square() * inside
        else:  # codes and exponents as earlier steps leave them: most values within a few powers of two of the largest
            s["exp_avg"] = (torch.randint(72, 126, (total,), generator=g, device="cuda", dtype=torch.uint8)
                            + torch.randint(0, 2, (total,), generator=g, device="cuda", dtype=torch.uint8) * 128) * inside
            s["exp_avg_sq"] = torch.randint(160, 250, (total,), generator=g, device="cuda", dtype=torch.uint8) * inside
            s["exp_avg_exponent"] = torch.randint(118, 121, (total // _BLOCK,), generator=g, device="cuda", dtype=torch.uint8)
            s["exp_avg_sq_exponent"] = torch.randint(112, 116, (total // _BLOCK,), generator=g, device="cuda", dtype=torch.uint8)
    if own:
        import paper_2103_07013_amd as bps
        s["bps"] = bps
        if op == "adamw":
            opt = bps.AdamW(s["params"], **_ADAMW, state_bits=s["bits"], max_grad_norm=s["clip"], seed=s["seed"])
            opt.steps = s["step"]
            for name in ("master", "exp_avg", "exp_avg_sq", "exp_avg_exponent", "exp_avg_sq_exponent"):
                if s.get(name) is not None:
                    getattr(opt, name).copy_(s.pop(name))
            s["opt"] = opt
    return s


def run(s):
    return (_own if own else _plain)[s["op"]](s)


# ---------------------------------------------------------------------------------------------- plain forms

def _scores(s):
    """(logits taking part, or -inf; log of the sum; log probabilities of all; entropy; log probability of the token)"""
    x = s["logits"].float()
    if s["mask"] is not None:
        x = torch.where(s["mask"], x, -math.inf)
    y = x * s["scale"]
    top = y.amax(1, keepdim=True)
    empty = top == -math.inf
    top = torch.where(empty, 0.0, top)
    lse = top + (y - top).exp().sum(1, keepdim=True).log()
    lp = torch.where(y == -math.inf, -math.inf, y - torch.where(empty, 0.0, lse))
    entropy = -torch.where(lp == -math.inf, 0.0, lp.exp() * lp).sum(1)
    t = s["tokens"].long()
    logp = torch.where(t < 0, 0.0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0])
    return x, lse[:, 0], lp, entropy, logp


def _plain_score(s):
    x, lse, lp, entropy, logp = _scores(s)
    out = dict(logp=logp, entropy=entropy, lse=lse)
    if s["top_k"]:
        best, ids = x.sort(dim=1, descending=True, stable=True)
        best, ids = best[:, :s["top_k"]], ids[:, :s["top_k"]]
        out["top_ids"] = torch.where(best == -math.inf, -1, ids).to(torch.int32)
        out["top_logp"] = lp.gather(1, ids)
    return out


def _plain_learn(s):
    _, lse, lp, entropy, logp = _scores(s)
    t = s["tokens"].long()
    gl = torch.where((t < 0) | (logp == -math.inf), 0.0, s["grad_logp"])[:, None]
    gh = s["grad_entropy"][:, None]
    grad = torch.where(lp == -math.inf, 0.0, -lp.exp() * (gl + gh * (lp + entropy[:, None])))
    grad.scatter_add_(1, t.clamp(min=0)[:, None], gl)
    return dict(logp=logp, entropy=entropy, lse=lse, grad_logits=(grad * s["scale"]).to(s["logits"].dtype))


def _plain_lookup(s):
    t = s["tokens"].long()
    rows = s["weight"][t.clamp(min=0)].float() * s["scale"]
    return dict(out=torch.where(t[:, None] < 0, 0.0, rows).to(s["weight"].dtype))


def _plain_embed(s):
    t = s["tokens"].long()
    grad = torch.zeros(s["weight"].shape, dtype=torch.float32, device="cuda")
    grad.index_add_(0, t.clamp(min=0), torch.where(t[:, None] < 0, 0.0, s["grad_out"].float()))
    return dict(_plain_lookup(s), grad_weight=grad * s["scale"])


def _flat(tensors, total):
    """Tensors one after the other, each in whole blocks."""
    flat = torch.cat([torch.nn.functional.pad(t.reshape(-1), (0, -t.numel() % _BLOCK)) for t in tensors])
    return flat[:total]


def _mixed(h):
    """32 bits of which each depends on all bits of h (a tensor of whole numbers, or one)."""
    h = h & 0xFFFFFFFF
    h = ((h ^ (h >> 16)) * _ROOT2) & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) * _ROOT3) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _power(biased):
    """2^(biased - 127) in float32"""
    return (biased << 23).to(torch.int32).view(torch.float32)


def _decoded(codes, exponents, top):
    """8-bit floating point numbers of 3 mantissa bits, the largest exponent `top` standing for the block's own."""
    c = codes.view(-1, _BLOCK).int()
    field = (c >> 3).clamp(min=1)
    return ((c - (field - 1) * 8).float() * _power(exponents.int()[:, None] - top + field - 3)).view(-1)


def _encoded(x, top, least, dither):
    """(codes, exponents) of x >= 0: rounded up or down with probabilities that leave the mean where it was."""
    x = x.view(-1, _BLOCK)
    bits = x.view(torch.int32)
    e = ((bits.amax(1, keepdim=True) + 0x0FFFFF) >> 23).clamp(min=least)
    field = ((bits >> 23) - e + top).clamp(min=1)
    n = (x * _power(254 - (e - top + field - 3)) + dither.view(-1, _BLOCK)).floor().int()
    return ((field - 1) * 8 + n).to(torch.uint8).view(-1), e[:, 0].to(torch.uint8)


def _plain_adamw(s):
    (b1, b2), lr, eps, wd = _ADAMW["betas"], _ADAMW["lr"], _ADAMW["eps"], _ADAMW["weight_decay"]
    s["step"] += 1
    g = _flat(s["grads"], s["total"]).float()
    out = {}
    if s["clip"]:
        out["grad_norm"] = (g * g).sum().sqrt().reshape(1)
        g = g * torch.where(out["grad_norm"] > s["clip"], s["clip"] / out["grad_norm"], 1.0)
    if s["bits"] == 32:
        m, v = s["exp_avg"], s["exp_avg_sq"]
    else:
        m = _decoded(s["exp_avg"] & 127, s["exp_avg_exponent"], 15)
        m = torch.where(s["exp_avg"] > 127, -m, m)
        v = _decoded(s["exp_avg_sq"], s["exp_avg_sq_exponent"], 31)
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * (1 - b2) * g
    p = _flat(s["params"], s["total"]) if s["master"] is None else s["master"]
    c1, c2 = 1 - b1 ** s["step"], 1 - b2 ** s["step"]
    p = p * (1 - lr * wd) - m / (v.sqrt() * (1 / math.sqrt(c2)) + eps) * (lr / c1)
    torch._foreach_copy_(s["params"], [p[a:a + n] for a, n in zip(s["starts"], s["sizes"])])
    if s["master"] is not None:
        out["master"] = s["master"].copy_(p)
    if s["bits"] == 32:
        return dict(out, params=s["params"], exp_avg=s["exp_avg"].copy_(m), exp_avg_sq=s["exp_avg_sq"].copy_(v))
    key = _mixed(s["seed"] + s["step"] * _GOLDEN)
    h = _mixed(torch.arange(s["total"], device="cuda") * _GOLDEN ^ key)
    code, e = _encoded(m.abs(), 15, 20, (h & 0xFFFF).float() * 2.0 ** -16)
    s["exp_avg"].copy_(code + (m < 0) * torch.tensor(128, dtype=torch.uint8, device="cuda"))
    s["exp_avg_exponent"].copy_(e)
    code, e = _encoded(v, 31, 36, (h >> 16).float() * 2.0 ** -16)
    s["exp_avg_sq"].copy_(code)
    s["exp_avg_sq_exponent"].copy_(e)
    m = _decoded(s["exp_avg"] & 127, s["exp_avg_exponent"], 15)
    return dict(out, params=s["params"], exp_avg=torch.where(s["exp_avg"] > 127, -m, m), exp_avg_sq=_decoded(s["exp_avg_sq"], s["exp_avg_sq_exponent"], 31))


_plain = dict(score=_plain_score, learn=_plain_learn, lookup=_plain_lookup, embed=_plain_embed, adamw=_plain_adamw)


# ---------------------------------------------------------------------------------------------- the framework's operators

def _own_score(s):
    r = s["bps"].log_probs(s["logits"], s["tokens"], mask=s["mask"], scale=s["scale"], top_k=s["top_k"])
    out = dict(logp=r.logp, entropy=r.entropy, lse=r.lse)
    return dict(out, top_ids=r.top_ids, top_logp=r.top_logp) if s["top_k"] else out


def _own_learn(s):
    r = s["bps"].log_probs(s["logits"], s["tokens"], mask=s["mask"], scale=s["scale"])
    grad = s["bps"].log_probs_backward(s["logits"], s["tokens"], r, s["grad_logp"], s["grad_entropy"], mask=s["mask"], scale=s["scale"])
    return dict(logp=r.logp, entropy=r.entropy, lse=r.lse, grad_logits=grad)


def _own_lookup(s):
    return dict(out=s["bps"].embedding(s["tokens"], s["weight"], scale=s["scale"]))


def _own_embed(s):
    return dict(_own_lookup(s), grad_weight=s["bps"].embedding_backward(s["tokens"], s["grad_out"], s["weight"].shape[0], scale=s["scale"]))


def _own_adamw(s):
    opt = s["opt"]
    opt.step(s["grads"])
    exp_avg, exp_avg_sq = opt.states()
    out = dict(params=s["params"], exp_avg=exp_avg, exp_avg_sq=exp_avg_sq)
    if opt.master is not None:
        out["master"] = opt.master
    return dict(out, grad_norm=opt.grad_norm) if s["clip"] else out


_own = dict(score=_own_score, learn=_own_learn, lookup=_own_lookup, embed=_own_embed, adamw=_own_adamw)


# ---------------------------------------------------------------------------------------------- work and exact values

def work(case):
    b = _BYTES[case["dtype"]]
    if case["op"] in ("score", "learn"):
        N, V = case["N"], case["V"]
        data = N * V * b + 16 * N + {"none": 0, "shared": V, "rows": N * V}[case["mask"]]
        if case["op"] == "score":
            return dict(bytes=data + 8 * N * min(case["top_k"], V), flops=8 * N * V)
        return dict(bytes=data + N * V * b + 8 * N, flops=16 * N * V)
    if case["op"] in ("lookup", "embed"):
        N, V, D = case["N"], case["V"], case["D"]
        data = 4 * N + min(N, V) * D * b + N * D * b
        return dict(bytes=data + (N * D * b + V * D * 4 if case["op"] == "embed" else 0), flops=N * D * (2 if case["op"] == "embed" else 1))
    P = sum(_sizes(case))
    # gradient read; float32 weight read and written; a 16-bit copy written; states read and written
    data = P * (b + 8 + (b if case["dtype"] != "f32" else 0))
    # 8-bit states are read and written, and what they stand for is written in 32 bits
    return dict(bytes=data + P * (16 if case["bits"] == 32 else 4 + 8), flops=14 * P)


def exact(case, seed):
    """run()'s outputs from the definition in 64 bits."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return dict(score=_exact_score, learn=_exact_score, lookup=_exact_embed, embed=_exact_embed, adamw=_exact_adamw)[case["op"]](case, s)


def _exact_score(case, s):
    learn = case["op"] == "learn"
    parts = []
    N, V, k = case["N"], case["V"], s["top_k"]
    step = max(1, 60_000_000 // V)
    for i in range(0, N, step):
        y = s["logits"][i:i + step].double() * s["scale"]
        if s["mask"] is not None:
            y.masked_fill_(~(s["mask"] if s["mask"].dim() == 1 else s["mask"][i:i + step]), -math.inf)
        n = y.shape[0]
        t = s["tokens"][i:i + step].long()
        lse = torch.logsumexp(y, 1)
        some = torch.isfinite(lse)
        p = torch.exp(y - torch.where(some, lse, 0.0)[:, None])
        # entropy: the mean of the surprise, lse - y
        away = torch.where(p > 0, lse[:, None] - y, 0.0)
        entropy = (p * away).sum(1)
        logp = y[torch.arange(n, device="cuda"), t.clamp(min=0)] - torch.where(some, lse, 0.0)
        logp[t < 0] = 0.0
        part = dict(logp=logp, entropy=entropy, lse=lse)
        if learn:
            gl = s["grad_logp"][i:i + step].double().clone()
            gl[(t < 0) | torch.isinf(logp)] = 0.0
            gh = s["grad_entropy"][i:i + step].double()
            d = p * (gh[:, None] * (away - entropy[:, None]) - gl[:, None])
            d[torch.arange(n, device="cuda"), t.clamp(min=0)] += gl
            part["grad_logits"] = (d * s["scale"]).float()  # held in 32 bits, which the 16-bit outputs are far from
            if s["logits"].dtype == torch.float32:
                part["grad_logits"] = d * s["scale"]
        elif k:
            part["top_logp"] = y.topk(k, dim=1).values - torch.where(some, lse, 0.0)[:, None]
        parts.append(part)
    out = {name: torch.cat([q[name] for q in parts]) for name in parts[0]}
    return dict(out, top_ids=None) if k else out


def _exact_embed(case, s):
    t = s["tokens"].long()
    used = t >= 0
    scale = float(s["scale"])
    result = torch.zeros((case["N"], case["D"]), dtype=torch.float64, device="cuda")
    result[used] = s["weight"].double()[t[used]] * scale
    if case["op"] == "lookup":
        return dict(out=result)
    grad = torch.zeros((case["V"], case["D"]), dtype=torch.float64, device="cuda")
    for i in range(0, case["N"], 32768):
        u = used[i:i + 32768]
        grad.index_put_((t[i:i + 32768][u],), s["grad_out"][i:i + 32768][u].double() * scale, accumulate=True)
    return dict(out=result, grad_weight=grad)


def _exact_adamw(case, s):
    (b1, b2), lr, eps, wd = _ADAMW["betas"], _ADAMW["lr"], _ADAMW["eps"], _ADAMW["weight_decay"]
    t = s["step"] + 1
    grads = [g.double() for g in s["grads"]]
    out = {}
    if s["clip"]:
        norm = math.sqrt(sum(float(g.square().sum()) for g in grads))
        out["grad_norm"] = torch.tensor([norm], dtype=torch.float64)
        if norm > s["clip"]:
            grads = [g.mul_(s["clip"] / norm) for g in grads]
    if s["bits"] == 32:
        m, v = s["exp_avg"].double(), s["exp_avg_sq"].double()
    else:
        m = _value_of(s["exp_avg"] & 127, s["exp_avg_exponent"], 15) * (1 - 2 * (s["exp_avg"] >> 7).double())
        v = _value_of(s["exp_avg_sq"], s["exp_avg_sq_exponent"], 31)
    master = torch.zeros(s["total"], dtype=torch.float64, device="cuda")
    params = []
    for w, g, a, n in zip(s["params"], grads, s["starts"], s["sizes"]):
        at = slice(a, a + n)
        m[at] = b1 * m[at] + (1 - b1) * g
        v[at] = b2 * v[at] + (1 - b2) * g ** 2
        w = (w.double() if s["master"] is None else s["master"][at].double()) * (1 - lr * wd)
        w -= lr * (m[at] / (1 - b1 ** t)) / ((v[at] / (1 - b2 ** t)).sqrt() + eps)
        params.append(w)
        master[at] = w
    out["params"] = params
    if s["master"] is not None:
        out["master"] = master
    # what 8-bit states are rounded to hangs on the last bits of 32: no value in 64 bits
    return dict(out, exp_avg=m if s["bits"] == 32 else None, exp_avg_sq=v if s["bits"] == 32 else None)


def _value_of(codes, exponents, top):
    c = codes.double().view(-1, _BLOCK)
    field = torch.floor(c / 8)
    mantissa = torch.where(field > 0, 1 + (c - field * 8) / 8, c / 8)
    return (mantissa * torch.exp2(exponents.double()[:, None] - 127 - top + field.clamp(min=1))).view(-1)
