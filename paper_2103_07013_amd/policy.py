"""Operators of the policy that consumes the frames, over the C ABI of include/bps.h: scores of tokens (actions), the
embedding of tokens, and AdamW over many tensors.  Marshalling only; tensors are torch's, on the GPU.

Calls take their device from the tensors and torch's current stream of it, unless `stream` names another (a
torch.cuda.Stream or a raw hipStream_t, 0 = the default stream), which is then current for the call: what it
allocates belongs to that stream.  A tensor that is used on another stream than its own has to be complete, and
to be kept alive or recorded on that stream, by the caller, as for every operator of torch.
"""
from __future__ import annotations

import collections
import ctypes

import torch

from .binding import BpsError, bps_last_error, load_library

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_TOKEN_BITS = {torch.int32: 32, torch.int64: 64}
STATE_BLOCK = 256

#: what log_probs returns; `held` is what log_probs_backward needs of it: float32 [5, ...]
LogProbs = collections.namedtuple("LogProbs", "logp entropy lse top_ids top_logp held")


class _Tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("master", ctypes.c_void_p), ("count", ctypes.c_uint64), ("start", ctypes.c_uint64),
                ("weight_decay", ctypes.c_float), ("lr_scale", ctypes.c_float)]


class _Config(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int32), ("state_bits", ctypes.c_int32), ("tensors", ctypes.c_uint32), ("seed", ctypes.c_uint32),
                ("total", ctypes.c_uint64), ("tensor", ctypes.POINTER(_Tensor)), ("exp_avg", ctypes.c_void_p), ("exp_avg_sq", ctypes.c_void_p),
                ("exp_avg_exponent", ctypes.c_void_p), ("exp_avg_sq_exponent", ctypes.c_void_p)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        p, i32, u32, i64, u64, f32, f64, size = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float,
                                                 ctypes.c_double, ctypes.c_size_t)
        for name, result, arguments in (
                ("bps_log_probs_workspace", size, [i32, u64, u32, u32]),
                ("bps_log_probs", i32, [p, i32, u64, u32, i64, p, i32, p, i64, f32, u32, p, p, p, p, p, p, p, size, p]),
                ("bps_log_probs_backward", i32, [p, i32, u64, u32, i64, p, i32, p, i64, f32, p, p, p, p, p, p, i64, p]),
                ("bps_embedding", i32, [p, i32, u64, p, i32, u32, u32, i64, f32, p, i64, p]),
                ("bps_embedding_backward_workspace", size, [u64, u32, u32]),
                ("bps_embedding_backward", i32, [p, i32, u64, p, i32, u32, u32, i64, f32, p, i32, i64, i32, p, size, p]),
                ("bps_adamw_create", i32, [ctypes.POINTER(_Config), ctypes.POINTER(p)]),
                ("bps_adamw_destroy", None, [p]),
                ("bps_adamw_step", i32, [p, p, i32, u64, f64, f64, f64, f64, f64, f64, p, p]),
                ("bps_adamw_read_states", i32, [p, p, p, p])):
            f = getattr(lib, name)
            f.restype, f.argtypes = result, arguments
        _lib = lib
    return _lib


def _checked(status):
    if status:
        raise BpsError(status, bps_last_error())


_current_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
# The library writes through addresses: autograd is told of tensors that were there before, so that graphs that saved them are refused.
_written = torch.autograd.graph.increment_version


def _on(index, call, *arguments):
    """call(*arguments, stream) with device `index` current and torch's stream of it."""
    if index == _current_device():
        return call(*arguments, _current_stream(index))
    with torch.cuda.device(index):
        return call(*arguments, _current_stream(index))


def _stream(stream, device):
    """A context in which `stream` is current."""
    if isinstance(stream, int):
        # the default stream's handle is 0, which ExternalStream would take for none given
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    elif stream.device != device:
        raise ValueError(f"stream: need one of {device}, got one of {stream.device}")
    return torch.cuda.stream(stream)


def _rows(t, name, width=None):
    """(leading shape, rows, width, elements from row to row) of a GPU tensor whose rows are a plain list in memory."""
    if not t.is_cuda or t.dtype not in _TYPES:
        raise ValueError(f"{name}: need a float32, bfloat16 or float16 CUDA tensor")
    shape, strides = t.shape, t.stride()
    if not shape or shape[-1] == 0 or (width is not None and shape[-1] != width):
        raise ValueError(f"{name}: the last dimension must be {'at least 1' if width is None else width}, got shape {tuple(shape)}")
    if 0 in shape:
        return shape[:-1], 0, shape[-1], shape[-1]
    if strides[-1] != 1 and shape[-1] != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    if len(shape) == 2:
        return shape[:-1], shape[0], shape[1], strides[0]
    rows, step = 1, None
    for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n != 1:
            if step is None:
                step = s
            elif s != step * rows:
                raise ValueError(f"{name}: the leading dimensions must be one list of rows (a contiguous tensor is)")
            rows *= n
    return shape[:-1], rows, shape[-1], shape[-1] if step is None else step


def _tokens(t, shape, device):
    if t.dtype not in _TOKEN_BITS or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"tokens: need a contiguous int32 or int64 tensor of shape {tuple(shape)} on {device}")
    return _TOKEN_BITS[t.dtype]


def _mask(mask, shape, rows, width, device):
    """(pointer, bytes from row to row)"""
    if mask is None:
        return None, 0
    if mask.dtype not in (torch.bool, torch.uint8) or mask.device != device:
        raise ValueError(f"mask: need a bool or uint8 tensor on {device}")
    if mask.shape == (width,):
        step = 0
    elif mask.shape == (*shape, width):
        step = width
    else:
        raise ValueError(f"mask: need shape {(width,)} or {(*shape, width)}, got {tuple(mask.shape)}")
    if not mask.is_contiguous():
        raise ValueError("mask: need a contiguous tensor")
    return mask.data_ptr(), step


def _vector(t, shape, device, name):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous float32 tensor of shape {tuple(shape)} on {device}")
    return t.data_ptr()


def _log_probs(logits, tokens, mask, scale, top_k):
    lib = _lib or _library()
    shape, rows, width, step = _rows(logits, "logits")
    device = logits.device
    bits = _tokens(tokens, shape, device)
    mask_at, mask_step = _mask(mask, shape, rows, width, device) if mask is not None else (None, 0)
    held = torch.empty(5, *shape, dtype=torch.float32, device=device)
    at, size = held.data_ptr(), 4 * rows
    dtype = _TYPES[logits.dtype]
    top_ids = top_logp = ids_at = top_at = space = None
    if top_k:
        if not 0 < top_k <= 64:
            raise ValueError("top_k must be 0 .. 64")
        top_ids = torch.empty((*shape, top_k), dtype=torch.int32, device=device)
        top_logp = torch.empty((*shape, top_k), dtype=torch.float32, device=device)
        ids_at, top_at = top_ids.data_ptr(), top_logp.data_ptr()
    space_size = lib.bps_log_probs_workspace(dtype, rows, width, top_k)
    if space_size:
        space = torch.empty(space_size, dtype=torch.uint8, device=device)
    status = _on(device.index, lib.bps_log_probs, logits.data_ptr(), dtype, rows, width, step, tokens.data_ptr(), bits, mask_at, mask_step, scale, top_k, at, at + size, at + 2 * size,
                 at + 3 * size, ids_at, top_at, None if space is None else space.data_ptr(), space_size)
    if status:
        _checked(status)
    logp, entropy, lse, _, _ = held.unbind(0)
    return LogProbs(logp, entropy, lse, top_ids, top_logp, held)


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, mask, scale, top_k):
        r = _log_probs(logits, tokens, mask, scale, top_k)
        ctx.save_for_backward(logits, tokens, mask, r.held)
        ctx.scale = scale
        # logp and entropy are the caller's, who may write to them; the gradient has what is held
        logp, entropy = r.logp.clone(), r.entropy.clone()
        ctx.mark_non_differentiable(*(t for t in r[2:] if t is not None))
        ctx.set_materialize_grads(False)
        return logp, entropy, *r[2:]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_logp, grad_entropy, *_):
        logits, tokens, mask, held = ctx.saved_tensors
        plain = [None if g is None else g.to(torch.float32).contiguous() for g in (grad_logp, grad_entropy)]
        return log_probs_backward(logits, tokens, held, *plain, mask=mask, scale=ctx.scale), None, None, None, None


def log_probs(logits, tokens, mask=None, scale=1.0, top_k=0, stream=None):
    """Log probabilities of `tokens` under softmax(scale * logits), with the entropy and the `top_k` best alternatives.

    logits  float32, bfloat16 or float16 [..., entries]; tokens int32 or int64 [...], -1 = none; mask bool [..., entries] or
    [entries], False = the entry is forbidden.  -> LogProbs(logp, entropy, lse, top_ids, top_logp, held), float32 [...] (top_ids int32,
    [..., top_k]; both None without top_k; held [5, ...], which the gradient needs).  logp and entropy carry a gradient to the
    logits; the rest is for reading.  Where no gradient is recorded logp, entropy and lse are parts of held: what is written to
    them is what log_probs_backward finds there.
    """
    if stream is not None:
        with _stream(stream, logits.device):
            return log_probs(logits, tokens, mask, scale, top_k)
    if logits.requires_grad and torch.is_grad_enabled():
        return LogProbs(*_LogProbs.apply(logits, tokens, mask, scale, top_k))
    return _log_probs(logits, tokens, mask, scale, top_k)


def log_probs_backward(logits, tokens, result, grad_logp=None, grad_entropy=None, mask=None, scale=1.0, out=None, stream=None):
    """The gradient of log_probs' logp and entropy with respect to the logits, in their type.

    result: what log_probs returned for the same arguments (or its `held`); grad_*: float32 [...] or None (zero); out: where it is
    written, may be the logits.
    """
    if stream is not None:
        with _stream(stream, logits.device):
            return log_probs_backward(logits, tokens, result, grad_logp, grad_entropy, mask, scale, out)
    lib = _lib or _library()
    shape, rows, width, step = _rows(logits, "logits")
    device = logits.device
    bits = _tokens(tokens, shape, device)
    mask_at, mask_step = _mask(mask, shape, rows, width, device) if mask is not None else (None, 0)
    at, size = _vector(result.held if isinstance(result, LogProbs) else result, (5, *shape), device, "result"), 4 * rows
    given = out is not None
    if not given:
        out = torch.empty(*shape, width, dtype=logits.dtype, device=device)
        out_step = width
    else:
        if out.dtype != logits.dtype or out.device != device or out.shape != logits.shape:
            raise ValueError("out: need a tensor of the logits' shape, type and device")
        out_step = _rows(out, "out", width)[3]
    status = _on(device.index, lib.bps_log_probs_backward, logits.data_ptr(), _TYPES[logits.dtype], rows, width, step, tokens.data_ptr(), bits, mask_at, mask_step, scale,
                 at, at + size, at + 3 * size, _vector(grad_logp, shape, device, "grad_logp"), _vector(grad_entropy, shape, device, "grad_entropy"), out.data_ptr(), out_step)
    if status:
        _checked(status)
    if given:
        _written(out)
    return out


def _embedding(tokens, weight, scale, out):
    lib = _lib or _library()
    if weight.dim() != 2:
        raise ValueError("weight: need a tensor [rows, width]")
    _, rows, width, step = _rows(weight, "weight")
    device = weight.device
    bits = _tokens(tokens, tokens.shape, device)
    given = out is not None
    if not given:
        out = torch.empty(*tokens.shape, width, dtype=weight.dtype, device=device)
        out_step = width
    else:
        if out.dtype != weight.dtype or out.device != device or out.shape != (*tokens.shape, width):
            raise ValueError(f"out: need a {weight.dtype} tensor of shape {(*tokens.shape, width)} on {device}")
        out_step = _rows(out, "out", width)[3] if out.numel() else width
    _checked(_on(device.index, lib.bps_embedding, tokens.data_ptr(), bits, tokens.numel(), weight.data_ptr(), _TYPES[weight.dtype], rows, width, step, scale,
                 out.data_ptr(), out_step))
    if given:
        _written(out)
    return out


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, weight, scale):
        ctx.save_for_backward(tokens)
        ctx.rows, ctx.dtype, ctx.scale = weight.shape[0], weight.dtype, scale
        return _embedding(tokens, weight, scale, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out):
        return None, embedding_backward(ctx.saved_tensors[0], grad_out.contiguous(), ctx.rows, ctx.scale, dtype=ctx.dtype), None


def embedding(tokens, weight, scale=1.0, out=None, stream=None):
    """Rows of `weight` [rows, width] for int32 or int64 tokens [...], times scale; zeros for token -1. -> [..., width]

    Carries a gradient to the weight, unless `out` is given, which shares no memory with it."""
    if stream is not None:
        with _stream(stream, weight.device):
            return embedding(tokens, weight, scale, out)
    if out is None and torch.is_grad_enabled() and weight.requires_grad:
        return _Embedding.apply(tokens, weight, scale)
    return _embedding(tokens, weight, scale, out)


def embedding_backward(tokens, grad_out, rows, scale=1.0, dtype=torch.float32, out=None, accumulate=False, stream=None):
    """The gradient of embedding's weight, [rows, width] of `dtype`: sums over equal tokens in float32, the same bits every time.

    out: where it is written; with accumulate the sums are added to what `out` holds."""
    if stream is not None:
        with _stream(stream, grad_out.device):
            return embedding_backward(tokens, grad_out, rows, scale, dtype, out, accumulate)
    lib = _lib or _library()
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    if grad_out.dim() == 0 or grad_out.shape[:-1] != tokens.shape:
        raise ValueError(f"grad_out: need shape {(*tokens.shape, 'width')}, got {tuple(grad_out.shape)}")
    device = grad_out.device
    if grad_out.numel():
        _, count, width, step = _rows(grad_out, "grad_out")
    else:
        count, width, step = 0, grad_out.shape[-1], grad_out.shape[-1]
    bits = _tokens(tokens, tokens.shape, device)
    given = out is not None
    if not given:
        out = torch.empty(rows, width, dtype=dtype, device=device)
        out_step = width
    else:
        if out.device != device or out.shape != (rows, width):
            raise ValueError(f"out: need a tensor of shape {(rows, width)} on {device}")
        out_step = _rows(out, "out", width)[3]
    if out.dtype not in _TYPES or grad_out.dtype not in _TYPES or not grad_out.is_cuda:
        raise ValueError("need float32, bfloat16 or float16 CUDA tensors")
    size = lib.bps_embedding_backward_workspace(count, rows, width)
    space = torch.empty(size, dtype=torch.uint8, device=device) if size else None
    _checked(_on(device.index, lib.bps_embedding_backward, tokens.data_ptr(), bits, count, grad_out.data_ptr(), _TYPES[grad_out.dtype], rows, width, step, scale,
                 out.data_ptr(), _TYPES[out.dtype], out_step, int(accumulate), space.data_ptr() if size else None, size))
    if given:
        _written(out)
    return out


class AdamW:
    """One AdamW step over all of a model's tensors at once (include/bps.h states the rule).

    params        contiguous tensors of one type on one GPU, each with at least one element, that share no memory; float32 ones are updated in place,
                  bfloat16 and float16 ones get the rounded values of float32 masters that are kept here
    weight_decay, lr_scale   one number, or one for each tensor
    state_bits    32, or 8: a byte and a 256th per state, rounded up or down so that the mean is kept (seed)
    max_grad_norm > 0: gradients are scaled down to this 2-norm over all tensors; a step whose norm is not finite changes nothing
                  (but it counts among `steps`)

    lr, betas, eps and max_grad_norm may be changed between steps.  State: master (or None), exp_avg, exp_avg_sq,
    with 8 bits exp_avg_exponent and exp_avg_sq_exponent, and steps; a tensor's part of them begins at starts[i].  The
    library has the tensors' addresses: saved states are copied into them (exp_avg.copy_(saved)), and a step or states() after one of
    them was replaced is refused.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, lr_scale=1.0, state_bits=32, max_grad_norm=0.0, seed=0):
        self._handle = None
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        first = self.params[0]
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8")
        if first.dtype not in _TYPES or not first.is_cuda:
            raise ValueError("parameters must be float32, bfloat16 or float16 CUDA tensors")
        for p in self.params:
            if p.dtype != first.dtype or p.device != first.device or not p.is_contiguous() or p.numel() == 0:
                raise ValueError("parameters must be contiguous, not empty, and of one type on one device")
        n = len(self.params)
        decay, lr_scale = ([float(v)] * n if isinstance(v, (int, float)) else [float(x) for x in v] for v in (weight_decay, lr_scale))
        if len(decay) != n or len(lr_scale) != n:
            raise ValueError("weight_decay and lr_scale: one number, or one for each parameter")
        self.lr, self.betas, self.eps, self.max_grad_norm = lr, tuple(betas), eps, max_grad_norm
        self.state_bits, self.seed, self.steps, self.device, self.dtype = state_bits, int(seed) & 0xFFFFFFFF, 0, first.device, first.dtype
        self.starts, self.total = [], 0
        for p in self.params:
            self.starts.append(self.total)
            self.total += -(-p.numel() // STATE_BLOCK) * STATE_BLOCK
        make = dict(device=self.device)
        self.master = None
        if first.dtype != torch.float32:
            self.master = torch.zeros(self.total, dtype=torch.float32, **make)
            for p, a in zip(self.params, self.starts):
                self.master[a:a + p.numel()].copy_(p.detach().reshape(-1))
        kind = torch.float32 if state_bits == 32 else torch.uint8
        self.exp_avg, self.exp_avg_sq = (torch.zeros(self.total, dtype=kind, **make) for _ in range(2))
        self.exp_avg_exponent = self.exp_avg_sq_exponent = None
        if state_bits == 8:
            self.exp_avg_exponent, self.exp_avg_sq_exponent = (torch.zeros(self.total // STATE_BLOCK, dtype=torch.uint8, **make) for _ in range(2))
        self.grad_norm = torch.zeros(1, dtype=torch.float32, **make)
        self._counts = [p.numel() for p in self.params]
        self._places = [p.data_ptr() for p in self.params]
        table = (_Tensor * n)()
        for i, (p, a) in enumerate(zip(self.params, self.starts)):
            table[i] = _Tensor(p.data_ptr(), None if self.master is None else self.master.data_ptr() + 4 * a, p.numel(), a, decay[i], lr_scale[i])
        at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        config = _Config(_TYPES[first.dtype], state_bits, n, self.seed, self.total, table, at(self.exp_avg), at(self.exp_avg_sq), at(self.exp_avg_exponent),
                         at(self.exp_avg_sq_exponent))
        handle = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _checked(_library().bps_adamw_create(ctypes.byref(config), ctypes.byref(handle)))
        self._handle = handle
        self._grads = (ctypes.c_void_p * n)()
        self._kept = [(name, t, t.data_ptr()) for name in ("master", "exp_avg", "exp_avg_sq", "exp_avg_exponent", "exp_avg_sq_exponent", "grad_norm")
                      if (t := getattr(self, name)) is not None]

    def _check_kept(self):
        for name, t, place in self._kept:
            if getattr(self, name) is not t or t.data_ptr() != place:
                raise ValueError(f"{name} was replaced: this optimiser works on the one that it was made with, into which values can be copied")

    def step(self, grads=None, grad_scale=1.0, stream=None):
        """One step with the parameters' gradients, or with `grads`: one contiguous tensor (or None) for each, of the
        parameters' type or all float32, times grad_scale (one over a loss scale).  With max_grad_norm > 0 grad_norm receives the
        norm.  Captured into a graph, it replays with the step number, and the rounding of 8-bit states, that it was captured with."""
        if stream is not None:
            with _stream(stream, self.device):
                return self.step(grads, grad_scale)
        if self._handle is None:
            raise ValueError("this optimiser is closed")
        if [p.data_ptr() for p in self.params] != self._places:
            raise ValueError("a parameter's memory is no longer where it was when this optimiser was made")
        self._check_kept()
        grads = [p.grad for p in self.params] if grads is None else list(grads)
        if len(grads) != len(self.params):
            raise ValueError("grads: one for each parameter")
        kind = None
        for g, n in zip(grads, self._counts):
            if g is None:
                continue
            if kind is None:
                kind = g.dtype
                if kind != self.dtype and kind != torch.float32:
                    raise ValueError("grads: the parameters' type, or float32")
            if g.dtype != kind or g.numel() != n or g.device != self.device or not g.is_contiguous():
                raise ValueError("grads: contiguous tensors of one type, each of its parameter's size and device")
        if kind is None:
            return
        self._grads[:] = [None if g is None else g.data_ptr() for g in grads]
        _checked(_on(self.device.index, _library().bps_adamw_step, self._handle, self._grads, _TYPES[kind], self.steps + 1, self.lr, *self.betas, self.eps, grad_scale,
                     self.max_grad_norm, self.grad_norm.data_ptr()))
        self.steps += 1
        _written([p for p, g in zip(self.params, grads) if g is not None] + [t for _, t, _ in self._kept])

    def states(self, stream=None):
        """(exp_avg, exp_avg_sq) as float32: the arrays themselves with 32 bits, what their codes stand for with 8."""
        if stream is not None:
            with _stream(stream, self.device):
                return self.states()
        self._check_kept()
        if self.state_bits == 32:
            return self.exp_avg, self.exp_avg_sq
        if self._handle is None:
            raise ValueError("this optimiser is closed")
        m, v = torch.empty((2, self.total), dtype=torch.float32, device=self.device).unbind(0)
        _checked(_on(self.device.index, _library().bps_adamw_read_states, self._handle, m.data_ptr(), v.data_ptr()))
        return m, v

    def close(self):
        if self._handle is not None:
            _library().bps_adamw_destroy(self._handle)
            self._handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
