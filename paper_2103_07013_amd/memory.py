"""Operators of the memory of a policy that consumes the frames, over the C ABI of include/bps_memory.h: a causal convolution, a selective state
space scan, and the norms around a block.  Marshalling only; tensors are torch's, on the GPU.

Sequences are [batch, steps, channels] with any strides over batch and steps (for scans below 2^26 elements from step to step), so that
rollouts gathered step by step are used as they are (x.transpose(0, 1)); `starts` [batch, steps] says where episodes begin, `lengths` [batch] where padded sequences end.  A call takes
a state and returns the next one; *_step does the same for one step, in place.  No gradient goes through states, and there are no
forward-mode derivatives: states that ask for a gradient and tensors with a tangent are refused.

Devices and streams are as for the policy's other operators: the tensors' device, torch's current stream of it unless `stream` names
another, which is then current for the call.
"""
from __future__ import annotations

import collections
import ctypes
import os

import torch

from . import build as _build
from .binding import load_library
from .policy import _TYPES, _checked, _no_tangent, _on, _rows, _stream, _written

#: what causal_conv returns: the outputs, and the inputs that the next call's windows begin with
CausalConv = collections.namedtuple("CausalConv", "out state")
ConvGrads = collections.namedtuple("ConvGrads", "x weight bias")
#: what selective_scan returns; `held` (None without hold) is what selective_scan_backward needs of it
SelectiveScan = collections.namedtuple("SelectiveScan", "out state held")
ScanGrads = collections.namedtuple("ScanGrads", "x delta A B C D gate delta_bias")
#: what residual_norm returns; `held` is what residual_norm_backward needs of it
ResidualNorm = collections.namedtuple("ResidualNorm", "residual out held")
NormGrads = collections.namedtuple("NormGrads", "residual block post_weight gate scale pre_weight")

EXPORTS = ["bps_causal_conv", "bps_causal_conv_backward_workspace", "bps_causal_conv_backward", "bps_selective_scan_workspace", "bps_selective_scan",
           "bps_selective_scan_backward_workspace", "bps_selective_scan_backward", "bps_residual_norm", "bps_residual_norm_backward_workspace", "bps_residual_norm_backward"]
HELD_STEPS = 16
_ACTIVATIONS = {"sigmoid": 0, "silu": 1}
_p, _i32, _u32, _i64, _u64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float


def _sequences(*names):
    return [f for n in names for f in ((n, _p), (n + "_batch_stride", _i64), (n + "_step_stride", _i64))]


class _Conv(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("weight_dtype", _i32), ("batch", _u32), ("steps", _u32), ("channels", _u32), ("taps", _u32), ("silu", _i32), *_sequences("x", "out"),
                ("weight", _p), ("bias", _p), *_sequences("starts"), ("lengths", _p), ("state", _p), ("state_out", _p), ("state_stride", _i64), ("state_out_stride", _i64),
                *_sequences("grad_out", "grad_x"), ("grad_weight", _p), ("grad_bias", _p)]


class _Scan(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("softplus", _i32), ("batch", _u32), ("steps", _u32), ("channels", _u32), ("states", _u32), ("groups", _u32),
                *_sequences("x", "delta", "gate", "B", "C", "out"), ("A", _p), ("D", _p), ("delta_bias", _p), *_sequences("starts"), ("lengths", _p), ("state", _p),
                ("state_out", _p), ("state_stride", _i64), ("state_out_stride", _i64), ("held", _p), *_sequences("grad_out", "grad_x", "grad_delta", "grad_gate", "grad_B", "grad_C"),
                ("grad_A", _p), ("grad_D", _p), ("grad_delta_bias", _p)]


class _Norm(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("residual_dtype", _i32), ("weight_dtype", _i32), ("activation", _i32), ("rows", _u64), ("width", _u32), ("eps", _f32),
                ("residual", _p), ("block", _p), ("gate", _p), ("residual_stride", _i64), ("block_stride", _i64), ("gate_stride", _i64), ("post_weight", _p), ("scale", _p),
                ("pre_weight", _p), ("residual_out", _p), ("out", _p), ("residual_out_stride", _i64), ("out_stride", _i64), ("roots", _p), ("grad_residual_out", _p),
                ("grad_out", _p), ("grad_residual_out_stride", _i64), ("grad_out_stride", _i64), ("grad_residual", _p), ("grad_block", _p), ("grad_gate", _p),
                ("grad_residual_stride", _i64), ("grad_block_stride", _i64), ("grad_gate_stride", _i64), ("grad_post_weight", _p), ("grad_scale", _p), ("grad_pre_weight", _p)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        load_library()
        if not os.path.exists(_build.MEMORY_LIB):
            _build.build_memory()
        lib = ctypes.CDLL(_build.MEMORY_LIB)
        size = ctypes.c_size_t
        for name, args, back, forth in (("bps_causal_conv", _Conv, True, False), ("bps_selective_scan", _Scan, True, True), ("bps_residual_norm", _Norm, True, False)):
            for f, space in ((name, forth), (name + "_backward", back)):
                call = getattr(lib, f)
                call.restype, call.argtypes = _i32, [ctypes.POINTER(args), *([_p, size] if space else []), _p]
                if space:
                    call = getattr(lib, f + "_workspace")
                    call.restype, call.argtypes = size, [ctypes.POINTER(args)]
        _lib = lib
    return _lib


def _sequence(t, name, shape, dtype, device):
    """(address, elements from batch to batch, from step to step); [batch, channels] is one step."""
    if t.dtype != dtype or t.device != device or t.shape != shape:
        raise ValueError(f"{name}: need a {dtype} tensor of shape {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] != 1 and t.numel():
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), strides[0], strides[1] if len(shape) == 3 else 0


def _shared(t, name, rows, channels, dtype, device):
    """The same of B or C, [..., states] or [..., groups, states], and its groups and states."""
    n = len(rows)
    if t.dtype != dtype or t.device != device or t.dim() not in (n + 1, n + 2) or t.shape[:n] != rows or 0 in t.shape[n:]:
        raise ValueError(f"{name}: need a {dtype} tensor of shape {(*rows, 'states')} or {(*rows, 'groups', 'states')} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    strides, states = t.stride(), t.shape[-1]
    groups = t.shape[n] if t.dim() == n + 2 else 1
    if t.numel() and ((strides[-1] != 1 and states != 1) or (groups != 1 and strides[n] != states)):
        raise ValueError(f"{name}: the groups and states of a step must be contiguous")
    if channels % groups:
        raise ValueError(f"{name}: {groups} groups for {channels} channels, which are no multiple of them")
    return (t.data_ptr(), strides[0], strides[1] if n == 2 else 0), groups, states


def _main(x, name):
    if not x.is_cuda or x.dtype not in _TYPES:
        raise ValueError(f"{name}: need a float32, bfloat16 or float16 CUDA tensor")
    if x.dim() not in (2, 3) or x.shape[-1] == 0:
        raise ValueError(f"{name}: need shape [batch, steps, channels] with at least one channel, got {tuple(x.shape)}")


def _starts(starts, shape, device):
    if starts is None:
        return None, 0, 0
    if starts.dtype not in (torch.bool, torch.uint8) or starts.device != device or starts.shape != shape:
        raise ValueError(f"starts: need a bool or uint8 tensor of shape {tuple(shape)} on {device}")
    return starts.data_ptr(), starts.stride(0), starts.stride(1) if len(shape) == 2 else 0


def _plain(t, name, shape, dtypes, device):
    """The address of a contiguous tensor."""
    if t is None:
        return None
    if t.dtype not in dtypes or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous {' or '.join(sorted({str(d) for d in dtypes}))} tensor of shape {tuple(shape)} on {device}")
    return t.data_ptr()


def _state(state, shape, dtype, device):
    """(address, elements from batch to batch)"""
    if state is None:
        return None, 0
    if state.dtype != dtype or state.device != device or state.shape != shape:
        raise ValueError(f"state: need a {dtype} tensor of shape {tuple(shape)} on {device}")
    if not state.is_contiguous() and state.numel() and not state[0].is_contiguous():
        raise ValueError("state: each sequence's must be contiguous")
    return state.data_ptr(), state.stride(0)


def _constant(state):
    """For calls that a gradient may be recorded of, where that is known: inside an autograd function nothing is recorded."""
    if state is not None and state.requires_grad and torch.is_grad_enabled():
        raise ValueError("state: no gradient goes through states (detach it)")


def _like(t):
    """A contiguous tensor of t's shape, type and device."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _any_grad(*tensors):
    for t in tensors:
        if t is not None and t.requires_grad:
            return True
    return False


def _no_gradient(what, *tensors):
    if torch.is_grad_enabled() and _any_grad(*tensors):
        raise ValueError(f"{what} has no gradient: call it under torch.no_grad(), or the call for sequences")


def _three(x, name):
    _main(x, name)
    if x.dim() != 3:
        raise ValueError(f"{name}: need shape [batch, steps, channels], got {tuple(x.shape)}")


def _call(index, f, args, size, device):
    space = torch.empty(size, dtype=torch.uint8, device=device) if size else None
    status = _on(index, f, args, None if space is None else space.data_ptr(), size)
    if status:
        _checked(status)


# ---------------------------------------------------------------------------------------------- convolution

def _conv_args(x, weight, bias, silu, starts, lengths, state):
    shape, dtype, device = x.shape, x.dtype, x.device
    batch, channels = shape[0], shape[-1]
    steps = shape[1] if len(shape) == 3 else 1
    if weight.dim() != 2 or weight.shape[0] != channels or not 1 <= weight.shape[1] <= 8:
        raise ValueError(f"weight: need shape {(channels, '1 .. 8')}, got {tuple(weight.shape)}")
    kind, taps = weight.dtype, weight.shape[1]
    if kind not in (dtype, torch.float32):
        raise ValueError(f"weight: need {dtype} or float32")
    weight_at, bias_at = _plain(weight, "weight", weight.shape, (kind,), device), _plain(bias, "bias", (channels,), (kind,), device)
    state_at, state_stride = _state(state, (batch, taps - 1, channels), dtype, device)
    a = _Conv(_TYPES[dtype], _TYPES[kind], batch, steps, channels, taps, bool(silu), *_sequence(x, "x", shape, dtype, device), None, 0, 0, weight_at, bias_at,
              *_starts(starts, shape[:-1], device), _plain(lengths, "lengths", (batch,), (torch.int32,), device), state_at, None, state_stride)
    return a, taps


def _causal_conv(x, weight, bias, silu, starts, lengths, state):
    lib = _lib or _library()
    _three(x, "x")
    a, taps = _conv_args(x, weight, bias, silu, starts, lengths, state)
    batch, steps, channels = x.shape
    out = _like(x)
    last = torch.empty(batch, taps - 1, channels, dtype=x.dtype, device=x.device)
    a.out, a.out_batch_stride, a.out_step_stride = out.data_ptr(), steps * channels, channels
    a.state_out, a.state_out_stride = last.data_ptr(), (taps - 1) * channels
    status = _on(x.device.index, lib.bps_causal_conv, a)
    if status:
        _checked(status)
    return CausalConv(out, last)


class _CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, silu, starts, lengths, state):
        r = _causal_conv(x, weight, bias, silu, starts, lengths, state)
        ctx.save_for_backward(x, weight, bias, starts, lengths, state)
        ctx.silu = silu
        ctx.mark_non_differentiable(r.state)
        ctx.set_materialize_grads(False)
        return r.out, r.state

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out, _):
        if grad_out is None:
            return (None,) * 7
        x, weight, bias, starts, lengths, state = ctx.saved_tensors
        return *causal_conv_backward(_as_taken(grad_out), x, weight, bias, ctx.silu, starts, lengths, state), None, None, None, None


def _as_taken(grad, steps_below=1 << 63):
    """What autograd brings, in an order that the calls take: its strides follow from what its user did with the outputs."""
    return grad if grad.stride(-1) == 1 and grad.stride(1) < steps_below else grad.contiguous()


def causal_conv(x, weight, bias=None, silu=True, starts=None, lengths=None, state=None, stream=None):
    """Each channel's inputs of the last few steps, weighted: u[t] = bias + sum of weight[:, k] x[t - taps + 1 + k], with silu u sigmoid(u).

    x float32, bfloat16 or float16 [batch, steps, channels]; weight [channels, taps], 1 to 8 taps, and bias [channels] of x's type or both
    float32; starts bool [batch, steps], where an episode begins (inputs from before count as zero); lengths int32 [batch], where padded
    sequences end; state [batch, taps - 1, channels] of x's type, the inputs before the first step (None: zeros).
    -> CausalConv(out, state): out is zero behind a sequence's end and carries a gradient to x, weight and bias; state is the next call's."""
    if stream is not None:
        with _stream(stream, x.device):
            return causal_conv(x, weight, bias, silu, starts, lengths, state)
    _no_tangent(x, weight, bias, state)
    _constant(state)
    if torch.is_grad_enabled() and _any_grad(x, weight, bias):
        return CausalConv(*_CausalConv.apply(x, weight, bias, silu, starts, lengths, state))
    return _causal_conv(x, weight, bias, silu, starts, lengths, state)


def causal_conv_backward(grad_out, x, weight, bias=None, silu=True, starts=None, lengths=None, state=None, stream=None):
    """The gradient of causal_conv's out for the same arguments. -> ConvGrads(x, weight, bias), each of its input's type (bias None without one)"""
    if stream is not None:
        with _stream(stream, x.device):
            return causal_conv_backward(grad_out, x, weight, bias, silu, starts, lengths, state)
    _no_tangent(grad_out, x, weight, bias, state)
    _constant(state)
    lib = _lib or _library()
    _three(x, "x")
    a, taps = _conv_args(x, weight, bias, silu, starts, lengths, state)
    batch, steps, channels = x.shape
    a.grad_out, a.grad_out_batch_stride, a.grad_out_step_stride = _sequence(grad_out, "grad_out", x.shape, x.dtype, x.device)
    grads = ConvGrads(_like(x), torch.empty_like(weight), None if bias is None else torch.empty_like(bias))
    a.grad_x, a.grad_x_batch_stride, a.grad_x_step_stride = grads.x.data_ptr(), steps * channels, channels
    a.grad_weight, a.grad_bias = grads.weight.data_ptr(), None if bias is None else grads.bias.data_ptr()
    _call(x.device.index, lib.bps_causal_conv_backward, a, lib.bps_causal_conv_backward_workspace(a), x.device)
    return grads


def causal_conv_step(x, state, weight, bias=None, silu=True, starts=None, stream=None):
    """causal_conv of one step: x [batch, channels] -> out [batch, channels].  The state [batch, taps - 1, channels] is moved on in place;
    starts bool [batch].  Has no gradient."""
    if stream is not None:
        with _stream(stream, x.device):
            return causal_conv_step(x, state, weight, bias, silu, starts)
    _no_tangent(x, state, weight, bias)
    _constant(state)
    lib = _lib or _library()
    _main(x, "x")
    if x.dim() != 2:
        raise ValueError(f"x: need shape [batch, channels], got {tuple(x.shape)}")
    _no_gradient("causal_conv_step", x, weight, bias)
    a, taps = _conv_args(x, weight, bias, silu, starts, None, state)
    if state is None:
        raise ValueError("a step needs a state")
    out = _like(x)
    a.out, a.out_batch_stride = out.data_ptr(), x.shape[1]
    a.state_out, a.state_out_stride = a.state, a.state_stride
    status = _on(x.device.index, lib.bps_causal_conv, a)
    if status:
        _checked(status)
    _written(state)
    return out


# ---------------------------------------------------------------------------------------------- scan

def _scan_args(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, state):
    shape, dtype, device = x.shape, x.dtype, x.device
    rows, batch, channels = shape[:-1], shape[0], shape[-1]
    b, groups, states = _shared(B, "B", rows, channels, dtype, device)
    c, *same = _shared(C, "C", rows, channels, dtype, device)
    if same != [groups, states]:
        raise ValueError(f"C: need B's groups and states, got {tuple(C.shape)} for {tuple(B.shape)}")
    f32 = (torch.float32,)
    if A is None:
        raise ValueError("A: need a tensor")
    state_at, state_stride = _state(state, (batch, states, channels), torch.float32, device)
    return _Scan(_TYPES[dtype], bool(softplus), batch, shape[1] if len(shape) == 3 else 1, channels, states, groups, *_sequence(x, "x", shape, dtype, device),
                 *_sequence(delta, "delta", shape, dtype, device), *((None, 0, 0) if gate is None else _sequence(gate, "gate", shape, dtype, device)), *b, *c, None, 0, 0,
                 _plain(A, "A", (states, channels), f32, device), _plain(D, "D", (channels,), f32, device), _plain(delta_bias, "delta_bias", (channels,), f32, device),
                 *_starts(starts, rows, device), _plain(lengths, "lengths", (batch,), (torch.int32,), device), state_at, None, state_stride)


def _selective_scan(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, state, hold):
    lib = _lib or _library()
    _three(x, "x")
    a = _scan_args(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, state)
    batch, steps, channels = x.shape
    device, states = x.device, a.states
    out = _like(x)
    last = torch.empty(batch, states, channels, dtype=torch.float32, device=device)
    held = torch.empty(batch, -(-steps // HELD_STEPS), states, channels, dtype=torch.float32, device=device) if hold else None
    a.out, a.out_batch_stride, a.out_step_stride = out.data_ptr(), steps * channels, channels
    a.state_out, a.state_out_stride = last.data_ptr(), states * channels
    if hold:
        a.held = held.data_ptr()
    _call(device.index, lib.bps_selective_scan, a, lib.bps_selective_scan_workspace(a), device)
    return SelectiveScan(out, last, held)


class _SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, state):
        r = _selective_scan(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, state, True)
        ctx.save_for_backward(x, delta, A, B, C, D, gate, delta_bias, starts, lengths, r.held)
        ctx.softplus = softplus
        ctx.mark_non_differentiable(r.state, r.held)
        ctx.set_materialize_grads(False)
        return tuple(r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out, *_):
        if grad_out is None:
            return (None,) * 12
        x, delta, A, B, C, D, gate, delta_bias, starts, lengths, held = ctx.saved_tensors
        g = selective_scan_backward(_as_taken(grad_out, 1 << 26), x, delta, A, B, C, held, D, gate, delta_bias, ctx.softplus, starts, lengths)
        return *g, None, None, None, None


def selective_scan(x, delta, A, B, C, D=None, gate=None, delta_bias=None, softplus=True, starts=None, lengths=None, state=None, hold=False, stream=None):
    """A linear recurrence for each channel and state whose decay and input depend on the step: with d = softplus(delta + delta_bias)
    (or delta + delta_bias),   h[n] = exp(d A[n]) h[n] + d x B[n];   out = (sum of C[n] h[n] + D x) * gate sigmoid(gate).

    x, delta, gate float32, bfloat16 or float16 [batch, steps, channels]; B, C of x's type [batch, steps, states], or [batch, steps, groups,
    states] where each group's are for channels / groups channels; A float32 [states, channels], 1 to 32 states, negative where states are to
    decay (what is below -1e38 counts as that); D, delta_bias float32 [channels]; starts bool [batch, steps], where an episode begins (with a state of zero); lengths int32
    [batch], where padded sequences end; state float32 [batch, states, channels] (None: zeros).
    -> SelectiveScan(out, state, held): out is zero behind a sequence's end and carries a gradient to all inputs but the state; state is the next
    call's; held float32 [batch, ceil(steps / 16), states, channels], with hold or where a gradient is recorded, is for
    selective_scan_backward."""
    if stream is not None:
        with _stream(stream, x.device):
            return selective_scan(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, state, hold)
    _no_tangent(x, delta, A, B, C, D, gate, delta_bias, state)
    _constant(state)
    if torch.is_grad_enabled() and _any_grad(x, delta, A, B, C, D, gate, delta_bias):
        return SelectiveScan(*_SelectiveScan.apply(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, state))
    return _selective_scan(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, state, hold)


def selective_scan_backward(grad_out, x, delta, A, B, C, result, D=None, gate=None, delta_bias=None, softplus=True, starts=None, lengths=None, stream=None):
    """The gradient of selective_scan's out for the same arguments.  result: what selective_scan returned with hold (or its `held`).
    -> ScanGrads(x, delta, A, B, C, D, gate, delta_bias), each of its input's type, None where there was none"""
    if stream is not None:
        with _stream(stream, x.device):
            return selective_scan_backward(grad_out, x, delta, A, B, C, result, D, gate, delta_bias, softplus, starts, lengths)
    _no_tangent(grad_out, x, delta, A, B, C, D, gate, delta_bias)
    lib = _lib or _library()
    _three(x, "x")
    a = _scan_args(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, lengths, None)
    batch, steps, channels = x.shape
    device, dtype, states, groups = x.device, x.dtype, a.states, a.groups
    held = result.held if isinstance(result, SelectiveScan) else result
    if held is None:
        raise ValueError("result: need what selective_scan returned with hold=True")
    a.held = _plain(held, "result", (batch, -(-steps // HELD_STEPS), states, channels), (torch.float32,), device)
    a.grad_out, a.grad_out_batch_stride, a.grad_out_step_stride = _sequence(grad_out, "grad_out", x.shape, dtype, device)
    gx, gd, gz, gb, gc, ga, g_skip, g_bias = (None if t is None else _like(t) for t in (x, delta, gate, B, C, A, D, delta_bias))
    for name, g, width in (("grad_x", gx, channels), ("grad_delta", gd, channels), ("grad_gate", gz, channels), ("grad_B", gb, groups * states), ("grad_C", gc, groups * states)):
        if g is not None:
            setattr(a, name, g.data_ptr())
            setattr(a, name + "_batch_stride", steps * width)
            setattr(a, name + "_step_stride", width)
    a.grad_A, a.grad_D, a.grad_delta_bias = (None if g is None else g.data_ptr() for g in (ga, g_skip, g_bias))
    _call(device.index, lib.bps_selective_scan_backward, a, lib.bps_selective_scan_backward_workspace(a), device)
    return ScanGrads(gx, gd, ga, gb, gc, g_skip, gz, g_bias)


def selective_scan_step(x, delta, state, A, B, C, D=None, gate=None, delta_bias=None, softplus=True, starts=None, stream=None):
    """selective_scan of one step: x, delta, gate [batch, channels], B, C [batch, states] or [batch, groups, states] -> out [batch, channels].
    The state float32 [batch, states, channels] is moved on in place; starts bool [batch].  Has no gradient."""
    if stream is not None:
        with _stream(stream, x.device):
            return selective_scan_step(x, delta, state, A, B, C, D, gate, delta_bias, softplus, starts)
    _no_tangent(x, delta, state, A, B, C, D, gate, delta_bias)
    _constant(state)
    lib = _lib or _library()
    _main(x, "x")
    if x.dim() != 2:
        raise ValueError(f"x: need shape [batch, channels], got {tuple(x.shape)}")
    _no_gradient("selective_scan_step", x, delta, A, B, C, D, gate, delta_bias)
    a = _scan_args(x, delta, A, B, C, D, gate, delta_bias, softplus, starts, None, state)
    if state is None:
        raise ValueError("a step needs a state")
    out = _like(x)
    a.out, a.out_batch_stride = out.data_ptr(), x.shape[1]
    a.state_out, a.state_out_stride = a.state, a.state_stride
    status = _on(x.device.index, lib.bps_selective_scan, a, None, 0)
    if status:
        _checked(status)
    _written(state)
    return out


# ---------------------------------------------------------------------------------------------- norms around a block

def _row_step(t, name, shape, kinds, device):
    """Elements from row to row"""
    if t.dtype not in kinds or t.device != device or t.shape != shape:
        raise ValueError(f"{name}: need a {' or '.join(str(k) for k in kinds)} tensor of shape {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return shape[-1] if t.is_contiguous() else _rows(t, name)[3]


def _norm_args(residual, block, post_weight, gate, scale, pre_weight, eps, activation, roots):
    shape, rows, width, step = _rows(block, "block")
    device, dtype = block.device, block.dtype
    shape = block.shape
    gate_at, gate_step = (None, 0) if gate is None else (gate.data_ptr(), _row_step(gate, "gate", shape, (dtype,), device))
    if activation not in _ACTIVATIONS:
        raise ValueError("activation: 'sigmoid' or 'silu'")
    kind, at = None, []
    for w, name in ((post_weight, "post_weight"), (scale, "scale"), (pre_weight, "pre_weight")):
        if w is None:
            at.append(None)
            continue
        if kind is None:
            kind = w.dtype
        if w.dtype != kind or kind not in (dtype, torch.float32):
            raise ValueError(f"post_weight, scale and pre_weight must be of one type, {dtype} or float32")
        at.append(_plain(w, name, (width,), (kind,), device))
    return _Norm(_TYPES[dtype], _TYPES.get(residual.dtype, -1), _TYPES[kind or dtype], _ACTIVATIONS[activation], rows, width, eps, residual.data_ptr(), block.data_ptr(),
                 gate_at, _row_step(residual, "residual", shape, (dtype, torch.float32), device), step, gate_step, *at, None, None, width, width, roots)


def _residual_norm(residual, block, post_weight, gate, scale, pre_weight, eps, activation):
    lib = _lib or _library()
    a = _norm_args(residual, block, post_weight, gate, scale, pre_weight, eps, activation, None)
    device, shape = block.device, block.shape
    held = torch.empty(2, *shape[:-1], dtype=torch.float32, device=device)
    total = _like(residual)
    out = None
    a.residual_out, a.roots = total.data_ptr(), held.data_ptr()
    if pre_weight is not None:
        out = _like(block)
        a.out = out.data_ptr()
    status = _on(device.index, lib.bps_residual_norm, a)
    if status:
        _checked(status)
    return ResidualNorm(total, out, held)


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, residual, block, post_weight, gate, scale, pre_weight, eps, activation):
        r = _residual_norm(residual, block, post_weight, gate, scale, pre_weight, eps, activation)
        ctx.save_for_backward(residual, block, post_weight, gate, scale, pre_weight, r.held)
        ctx.rest = eps, activation
        ctx.mark_non_differentiable(r.held)
        ctx.set_materialize_grads(False)
        return tuple(r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_residual, grad_out, _):
        residual, block, post_weight, gate, scale, pre_weight, held = ctx.saved_tensors
        if grad_residual is None and grad_out is None:
            return (None,) * 8
        plain = [None if g is None else g.contiguous() for g in (grad_residual, grad_out)]
        return *residual_norm_backward(residual, block, held, *plain, post_weight, gate, scale, pre_weight, *ctx.rest), None, None


def residual_norm(residual, block, post_weight=None, gate=None, scale=None, pre_weight=None, eps=1e-6, activation="sigmoid", stream=None):
    """A block's output joined to the residual stream, and what the next block begins with.  With N(v; w) = v / sqrt(mean(v^2) + eps) * w,
    residual + scale * activation(gate) * N(block; post_weight) is the sum, and N(sum; pre_weight) the next block's input.

    block, gate float32, bfloat16 or float16 [..., width]; residual of block's type or float32 [..., width]; post_weight, scale, pre_weight
    [width] of block's type or all float32.  post_weight None: the block's output is not normed; pre_weight None: there is no out; gate, scale
    None: 1.  activation "sigmoid" or "silu".  At most 16384 wide.
    -> ResidualNorm(residual, out, held): residual and out carry a gradient to all inputs; held [2, ...] is for residual_norm_backward."""
    if stream is not None:
        with _stream(stream, block.device):
            return residual_norm(residual, block, post_weight, gate, scale, pre_weight, eps, activation)
    _no_tangent(residual, block, post_weight, gate, scale, pre_weight)
    if torch.is_grad_enabled() and _any_grad(residual, block, post_weight, gate, scale, pre_weight):
        return ResidualNorm(*_ResidualNorm.apply(residual, block, post_weight, gate, scale, pre_weight, eps, activation))
    return _residual_norm(residual, block, post_weight, gate, scale, pre_weight, eps, activation)


def residual_norm_backward(residual, block, result, grad_residual=None, grad_out=None, post_weight=None, gate=None, scale=None, pre_weight=None, eps=1e-6, activation="sigmoid",
                           stream=None):
    """The gradient of residual_norm's residual and out for the same arguments; grad_* None: zero.  result: what residual_norm returned (or its
    `held`).  -> NormGrads(residual, block, post_weight, gate, scale, pre_weight), each of its input's type, None where there was none"""
    if stream is not None:
        with _stream(stream, block.device):
            return residual_norm_backward(residual, block, result, grad_residual, grad_out, post_weight, gate, scale, pre_weight, eps, activation)
    _no_tangent(residual, block, grad_residual, grad_out, post_weight, gate, scale, pre_weight)
    lib = _lib or _library()
    device = block.device
    held = _plain(result.held if isinstance(result, ResidualNorm) else result, "result", (2, *block.shape[:-1]), (torch.float32,), device)
    a = _norm_args(residual, block, post_weight, gate, scale, pre_weight, eps, activation, held)
    if grad_out is not None and pre_weight is None:
        raise ValueError("grad_out: without pre_weight there is no out")
    if grad_residual is not None:
        a.grad_residual_out, a.grad_residual_out_stride = grad_residual.data_ptr(), _row_step(grad_residual, "grad_residual", block.shape, (residual.dtype,), device)
    if grad_out is not None:
        a.grad_out, a.grad_out_stride = grad_out.data_ptr(), _row_step(grad_out, "grad_out", block.shape, (block.dtype,), device)
    gr, gb, gz, gp, gs, gn = (None if t is None else _like(t) for t in (residual, block, gate, post_weight, scale, pre_weight))
    a.grad_residual, a.grad_block, a.grad_gate = gr.data_ptr(), gb.data_ptr(), None if gz is None else gz.data_ptr()
    a.grad_residual_stride = a.grad_block_stride = a.grad_gate_stride = a.width
    a.grad_post_weight, a.grad_scale, a.grad_pre_weight = (None if g is None else g.data_ptr() for g in (gp, gs, gn))
    _call(device.index, lib.bps_residual_norm_backward, a, lib.bps_residual_norm_backward_workspace(a), device)
    return NormGrads(gr, gb, gp, gz, gs, gn)
