"""Sequence operators of librocket.so on torch tensors: what a trained head over
ROCKET features runs (the C ABI in include/rocket.h has the formulas).

Sequences are [n, steps, channels] tensors on the current GPU, float32,
bfloat16 or float16, with contiguous channels and any strides of series and
steps (a block of columns of a projection's output is taken as it is).
Statistics, weights, states and their gradients are float32 and contiguous.

    group_norm(x, groups, weight, bias)     -> y, mean, rstd
    group_norm_backward(dy, x, groups, mean, rstd, weight, bias) -> dx, dweight, dbias
    recurrence(v, f, o)                     -> y, h_last, states
    recurrence_backward(dy, v, f, states, o) -> dv, df, do, dh0
    recurrence_step(v, f, h, o)             -> y, h
    dropout(x, p, seed, call)               -> y
    dropout_backward(dy, p, seed, call)     -> dx

The backward passes are calls of their own: nothing here records itself for
torch's autograd (examples/window_head.py wraps them for it).  Where autograd
records, operands that require gradients are refused, since their gradients
would be lost: call under torch.no_grad(), or in a torch.autograd.Function.

Every call is asynchronous on `stream` (default: torch's current stream); what
it returns is allocated for that stream.  An operand that belongs to another
stream is the caller's to order and to keep alive (Tensor.record_stream).
"""
from __future__ import annotations

import ctypes

import torch

from . import rocket
from .rocket import CSequence, CSequenceShape

ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
EVERY = 128   # steps between the states a recurrence keeps (ROCKET_RECURRENCE_EVERY)
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_byref, _empty, _f32, _recording = ctypes.byref, torch.empty, torch.float32, torch.is_grad_enabled


def _dense(x):
    """A contiguous tensor of x's shape and type (the quickest way to one)."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


# The current GPU and the handle of its current stream; torch.cuda's own
# functions make objects of them, which takes as long as a small kernel.
_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    _stream = torch._C._cuda_getCurrentRawStream
else:
    def _stream(device):
        return torch.cuda.current_stream(device).cuda_stream


def _dtype(x, name: str) -> int:
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("%s must be a torch tensor on the GPU" % name)
    code = _DTYPES.get(x.dtype)
    if code is None:
        raise ValueError("%s must be float32, bfloat16 or float16" % name)
    if x.get_device() != _device():
        raise ValueError("%s must be on the current GPU" % name)
    return code


def _like(t, x, name: str):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch tensor on the GPU" % name)
    if t.dtype != x.dtype or t.shape != x.shape or t.get_device() != x.get_device():
        raise ValueError("%s must have the shape, type and device of the call's first sequence" % name)


def _written(*tensors):
    """Tells autograd that these tensors of the caller's were written: what it
    saved of them before is no longer what it was."""
    torch.autograd.graph.increment_version(tensors)


def _unrecorded(*operands):
    """Refuses operands whose gradients autograd would miss."""
    if _recording():
        for t in operands:
            if t is not None and t.requires_grad:
                raise ValueError("an operand requires gradients, which this call does not record: call it under "
                                 "torch.no_grad() or in a torch.autograd.Function")


def _sequence(t, name: str) -> CSequence:
    s = t.stride()
    if s[2] != 1 and t.shape[2] > 1:
        raise ValueError("%s must have contiguous channels" % name)
    return CSequence(t.data_ptr(), s[0], s[1])


def _shape(x, lengths, name: str) -> CSequenceShape:
    code = _dtype(x, name)
    if x.dim() != 3:
        raise ValueError("%s must be [n, steps, channels]" % name)
    n, steps, channels = x.shape
    if lengths is not None:
        if not isinstance(lengths, torch.Tensor) or not lengths.is_cuda:
            raise TypeError("lengths must be a torch tensor on the GPU")
        if (lengths.dtype != torch.int32 or lengths.shape != (n,) or lengths.get_device() != x.get_device()
                or not lengths.is_contiguous()):
            raise ValueError("lengths must be contiguous int32 [%d] on the sequences' GPU" % n)
        lengths = lengths.data_ptr()
    return CSequenceShape(n, steps, channels, code, lengths)


def _floats(t, shape, x, name: str):
    """The address of a contiguous float32 tensor of that shape; None stays None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch tensor on the GPU" % name)
    if t.dtype != torch.float32 or t.shape != shape or t.get_device() != x.get_device() or not t.is_contiguous():
        raise ValueError("%s must be contiguous float32 %s on the sequences' GPU" % (name, list(shape)))
    return t.data_ptr()


def _activation(name) -> int:
    code = ACTIVATIONS.get(name)
    if code is None:
        raise ValueError("activation must be one of %s" % ", ".join(sorted(ACTIVATIONS)))
    return code


def _workspace(size: int, device):
    """A workspace tensor (or None) and its address, on the current stream."""
    if size == 0:
        return None, None
    t = _empty(size, dtype=torch.uint8, device=device)
    return t, t.data_ptr()


def _norm_workspace(lib, shape, groups: int, backward: int) -> int:
    if not -(1 << 31) <= groups < 1 << 31:   # ctypes would take it modulo 2^32
        raise ValueError("groups must divide the channels")
    size = ctypes.c_int64()
    rocket._check(lib.rocket_group_norm_workspace(_byref(shape), groups, backward, _byref(size)),
                  "rocket_group_norm_workspace")
    return size.value


def group_norm(x, groups: int, weight=None, bias=None, *, eps: float = 1e-5, activation: str = "none", lengths=None,
               out=None, stream=None):
    """rocket_group_norm_forward: (y, mean [n, groups], rstd [n, groups]).
    `out` (may be x) takes y."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return group_norm(x, groups, weight, bias, eps=eps, activation=activation, lengths=lengths, out=out)
    lib = rocket.library()
    shape, act = _shape(x, lengths, "x"), _activation(activation)
    n, _, channels = x.shape
    w, b = _floats(weight, (channels,), x, "weight"), _floats(bias, (channels,), x, "bias")
    if out is not None:
        _like(out, x, "out")
    _unrecorded(x, weight, bias, out)
    given = out
    if out is None:
        out = _dense(x)
    size = _norm_workspace(lib, shape, groups, 0)
    mean = _empty(n, groups, dtype=_f32, device=x.device)
    rstd = _dense(mean)
    work, at = _workspace(size, x.device)
    status = lib.rocket_group_norm_forward(
        _byref(shape), groups, _byref(_sequence(x, "x")), w, b, eps, act, _byref(_sequence(out, "out")),
        mean.data_ptr(), rstd.data_ptr(), at, size, _stream(x.get_device()))
    rocket._check(status, "rocket_group_norm_forward")
    if given is not None:
        _written(given)
    return out, mean, rstd


def group_norm_backward(dy, x, groups: int, mean, rstd, weight=None, bias=None, *, activation: str = "none",
                        lengths=None, out=None, stream=None):
    """rocket_group_norm_backward: (dx, dweight, dbias), from the forward pass's
    mean and rstd.  `out` (may be dy or x) takes dx."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return group_norm_backward(dy, x, groups, mean, rstd, weight, bias, activation=activation,
                                       lengths=lengths, out=out)
    lib = rocket.library()
    shape, act = _shape(x, lengths, "x"), _activation(activation)
    _like(dy, x, "dy")
    n, _, channels = x.shape
    w, b = _floats(weight, (channels,), x, "weight"), _floats(bias, (channels,), x, "bias")
    if mean is None or rstd is None:
        raise TypeError("mean and rstd must be torch tensors on the GPU")
    size = _norm_workspace(lib, shape, groups, 1)
    m, r = _floats(mean, (n, groups), x, "mean"), _floats(rstd, (n, groups), x, "rstd")
    if out is not None:
        _like(out, x, "out")
    _unrecorded(dy, x, mean, rstd, weight, bias, out)
    given = out
    if out is None:
        out = _dense(x)
    dweight = _empty(channels, dtype=_f32, device=x.device)
    dbias = _dense(dweight)
    work, at = _workspace(size, x.device)
    status = lib.rocket_group_norm_backward(
        _byref(shape), groups, _byref(_sequence(dy, "dy")), _byref(_sequence(x, "x")), w, b, act, m, r,
        _byref(_sequence(out, "out")), dweight.data_ptr(), dbias.data_ptr(), at, size, _stream(x.get_device()))
    rocket._check(status, "rocket_group_norm_backward")
    if given is not None:
        _written(given)
    return out, dweight, dbias


def _recurrence_workspace(lib, shape) -> int:
    size = ctypes.c_int64()
    rocket._check(lib.rocket_recurrence_workspace(_byref(shape), _byref(size)), "rocket_recurrence_workspace")
    return size.value


def _optional(t, name: str):
    return None if t is None else _byref(_sequence(t, name))


def recurrence(v, f, o=None, *, h0=None, lengths=None, keep_states: bool = False, out=None, stream=None):
    """rocket_recurrence_forward: (y, h_last [n, channels], states), states
    [n, ceil(steps / EVERY), channels] with keep_states (for
    recurrence_backward), else None.  `out` (may be v, f or o) takes y."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return recurrence(v, f, o, h0=h0, lengths=lengths, keep_states=keep_states, out=out)
    lib = rocket.library()
    shape = _shape(v, lengths, "v")
    _like(f, v, "f")
    if o is not None:
        _like(o, v, "o")
    n, steps, channels = v.shape
    first = _floats(h0, (n, channels), v, "h0")
    if out is not None:
        _like(out, v, "out")
    _unrecorded(v, f, o, h0, out)
    given = out
    if out is None:
        out = _dense(v)
    size = _recurrence_workspace(lib, shape)
    h_last = _empty(n, channels, dtype=_f32, device=v.device)
    states = _empty(n, -(-steps // EVERY), channels, dtype=_f32, device=v.device) if keep_states else None
    work, at = _workspace(size, v.device)
    status = lib.rocket_recurrence_forward(
        _byref(shape), _byref(_sequence(v, "v")), _byref(_sequence(f, "f")), _optional(o, "o"), first,
        _byref(_sequence(out, "out")), h_last.data_ptr(), None if states is None else states.data_ptr(), at, size,
        _stream(v.get_device()))
    rocket._check(status, "rocket_recurrence_forward")
    if given is not None:
        _written(given)
    return out, h_last, states


def recurrence_backward(dy, v, f, states, o=None, *, dh_last=None, lengths=None, out=None, stream=None):
    """rocket_recurrence_backward: (dv, df, do, dh0 [n, channels]); do is None
    without an output gate.  `out`: the tensors that take dv, df (and do), for
    example blocks of a projection's gradient."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return recurrence_backward(dy, v, f, states, o, dh_last=dh_last, lengths=lengths, out=out)
    lib = rocket.library()
    shape = _shape(v, lengths, "v")
    _like(dy, v, "dy")
    _like(f, v, "f")
    if o is not None:
        _like(o, v, "o")
    n, steps, channels = v.shape
    if states is None:
        raise TypeError("states must be the forward pass's (keep_states)")
    kept = _floats(states, (n, -(-steps // EVERY), channels), v, "states")
    last = _floats(dh_last, (n, channels), v, "dh_last")
    wanted = 2 if o is None else 3
    given = out
    if out is None:
        out = [_dense(v) for _ in range(wanted)]
    elif len(out) != wanted:
        raise ValueError("out must hold %d tensors" % wanted)
    else:
        for t in out:
            _like(t, v, "out")
    _unrecorded(dy, v, f, states, o, dh_last, *out)
    size = _recurrence_workspace(lib, shape)
    dh0 = _empty(n, channels, dtype=_f32, device=v.device)
    work, at = _workspace(size, v.device)
    do = out[2] if o is not None else None
    status = lib.rocket_recurrence_backward(
        _byref(shape), _byref(_sequence(dy, "dy")), _byref(_sequence(v, "v")), _byref(_sequence(f, "f")),
        _optional(o, "o"), kept, last, _byref(_sequence(out[0], "out")), _byref(_sequence(out[1], "out")),
        _optional(do, "out"), dh0.data_ptr(), at, size, _stream(v.get_device()))
    rocket._check(status, "rocket_recurrence_backward")
    if given is not None:
        _written(*given)
    return out[0], out[1], do, dh0


def _matrix(t, name: str):
    """Address and row stride of [n, channels] with contiguous channels."""
    if t is None:
        return None, 0
    rows, channels = t.stride()
    if channels != 1 and t.shape[1] > 1:
        raise ValueError("%s must have contiguous channels" % name)
    return t.data_ptr(), rows


def recurrence_step(v, f, h, o=None, *, h_out=None, out=None, stream=None):
    """rocket_recurrence_step on [n, channels]: (y, the new state).  `h_out`
    (may be h) takes the new state, `out` takes y."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return recurrence_step(v, f, h, o, h_out=h_out, out=out)
    lib = rocket.library()
    code = _dtype(v, "v")
    if v.dim() != 2:
        raise ValueError("v must be [n, channels]")
    _like(f, v, "f")
    if o is not None:
        _like(o, v, "o")
    if h is None:
        raise TypeError("h must be a torch tensor on the GPU")
    at_h = _floats(h, v.shape, v, "h")
    if out is not None:
        _like(out, v, "out")
    at_out = _floats(h_out, v.shape, v, "h_out")
    _unrecorded(v, f, h, o, h_out, out)
    given = [t for t in (out, h_out) if t is not None]
    if out is None:
        out = _dense(v)
    if h_out is None:
        h_out = _dense(h)
        at_out = h_out.data_ptr()
    n, channels = v.shape
    status = lib.rocket_recurrence_step(n, channels, code, *_matrix(v, "v"), *_matrix(f, "f"), *_matrix(o, "o"), at_h,
                                        at_out, *_matrix(out, "out"), _stream(v.get_device()))
    rocket._check(status, "rocket_recurrence_step")
    if given:
        _written(*given)
    return out, h_out


def _rows(t, name: str):
    """(address, rows, columns, row stride) of a tensor whose elements lie in
    rows of equal distance, the last axis contiguous."""
    if t.is_contiguous():
        return t.data_ptr(), 1, t.numel(), t.numel()
    cols = t.shape[-1]
    if t.stride(-1) != 1 and cols > 1:
        raise ValueError("%s must have a contiguous last axis" % name)
    rows, stride = 1, None
    for size, step in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if stride is None:
            stride = step
        elif step != rows * stride:
            raise ValueError("%s must have rows of equal distance" % name)
        rows *= size
    return t.data_ptr(), rows, cols, cols if stride is None else stride


def dropout(x, p: float, seed: int, call: int = 0, *, residual=None, out=None, stream=None):
    """rocket_dropout over all elements of x in their order: dropout(x), plus
    `residual` where given.  `seed` and `call` are taken modulo 2^64.  `out`
    (may be x or residual) takes the result."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return dropout(x, p, seed, call, residual=residual, out=out)
    lib = rocket.library()
    code = _dtype(x, "x")
    if residual is not None:
        _like(residual, x, "residual")
    if out is not None:
        _like(out, x, "out")
    _unrecorded(x, residual, out)
    given = out
    if out is None:
        out = _dense(x)
    vx, vy = _rows(x, "x"), _rows(out, "out")
    vr = (None, 1, 0, 0) if residual is None else _rows(residual, "residual")
    rows, cols = max(vx[1], vr[1], vy[1]), x.numel()
    if rows > 1:   # a contiguous operand beside one in rows
        cols = x.shape[-1]
        vx, vr, vy = ((v[0], rows, cols, cols) if v[1] == 1 else v for v in (vx, vr, vy))
    status = lib.rocket_dropout(vx[0], vr[0], vy[0], rows, cols, vx[3], vr[3], vy[3], code, p, seed & (2 ** 64 - 1),
                                call & (2 ** 64 - 1), _stream(x.get_device()))
    rocket._check(status, "rocket_dropout")
    if given is not None:
        _written(given)
    return out


def dropout_backward(dy, p: float, seed: int, call: int = 0, *, out=None, stream=None):
    """The gradient of dropout with respect to x: the same map on dy (that of
    the residual is dy itself)."""
    return dropout(dy, p, seed, call, out=out, stream=stream)
