"""Operators of a recurrent language model over torch CUDA tensors, next to the embedding and the optimizer of `operators`.

    layer_norm        rows normed, with the gradients of rows, weight and bias
    dropout           with a mask that is drawn from a counter-based generator, twice, and never stored; adds a residual
    recurrence        h_t = f_t h_{t-1} + (1 - f_t) value_t with f = sigmoid(gate), over padded batches of sequences, and its gradient
    recurrence_step   one step of it for serving, the states updated in place

layer_norm, dropout and recurrence take part in autograd where an input needs a gradient (backwards; forward mode is an error).
Every call enqueues its kernels on the current stream of the tensors' device and returns without waiting; tensors that another
stream is still writing are ordered by the caller, as for torch's own operators.  Nothing is kept from one call for the next, so calls
may be made from several threads and on several streams, and captured (a captured `backward()`, as one through torch's own
operators, wants leaves that no eager graph still holds; torch.autograd.grad does not mind).  There is no fallback: a missing
library, a CPU tensor or a refused argument is an error.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Union

import torch
import torch.autograd.forward_ad as _forward

from . import binding as B
from .operators import _FLOATS, _current_stream, _need, _written

MARK = 8            # steps between the marks that the gradient of a recurrence starts from
_at = C.byref


def _device_of(x, name):
    index = x.get_device()
    if index < 0:
        raise ValueError(f"{name}: on {x.device}; no CUDA device: the operators have no CPU implementation")
    return index


def _wants_gradient(*tensors):
    """Whether autograd has to know of the call: backwards, or forwards (which it then refuses: a tangent would be lost silently)."""
    if torch.is_grad_enabled():
        for x in tensors:
            if x is not None and x.requires_grad:
                return True
    if _forward._current_level >= 0 and not torch.is_inference_mode_enabled():
        for x in tensors:
            if x is not None and _forward.unpack_dual(x).tangent is not None:
                return True
    return False


# ------------------------------------------------------------------ layer norm
def _flat(x, d, name):
    """x as rows of d elements that lie next to each other, (n, d)."""
    shape = x.shape
    if len(shape) == 0 or shape[-1] != d or d == 0 or x.dtype not in _FLOATS:
        raise ValueError(f"{name}: {tuple(shape)} of {x.dtype}; (..., {d}) of float32, bfloat16 or float16 goes")
    if len(shape) != 2:
        x = x.reshape(x.numel() // d, d)
    row, column = x.stride()
    if (column != 1 and d > 1) or (row < d and x.shape[0] > 1):      # transposed or broadcast: laid out first
        x = x.contiguous()
    return x


def _rows(x, n, d):
    return B.Rows(x.data_ptr(), x.stride(0) if n > 1 else d, d, _FLOATS[x.dtype])


def _norm_of(weight, bias, mean, rstd, n, d, eps, index):
    kind = _FLOATS.get(weight.dtype)
    if (kind is None or weight.dim() != 1 or weight.get_device() != index or not weight.is_contiguous()
            or bias is not None and (bias.shape != weight.shape or bias.dtype != weight.dtype or bias.get_device() != index
                                     or not bias.is_contiguous())):
        raise ValueError(f"weight and bias: contiguous ({d},) of one type, float32, bfloat16 or float16, on the rows' device; "
                         f"got {tuple(weight.shape)} of {weight.dtype} on {weight.device}"
                         + ("" if bias is None else f" and {tuple(bias.shape)} of {bias.dtype} on {bias.device}"))
    return B.Norm(weight.data_ptr(), None if bias is None else bias.data_ptr(), None if mean is None else mean.data_ptr(),
                  None if rstd is None else rstd.data_ptr(), n, kind, eps)


def layer_norm(x, weight, bias=None, eps: float = 1e-5, out=None, dtype=None, stats: bool = False):
    """(x - mean) / sqrt(variance + eps) * weight + bias over the last dimension.

    weight and bias (d,) are of one type.  The result is of x's type, or, where x is float32, of `dtype`.  stats: also the rows'
    means and 1 / sqrt(variance + eps), float32 (n,), which `layer_norm_gradient` takes."""
    if _wants_gradient(x, weight, bias):
        _need(out is None and not stats, "out and stats go without autograd alone")
        return _LayerNorm.apply(x, weight, bias, eps, dtype)
    return _layer_norm(x, weight, bias, eps, out, dtype, stats)


def _layer_norm(x, weight, bias, eps, out, dtype, stats):
    index = _device_of(x, "x")
    d = weight.numel()
    rows = _flat(x, d, "x")
    n, kind = rows.shape[0], _FLOATS[rows.dtype]
    mean = rstd = None
    if stats:
        mean, rstd = torch.empty((2, n), dtype=torch.float32, device=x.device)
    norm = _norm_of(weight, bias, mean, rstd, n, d, eps, index)
    given = out
    if out is None:
        # (of the rows, whose layout is that of a matrix whatever x's is)
        if dtype is None or dtype is x.dtype:
            out, to = torch.empty_like(rows, memory_format=torch.contiguous_format), kind
        else:
            to = _FLOATS.get(dtype)
            if to is None:
                raise ValueError("dtype: float32, bfloat16 or float16")
            out = torch.empty_like(rows, dtype=dtype, memory_format=torch.contiguous_format)
        ro = B.Rows(out.data_ptr(), d, d, to)
        shaped = out if x.dim() == 2 else out.view(x.shape)
    else:
        _need(out.shape == x.shape and out.dtype in _FLOATS and out.get_device() == index, "out: of x's shape, on its device")
        shaped = out
        out = out.view(n, d)
        _need((out.stride(1) == 1 or d == 1) and (out.stride(0) >= d or n < 2), "out: rows of columns next to each other, apart")
        ro = _rows(out, n, d)
    rc = B.lib().tensair_layer_norm(_at(norm), _at(B.Rows(rows.data_ptr(), rows.stride(0) if n > 1 else d, d, kind)), _at(ro),
                                    _current_stream(index))
    if rc:
        B._check(rc, "tensair_layer_norm")
    if given is not None:
        _written(given)
    return (shaped, mean, rstd) if stats else shaped


def layer_norm_gradient(grad, x, weight, mean, rstd, bias: bool = True, params: bool = True):
    """(dx, dweight, dbias) of `layer_norm` for the gradient of its result, with the rows' statistics that it gave.

    bias False: no dbias; params False: neither dweight nor dbias (None in their places)."""
    index = _device_of(x, "x")
    d = weight.numel()
    rows = _flat(x, d, "x")
    n = rows.shape[0]
    _need(grad.shape == x.shape and grad.get_device() == index, "grad: of x's shape, on its device")
    for s in (mean, rstd):
        if s.shape != (n,) or s.dtype != torch.float32 or s.get_device() != index or not s.is_contiguous():
            raise ValueError(f"mean and rstd: contiguous float32 of ({n},) on the rows' device")
    grad = _flat(grad, d, "grad")
    norm = _norm_of(weight, None, mean, rstd, n, d, 0.0, index)
    dx = torch.empty_like(rows, memory_format=torch.contiguous_format)
    if x.dim() != 2:
        dx = dx.view(x.shape)
    dw = torch.empty_like(weight) if params else None
    db = torch.empty_like(weight) if params and bias else None
    workspace, size = None, 0
    lib = B.lib()
    if params:
        need = C.c_uint64(0)
        lib.tensair_norm_workspace_bytes(n, d, _at(need))
        size = need.value
        # out of the allocator of the current stream, or of the graph that captures the call: nobody else has it meanwhile
        workspace = torch.empty(max(1, size), dtype=torch.uint8, device=x.device)
    rc = lib.tensair_layer_norm_gradient(_at(norm), _at(_rows(grad, n, d)), _at(_rows(rows, n, d)), _at(B.Rows(dx.data_ptr(), d, d, _FLOATS[dx.dtype])),
                                         None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
                                         None if workspace is None else workspace.data_ptr(), size, _current_stream(index))
    if rc:
        B._check(rc, "tensair_layer_norm_gradient")
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, dtype):
        y, mean, rstd = _layer_norm(x, weight, bias, eps, None, dtype, True)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, weight, mean, rstd = ctx.saved_tensors
        _, dw, db = ctx.needs_input_grad[:3]
        dx, dweight, dbias = layer_norm_gradient(grad, x, weight, mean, rstd, bias=db, params=dw or db)
        return dx, dweight, dbias, None, None


# ------------------------------------------------------------------ dropout
def dropout(x, p: float, seed: int, call: Union[int, torch.Tensor], residual=None, out=None):
    """x / (1 - p) where the element's word of the generator reaches p 2^32, else 0; plus `residual`, of x's shape and type.

    seed and call fix the mask: the words are those of Philox4x32-10 of (element / 4, call) under the key `seed`.  Every mask that is to
    differ needs a number of its own, as call = step * layers + layer.  call may be an int64 tensor of one element on x's device, which
    is read when the stream gets there: a captured call needs that, and something in the graph that counts it up."""
    if _wants_gradient(x, residual):
        _need(out is None, "out goes without autograd alone")
        return _Dropout.apply(x, residual, p, seed, call)
    return _dropout(x, p, seed, call, residual, out)


def _dropout(x, p, seed, call, residual, out):
    index = _device_of(x, "x")
    kind = _FLOATS.get(x.dtype)
    if kind is None:
        raise ValueError(f"x: {x.dtype}; float32, bfloat16 or float16 goes")
    given = out
    if not x.is_contiguous():
        x = x.contiguous()
    if residual is not None:
        if residual.shape != x.shape or residual.dtype != x.dtype or residual.get_device() != index:
            raise ValueError(f"residual: {tuple(residual.shape)} of {residual.dtype} on {residual.device}, for x {tuple(x.shape)} of {x.dtype}")
        if not residual.is_contiguous():
            residual = residual.contiguous()
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype or out.get_device() != index or not out.is_contiguous():
        raise ValueError("out: contiguous, of x's shape and type, on its device")
    number, at = call, None
    if isinstance(call, torch.Tensor):
        _need(call.dtype == torch.int64 and call.numel() == 1 and call.get_device() == index, "call: an int, or one int64 on x's device")
        number, at = 0, call.data_ptr()
    _need(0 <= number < 1 << 56 and 0 <= seed < 1 << 64, "call and seed: 0 .. 2^56 - 1 and 0 .. 2^64 - 1")
    h = B.DropoutCall(x.data_ptr(), None if residual is None else residual.data_ptr(), out.data_ptr(), x.numel(), p, seed, number, at, kind, 0)
    rc = B.lib().tensair_dropout(_at(h), _current_stream(index))
    if rc:
        B._check(rc, "tensair_dropout")
    if given is not None:
        _written(given)
    return out


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, call):
        ctx.p, ctx.seed = p, seed
        if isinstance(call, torch.Tensor):
            call = call.clone()          # it will have been counted up when the gradient comes
            ctx.save_for_backward(call)
            ctx.call = None
        else:
            ctx.call = call
        return _dropout(x, p, seed, call, residual, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        call = ctx.saved_tensors[0] if ctx.call is None else ctx.call
        dx = _dropout(grad, ctx.p, ctx.seed, call, None, None) if ctx.needs_input_grad[0] else None
        return dx, grad if ctx.needs_input_grad[1] else None, None, None, None


# ------------------------------------------------------------------ recurrence
def _step_rows(x, shape, kind, index, name):
    """(x, its Steps): [B, T, d] with channels next to each other, whatever the strides of the others are."""
    if x.shape != shape or x.dtype != kind or x.get_device() != index:
        raise ValueError(f"{name}: {tuple(x.shape)} of {x.dtype} on {x.device}; {tuple(shape)} of {kind} on device {index} goes")
    batch, step, channel = x.stride()
    if channel != 1 and shape[2] > 1:
        x = x.contiguous()
        batch, step, _ = x.stride()
    return x, B.Steps(x.data_ptr(), batch, step)


def _states(x, shape, index, name):
    if x is None:
        return None
    if x.shape != shape or x.dtype != torch.float32 or x.get_device() != index or not x.is_contiguous():
        raise ValueError(f"{name}: contiguous float32 of {tuple(shape)} on device {index}, not {tuple(x.shape)} of {x.dtype} on {x.device}")
    return x.data_ptr()


def _sequences(gate, value, lengths):
    index = _device_of(value, "value")
    shape = value.shape
    if len(shape) != 3 or value.dtype not in _FLOATS:
        raise ValueError(f"value: {tuple(shape)} of {value.dtype}; (B, T, d) of float32, bfloat16 or float16 goes")
    gate, g = _step_rows(gate, shape, value.dtype, index, "gate")
    value, v = _step_rows(value, shape, value.dtype, index, "value")
    n = None
    if lengths is not None:
        if lengths.shape != shape[:1] or lengths.dtype != torch.int32 or lengths.get_device() != index or not lengths.is_contiguous():
            raise ValueError(f"lengths: contiguous int32 of ({shape[0]},) on device {index}")
        n = lengths.data_ptr()
    return gate, value, B.Sequences(g, v, n, shape[0], shape[1], shape[2], _FLOATS[value.dtype]), index


def recurrence(gate, value, state=None, lengths=None, out=None, marks: bool = False):
    """(h, last): h_t = f_t h_{t-1} + (1 - f_t) value_t with f = sigmoid(gate), channel by channel, for gate and value (B, T, d).

    state (B, d) float32 is what h begins with (default 0); last, float32, is h after the last step.  lengths (int32, B): the steps of
    each sequence from there on are padding: they are not used, h is zero there and the state stays as it is.  Nothing is rounded
    between steps; h is rounded to value's type when it is stored.  marks: also the states that `recurrence_gradient` starts from."""
    if _wants_gradient(gate, value, state):
        _need(out is None and not marks, "out and marks go without autograd alone")
        return _Recurrence.apply(gate, value, state, lengths)
    return _recurrence(gate, value, state, lengths, out, marks)


def _recurrence(gate, value, state, lengths, out, marks):
    gate, value, seq, index = _sequences(gate, value, lengths)
    shape = value.shape
    states = (shape[0], shape[2])
    first = _states(state, states, index, "state")
    given = out
    if out is None:
        out = torch.empty(shape, dtype=value.dtype, device=value.device)
    else:
        _need(out.dim() == 3 and (out.stride(2) == 1 or shape[2] == 1), "out: channels next to each other")
    out, o = _step_rows(out, shape, value.dtype, index, "out")
    last = torch.empty(states, dtype=torch.float32, device=value.device)
    kept = torch.empty((shape[0], -(-shape[1] // MARK), shape[2]), dtype=torch.float32, device=value.device) if marks else None
    rc = B.lib().tensair_recurrence(_at(seq), first, _at(o), last.data_ptr(), None if kept is None else kept.data_ptr(),
                                    _current_stream(index))
    if rc:
        B._check(rc, "tensair_recurrence")
    if given is not None:
        _written(given)
    return (out, last, kept) if marks else (out, last)


def recurrence_gradient(grad, gate, value, marks, lengths=None, grad_state=None, out=None):
    """(dgate, dvalue, dstate) of `recurrence` for the gradients of its h (`grad`) and of its last states (`grad_state`, default 0),
    from the marks that it left.  out: tensors for dgate and dvalue, of value's shape with channels next to each other (so they can be two
    halves of one)."""
    gate, value, seq, index = _sequences(gate, value, lengths)
    shape = value.shape
    states = (shape[0], shape[2])
    grad, g = _step_rows(grad, shape, value.dtype, index, "grad")
    _states(marks, (shape[0], -(-shape[1] // MARK), shape[2]), index, "marks")
    end = _states(grad_state, states, index, "grad_state")
    given = out
    if out is None:
        out = torch.empty((2, *shape), dtype=value.dtype, device=value.device).unbind()
    else:
        _need(all(x.dim() == 3 and (x.stride(2) == 1 or shape[2] == 1) for x in out), "out: channels next to each other")
    dgate, dg = _step_rows(out[0], shape, value.dtype, index, "out[0]")
    dvalue, dv = _step_rows(out[1], shape, value.dtype, index, "out[1]")
    dstate = torch.empty(states, dtype=torch.float32, device=value.device)
    rc = B.lib().tensair_recurrence_gradient(_at(seq), _at(g), end, marks.data_ptr(), _at(dg), _at(dv), dstate.data_ptr(), _current_stream(index))
    if rc:
        B._check(rc, "tensair_recurrence_gradient")
    if given is not None:
        _written(given)
    return dgate, dvalue, dstate


class _Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, value, state, lengths):
        out, last, marks = _recurrence(gate, value, state, lengths, None, True)
        ctx.save_for_backward(gate, value, marks, lengths)
        ctx.set_materialize_grads(False)
        return out, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad, grad_last):
        gate, value, marks, lengths = ctx.saved_tensors
        if grad is None:
            grad = torch.zeros(value.shape[2], dtype=value.dtype, device=value.device).expand(value.shape)
        if grad_last is not None:
            grad_last = grad_last.contiguous()
        dgate, dvalue, dstate = recurrence_gradient(grad, gate, value, marks, lengths, grad_last)
        return dgate, dvalue, dstate if ctx.needs_input_grad[2] else None, None


def recurrence_step(gate, value, state, out=None):
    """The next step of B streams: gate and value (B, d); state (B, d) float32 is updated in place.  Returns h, of value's type."""
    _need(not _wants_gradient(gate, value, state), "recurrence_step has no gradient: `recurrence` over one step has")
    index = _device_of(value, "value")
    shape, dtype = value.shape, value.dtype
    kind = _FLOATS.get(dtype)
    if kind is None or len(shape) != 2 or gate.shape != shape or gate.dtype is not dtype or gate.get_device() != index:
        raise ValueError(f"gate and value: (B, d) of one type, float32, bfloat16 or float16, on one device; got {tuple(gate.shape)} of {gate.dtype} "
                         f"on {gate.device} and {tuple(shape)} of {dtype} on {value.device}")
    h = _states(state, shape, index, "state")
    _need(h is not None, "state: None")
    streams, d = shape
    gate_row, column = gate.stride()
    if column != 1 and d > 1:
        gate = gate.contiguous()
        gate_row = d
    value_row, column = value.stride()
    if column != 1 and d > 1:
        value = value.contiguous()
        value_row = d
    given = out
    if out is None:
        out, out_row = torch.empty_like(value, memory_format=torch.contiguous_format), d
    else:
        out_row, column = out.stride() if out.dim() == 2 else (0, 0)
        if out.shape != shape or out.dtype is not dtype or out.get_device() != index or (column != 1 and d > 1):
            raise ValueError("out: of value's shape and type, on its device, channels next to each other")
    seq = B.Sequences((gate.data_ptr(), gate_row, 0), (value.data_ptr(), value_row, 0), None, streams, 1, d, kind)
    rc = B.lib().tensair_recurrence_step(_at(seq), h, _at(B.Steps(out.data_ptr(), out_row, 0)), _current_stream(index))
    if rc:
        B._check(rc, "tensair_recurrence_step")
    _written(state if given is None else (state, given))
    return out
