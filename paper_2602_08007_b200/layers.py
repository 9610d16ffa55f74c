"""Layer operators through the tsr_norm / tsr_linear / tsr_dropout calls (see include/tsr.h): the norms, linear layers and dropout
whose gradients the optimizer steps.

Two forms.  norm_forward, norm_backward, linear_forward, linear_backward, dropout_forward and dropout_backward marshal arguments to the C calls: they
take tensors as they lie (last dimension contiguous; the others collapse to rows of one pitch) and refuse anything else.
layer_norm, rms_norm, linear and dropout are differentiable torch functions over them, which copy what does not lie that way.  They have a first derivative
only (no second one, no vmap, no forward mode) and ignore autocast: an input and its weight have one type.

All of them run on torch's current stream of the tensors' device, or on `stream`; results and scratch come from torch's allocator on that
stream, so calls on different streams share nothing and a capture keeps its own.  Tensors of the caller need record_stream
where they are dropped while another stream than their own uses them."""
from __future__ import annotations

import contextlib
import ctypes
import functools
import inspect
import threading
import weakref
from typing import Optional

import torch

from .binding import (
    TSR_ACT_GELU, TSR_ACT_GELU_TANH, TSR_ACT_NONE, TSR_ACT_RELU, TSR_ACT_SILU, TSR_BF16, TSR_F32, TSR_OK,
    DropoutDesc, LinearDesc, LinearGrads, LinearIO, Matrix, NormDesc, TsrError, lib,
)

_DTYPE = {torch.float32: TSR_F32, torch.bfloat16: TSR_BF16}
ACTIVATIONS = {None: TSR_ACT_NONE, "none": TSR_ACT_NONE, "relu": TSR_ACT_RELU, "gelu": TSR_ACT_GELU, "gelu_tanh": TSR_ACT_GELU_TANH, "silu": TSR_ACT_SILU}
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_NO_MATRIX = Matrix(None, 0)


class Dropout:
    """Which entries fall: probability p, a seed, an offset (another one for every use of a seed: layer, step), and optionally an int64 tensor
    of one element on the device that is added to the offset when a kernel runs (advance it between the replays of a captured graph, not between
    a forward pass and its backward).  The same Dropout draws the same entries in the forward and the backward call."""

    def __init__(self, p: float, seed: int, offset: int = 0, step: Optional[torch.Tensor] = None):
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie in [0, 1]")
        if step is not None and (step.dtype != torch.int64 or step.numel() != 1 or not step.is_cuda):
            raise ValueError("step must be an int64 tensor of one element on a CUDA device")
        self.p, self.seed, self.offset, self.step = float(p), int(seed), int(offset), step
        self.desc = DropoutDesc(self.p, 0, self.seed & (2**64 - 1), self.offset & (2**64 - 1), step.data_ptr() if step is not None else None)


_NO_DROPOUT = DropoutDesc(0.0, 0, 0, 0, None)


def _layout(t: torch.Tensor):
    """(rows, columns, pitch) of a tensor whose last dimension is contiguous and whose others collapse to rows of one pitch, or None."""
    if t.dim() == 0:
        return None
    cols = t.shape[-1]
    if t.is_contiguous():
        if cols:
            return t.numel() // cols, cols, cols
        rows = 1
        for n in t.shape[:-1]:
            rows *= n
        return rows, 0, 0
    if cols > 1 and t.stride(-1) != 1:
        return None
    rows, ld = 1, None
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n != 1 and rows * n:
            if ld is None:
                ld = s
            elif s != ld * rows:
                return None
        rows *= n
    if rows <= 1 or ld is None:
        ld = cols
    return (rows, cols, ld) if ld >= cols else None


def _matrix(t: torch.Tensor, what: str, shape, dtype: torch.dtype, device: torch.device) -> Matrix:
    if t.dtype != dtype or t.device != device:
        raise ValueError("%s must be a %s tensor on %s" % (what, dtype, device))
    if t.shape != shape:
        raise ValueError("%s must have the shape %s, not %s" % (what, tuple(shape), tuple(t.shape)))
    if t.is_contiguous():
        return Matrix(t.data_ptr(), shape[-1])
    m = _layout(t)
    if m is None:
        raise ValueError(_ROWS % what)
    return Matrix(t.data_ptr(), m[2])


_ROWS = "%s must have a contiguous last dimension and rows of one pitch that do not overlap"


def _vector(t: Optional[torch.Tensor], what: str, n: int, device: torch.device):
    """(pointer, type) of an optional vector."""
    if t is None:
        return None, TSR_F32
    kind = _DTYPE.get(t.dtype)
    if kind is None or t.shape != (n,) or t.device != device or not t.is_contiguous():
        raise ValueError("%s must be a contiguous FP32 or BF16 vector of %d elements on %s" % (what, n, device))
    return t.data_ptr(), kind


def _input(x: torch.Tensor, what: str):
    """(type, (rows, columns, pitch), device) of a call's leading tensor."""
    kind = _DTYPE.get(x.dtype)
    if kind is None or not x.is_cuda:
        raise ValueError("%s must be an FP32 or BF16 tensor on a CUDA device" % what)
    m = _layout(x)
    if m is None:
        raise ValueError(_ROWS % what)
    return kind, m, x.device


def _dropout_desc(drop: Optional[Dropout], device: torch.device) -> DropoutDesc:
    if drop is None:
        return _NO_DROPOUT
    if drop.step is not None and drop.step.device != device:
        raise ValueError("the step of a Dropout must be on %s" % device)
    return drop.desc


def _activation(a) -> int:
    if isinstance(a, int):
        return a
    if a not in ACTIVATIONS:
        raise ValueError("activation must be one of %s" % sorted(k for k in ACTIVATIONS if k))
    return ACTIVATIONS[a]


def _placed(call):
    """Runs the call on the tensors' device and on `stream`, whatever is current.  (A wrapper that steps aside where nothing is to be changed: small
    calls are bound by what the host does, and a context costs 1 us.)"""
    @functools.wraps(call)
    def placed(*args, stream=None, **kwargs):
        device = (args[0] if args else kwargs[first]).device
        if stream is None:
            if device.index is None or device.index == _current_device():
                return call(*args, **kwargs)
            with torch.cuda.device(device):
                return call(*args, **kwargs)
        if stream.device != device:
            raise ValueError("stream must belong to %s" % device)
        with torch.cuda.stream(stream):
            return call(*args, **kwargs)

    first = next(iter(inspect.signature(call).parameters))
    return placed


def _check(status: int, what: str):
    if status != TSR_OK:
        raise TsrError(status, what)


def _scratch(size: int, device: torch.device):
    """(tensor to hold on to, 256-byte aligned address)"""
    if not size:
        return None, None
    t = torch.empty(size + 256, dtype=torch.uint8, device=device)
    return t, (t.data_ptr() + 255) // 256 * 256


def _like(t: torch.Tensor) -> torch.Tensor:
    """A new contiguous tensor of t's shape and type (empty_like costs half of what the other ways to make one do)."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


# ---- the C calls ----------------------------------------------------------------------------------------------------------

# (`stream` is taken by the wrapper)

@_placed
def norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, center: bool = True,
                 out: Optional[torch.Tensor] = None):
    """(y, stats): the norm of every row of x (its last dimension) with weight and bias, and (mean, 1 / deviation) per row in FP32 for
    norm_backward.  center False: without the mean.  out: where y goes; x itself is allowed.  stream: as in every call here."""
    kind, (rows, cols, ld), dev = _input(x, "x")
    w, wt = _vector(weight, "weight", cols, dev)
    b, bt = _vector(bias, "bias", cols, dev)
    if wt != bt:
        if w is not None and b is not None:
            raise ValueError("weight and bias must have the same type")
        wt = wt if w is not None else bt
    if out is None:
        out = _like(x)
        my = Matrix(out.data_ptr(), cols)
    else:
        my = _matrix(out, "out", x.shape, x.dtype, dev)
    stats = x.new_empty((rows, 2), dtype=torch.float32)
    desc = NormDesc(rows, cols, kind, wt, TSR_F32, 1 if center else 0, 0, eps)
    _check(lib().tsr_norm_forward(desc, Matrix(x.data_ptr(), ld), w, b, my, stats.data_ptr(), _current_stream(dev.index)), "tsr_norm_forward")
    return out, stats


@_placed
def norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], stats: torch.Tensor, center: bool = True, bias: bool = True,
                  dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, accumulate: bool = False,
                  want_dx: bool = True, want_dweight: Optional[bool] = None):
    """(dx, dweight, dbias) for the dy of norm_forward's y.  dx, dweight, dbias: where they go (dx may be dy itself); otherwise they are new, dweight and
    dbias in FP32.  accumulate: the given dweight and dbias are added to.  bias, want_dx, want_dweight: what is not wanted is None (dweight is
    wanted where there is a weight)."""
    kind, (rows, cols, ld), dev = _input(x, "x")
    mdy = _matrix(dy, "dy", x.shape, x.dtype, dev)
    w, wt = _vector(weight, "weight", cols, dev)
    if stats.dtype != torch.float32 or stats.device != dev or tuple(stats.shape) != (rows, 2) or not stats.is_contiguous():
        raise ValueError("stats must be the second result of norm_forward")
    if want_dweight is None:
        want_dweight = weight is not None or dweight is not None
    if accumulate and ((want_dweight and dweight is None) or (bias and dbias is None)):
        raise ValueError("accumulate needs the dweight and dbias to add to")
    if not want_dx:
        dx, mdx = None, _NO_MATRIX
    elif dx is None:
        dx = _like(x)
        mdx = Matrix(dx.data_ptr(), cols)
    else:
        mdx = _matrix(dx, "dx", x.shape, x.dtype, dev)
    def vector():
        return torch.empty_like(weight) if wt == TSR_F32 and weight is not None else x.new_empty(cols, dtype=torch.float32)

    dweight = (vector() if dweight is None else dweight) if want_dweight else None
    dbias = (vector() if dbias is None else dbias) if bias else None
    gw, gwt = _vector(dweight, "dweight", cols, dev)
    gb, gbt = _vector(dbias, "dbias", cols, dev)
    if gw is not None and gb is not None and gwt != gbt:
        raise ValueError("dweight and dbias must have the same type")
    desc = NormDesc(rows, cols, kind, wt, gwt if gw is not None else gbt, 1 if center else 0, 1 if accumulate else 0, 0.0)
    hold, at, size = None, None, ctypes.c_size_t()
    if want_dweight or bias:
        _check(lib().tsr_norm_workspace_bytes(desc, size), "tsr_norm_workspace_bytes")
        hold, at = _scratch(size.value, dev)
    _check(lib().tsr_norm_backward(desc, mdy, Matrix(x.data_ptr(), ld), w, stats.data_ptr(), mdx, gw, gb, at, size.value, _current_stream(dev.index)), "tsr_norm_backward")
    return dx, dweight, dbias


@_placed
def linear_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, activation=None, dropout: Optional[Dropout] = None,
                   residual: Optional[torch.Tensor] = None, keep_pre: bool = False, out: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None):
    """(y, pre): y = residual + dropout(act(x weight^T + bias)), and the argument of the activation where keep_pre asks for it or `pre` says where it
    goes (None otherwise).  weight: (outs, ins).  activation: None, "relu", "gelu", "gelu_tanh" or "silu".  out: where y goes;
    the residual itself is allowed."""
    kind, (rows, ins, ld), dev = _input(x, "x")
    if weight.dim() != 2 or weight.shape[1] != ins:
        raise ValueError("weight must be a matrix with x's last dimension as its columns")
    outs = weight.shape[0]
    shape = x.shape[:-1] + (outs,)
    mw = _matrix(weight, "weight", weight.shape, x.dtype, dev)
    b, bt = _vector(bias, "bias", outs, dev)
    mres = _matrix(residual, "residual", shape, x.dtype, dev) if residual is not None else _NO_MATRIX
    if out is None:
        out = x.new_empty(shape) if residual is None else _like(residual)
        my = Matrix(out.data_ptr(), outs)
    else:
        my = _matrix(out, "out", shape, x.dtype, dev)
    if pre is not None:
        mpre = _matrix(pre, "pre", shape, x.dtype, dev)
    elif keep_pre:
        pre = _like(out)
        mpre = Matrix(pre.data_ptr(), outs)
    else:
        mpre = _NO_MATRIX
    desc = LinearDesc(rows, ins, outs, kind, bt, TSR_F32, TSR_F32, _activation(activation), 0, _dropout_desc(dropout, dev))
    io = LinearIO(Matrix(x.data_ptr(), ld), mw, mres, mpre, my, b)
    size = ctypes.c_size_t()
    _check(lib().tsr_linear_forward_bytes(desc, io, size), "tsr_linear_forward_bytes")
    hold, at = _scratch(size.value, dev)
    _check(lib().tsr_linear_forward(desc, io, at, size.value, _current_stream(dev.index)), "tsr_linear_forward")
    return out, pre


@_placed
def linear_backward(dy: torch.Tensor, x: Optional[torch.Tensor], weight: torch.Tensor, pre: Optional[torch.Tensor] = None, activation=None,
                    dropout: Optional[Dropout] = None, dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                    accumulate: bool = False, want_dx: bool = True, want_dweight: bool = True):
    """(dx, dweight, dbias) for the dy of linear_forward's y; the residual's gradient is dy itself.  dx, dweight: where they go; otherwise they are
    new, in the type of x.  dweight may be FP32 or BF16 with any row pitch: the G of a TSR block, for instance.  dbias: where it goes, or None: not
    wanted.  accumulate: the given dweight and dbias are added to.  What want_dx and want_dweight leave out is None."""
    kind, (rows, outs, ld), dev = _input(dy, "dy")
    if weight.dim() != 2 or weight.shape[0] != outs:
        raise ValueError("weight must be a matrix with dy's last dimension as its rows")
    ins = weight.shape[1]
    shape = dy.shape[:-1] + (ins,)
    act = _activation(activation)
    mw = _matrix(weight, "weight", weight.shape, dy.dtype, dev)
    if want_dweight and x is None:
        raise ValueError("dweight needs x")
    mx = _matrix(x, "x", shape, dy.dtype, dev) if x is not None else _NO_MATRIX
    if act != TSR_ACT_NONE and pre is None:
        raise ValueError("a layer with an activation needs pre (linear_forward with keep_pre)")
    mpre = _matrix(pre, "pre", dy.shape, dy.dtype, dev) if act != TSR_ACT_NONE else _NO_MATRIX
    if accumulate and want_dweight and dweight is None:
        raise ValueError("accumulate needs the dweight to add to")
    gb, gbt = _vector(dbias, "dbias", outs, dev)
    if not want_dx:
        dx, mdx = None, _NO_MATRIX
    elif dx is None:
        dx = dy.new_empty(shape) if x is None else _like(x)
        mdx = Matrix(dx.data_ptr(), ins)
    else:
        mdx = _matrix(dx, "dx", shape, dy.dtype, dev)
    gwt = TSR_F32
    if not want_dweight:
        dweight, mdw = None, _NO_MATRIX
    else:
        if dweight is None:
            dweight = _like(weight)
        gwt = _DTYPE.get(dweight.dtype)
        if gwt is None:
            raise ValueError("dweight must be FP32 or BF16")
        mdw = _matrix(dweight, "dweight", weight.shape, dweight.dtype, dev)
    desc = LinearDesc(rows, ins, outs, kind, TSR_F32, gwt, gbt, act, 1 if accumulate else 0, _dropout_desc(dropout, dev))
    io = LinearGrads(Matrix(dy.data_ptr(), ld), mx, mw, mpre, mdx, mdw, gb)
    size = ctypes.c_size_t()
    _check(lib().tsr_linear_backward_bytes(desc, io, size), "tsr_linear_backward_bytes")
    hold, at = _scratch(size.value, dev)
    _check(lib().tsr_linear_backward(desc, io, at, size.value, _current_stream(dev.index)), "tsr_linear_backward")
    return dx, dweight, dbias


@_placed
def dropout_forward(x: torch.Tensor, dropout: Dropout, residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + dropout(x); out: where it goes (x or the residual itself is allowed)."""
    kind, (rows, cols, ld), dev = _input(x, "x")
    mres = _matrix(residual, "residual", x.shape, x.dtype, dev) if residual is not None else _NO_MATRIX
    if out is None:
        out = _like(x)
        my = Matrix(out.data_ptr(), cols)
    else:
        my = _matrix(out, "out", x.shape, x.dtype, dev)
    _check(lib().tsr_dropout(_dropout_desc(dropout, dev), kind, rows, cols, Matrix(x.data_ptr(), ld), mres, my, _current_stream(dev.index)), "tsr_dropout")
    return out


def dropout_backward(dy: torch.Tensor, dropout: Dropout, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The gradient of dropout_forward's x; the residual's is dy itself."""
    return dropout_forward(dy, dropout, out=out, stream=stream)


def layer_poll_status(device=None) -> int:
    """Reads and clears the status word of the layer calls on a device (TSR_OK unless a bounded wait ran out); synchronises the current stream."""
    with torch.cuda.device(device) if device is not None else contextlib.nullcontext():
        status = ctypes.c_int32()
        _check(lib().tsr_layer_poll_status(ctypes.byref(status), _current_stream(torch.cuda.current_device())), "tsr_layer_poll_status")
    return status.value


# ---- differentiable forms -------------------------------------------------------------------------------------------------

def _lies(t: torch.Tensor) -> torch.Tensor:
    """The tensor, or a contiguous copy where its layout is not one the calls take (an expanded gradient, a transposed input)."""
    return t if _layout(t) is not None else t.contiguous()


_EAGER = weakref.WeakSet()     # graphs (their contexts) that were made on the default stream, outside of a capture, and still live
_EAGER_LOCK = threading.RLock()  # (one that a destructor which runs inside may take again)


def _on_default_stream(t: torch.Tensor) -> bool:
    return not t.is_cuda or _current_stream(t.device.index) == 0


def _leaves(tensors, nodes=()) -> dict:
    """The leaves that the graphs of tensors and nodes end in, by id (and held, so that the ids stay theirs)."""
    found, seen, todo = {id(t): t for t in tensors if t.is_leaf}, set(), [t.grad_fn for t in tensors] + list(nodes)
    while todo:
        node = todo.pop()
        if node is None or node in seen:
            continue
        seen.add(node)
        if type(node).__name__ == "AccumulateGrad":
            found[id(node.variable)] = node.variable
        try:
            todo += [n for n, _ in node.next_functions]
        except RuntimeError:      # (a call that another thread is still in: its node has no edges yet)
            pass
    return found


def _guard_capture(ctx, graph: bool, *tensors):
    """Torch keeps one gradient accumulator per leaf, bound to the stream of the graph that made it.  A backward pass that is captured while
    a graph of the same leaf from the default stream is alive reaches that stream from within the capture, which the default stream does not take, and
    ends the process.  So the capture is refused here, where it can still be an error: for every leaf that the inputs of these functions are or
    were computed from, beside every such graph that a call of these functions is part of.  (Graphs of other functions alone are not seen.  Other streams join the
    capture; a graph of theirs counts where it may share accumulators with one of the default stream.)  graph: whether torch records one."""
    tensors = [t for t in tensors if graph and t is not None and t.requires_grad]
    if not tensors:
        return
    if torch.cuda.is_current_stream_capturing():
        with _EAGER_LOCK:
            living = list(_EAGER)
        if living and _leaves(tensors).keys() & _leaves((), living).keys():
            raise RuntimeError("a graph of this tensor from outside of the capture is still alive: drop its outputs before capturing")
        return
    with _EAGER_LOCK:
        if len(_EAGER) or _on_default_stream(tensors[0]):
            _EAGER.add(ctx)


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, graph, x, weight, bias, eps, center):
        _guard_capture(ctx, graph, x, weight, bias)
        x = _lies(x)
        weight, bias = (None if t is None else t.contiguous() for t in (weight, bias))
        y, stats = norm_forward(x, weight, bias, eps=eps, center=center)
        ctx.save_for_backward(x, weight, stats)
        ctx.center, ctx.types = center, [None if t is None else t.dtype for t in (weight, bias)]
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, stats = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dw, db = norm_backward(_lies(dy), x, weight, stats, center=ctx.center, bias=need[3], want_dx=need[1], want_dweight=need[2])
        wt, bt = ctx.types
        return None, dx, None if dw is None else dw.to(wt), None if db is None else db.to(bt), None, None


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, graph, x, weight, bias, residual, activation, drop, weight_grad, accumulate):
        _guard_capture(ctx, graph, x, weight, bias, residual)
        x, weight = _lies(x), _lies(weight)
        act = _activation(activation)
        keep = act != TSR_ACT_NONE and graph and any(ctx.needs_input_grad[1:4])
        y, pre = linear_forward(x, weight, None if bias is None else bias.contiguous(), act, drop, None if residual is None else _lies(residual), keep_pre=keep)
        ctx.save_for_backward(x, weight, pre)
        ctx.act, ctx.drop, ctx.weight_grad, ctx.accumulate = act, drop, weight_grad, accumulate
        ctx.bias_type = None if bias is None else bias.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, pre = ctx.saved_tensors
        need = ctx.needs_input_grad[1:]
        dres = dy if need[3] else None
        if not any(need[:3]):
            return None, None, None, None, dres, None, None, None, None
        g = _lies(dy)
        kept = ctx.weight_grad if need[1] else None
        db = torch.empty(weight.shape[0], dtype=torch.float32, device=dy.device) if need[2] else None
        if kept is not None and ctx.accumulate and db is not None:     # the kept gradient is added to, the bias's is new
            db.zero_()
        dx, dw, db = linear_backward(g, x, weight, pre, ctx.act, ctx.drop, dweight=kept, dbias=db, accumulate=kept is not None and ctx.accumulate,
                                     want_dx=need[0], want_dweight=need[1])
        return None, dx, None if kept is not None else dw, None if db is None else db.to(ctx.bias_type), dres, None, None, None, None


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, graph, x, drop, residual):
        _guard_capture(ctx, graph, x, residual)
        ctx.drop = drop
        return dropout_forward(_lies(x), drop, None if residual is None else _lies(residual))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        dx = dropout_backward(_lies(dy), ctx.drop) if ctx.needs_input_grad[1] else None
        return None, dx, None, dy if ctx.needs_input_grad[3] else None


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5) -> torch.Tensor:
    """Differentiable norm_forward."""
    return _Norm.apply(torch.is_grad_enabled(), x, weight, bias, eps, True)


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6) -> torch.Tensor:
    """Differentiable norm_forward without the mean."""
    return _Norm.apply(torch.is_grad_enabled(), x, weight, None, eps, False)


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, activation=None, dropout: Optional[Dropout] = None,
           residual: Optional[torch.Tensor] = None, weight_grad: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
    """Differentiable linear_forward.  weight_grad: a matrix (the G of a TSR block, the gradient of a dense plan) that the backward pass writes the weight's
    gradient to, or adds it to (accumulate), instead of handing it to torch; weight still has to require a gradient.  A weight that a graph uses
    more than once needs accumulate, over a matrix that was set to zero."""
    if weight_grad is not None and torch.is_grad_enabled() and not weight.requires_grad:
        raise ValueError("weight_grad needs a weight that requires a gradient")
    return _Linear.apply(torch.is_grad_enabled(), x, weight, bias, residual, activation, dropout, weight_grad, accumulate)


def dropout(x: torch.Tensor, dropout: Dropout, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Differentiable dropout_forward."""
    return _Dropout.apply(torch.is_grad_enabled(), x, dropout, residual)
