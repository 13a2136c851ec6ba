"""Operators of a layer on the caller's tensors (see include/recycle_stage.h):
dropout, layer norm of a residual sum, and linear layers, each with its
backward pass.

Argument marshalling only, as for the attention operator: every step runs in the
HIP library, on PyTorch's current stream of the tensors' device, with outputs
and work memory from PyTorch, so the calls may be captured into a graph.
Autograd does not record them: a forward pass that it would have to record is
refused, and a backward pass is a call of its own.

Matrices are tensors [..., columns] in bf16 or fp32, whose leading dimensions
have one stride between them; columns are contiguous.  Vectors of parameters are
bf16 or fp32 (one type in a call); gradients of parameters are fp32.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

from . import _lib as L
from . import operators as _ops
from .operators import _call, _import, _kind, _on

_ACTIVATIONS = {None: L.RC_ACT_NONE, "gelu": L.RC_ACT_GELU, "relu": L.RC_ACT_RELU, "silu": L.RC_ACT_SILU}
_ref = ctypes.byref


class Dropout:
    """What a dropout call draws: each element is kept with probability 1 - p (p in
    steps of 2^-16) and then divided by it.  The mask is a function of seed, offset,
    row and column alone, so the backward pass takes the same object; a program gives
    each use of its own an offset of its own.  step: an int64 device tensor of one
    number that is added to offset when the kernel runs (what a captured graph
    changes between its replays)."""

    __slots__ = ("p", "seed", "offset", "step", "_c")

    def __init__(self, p: float, seed: int, offset: int = 0, *, step=None):
        _import()
        p = float(p)
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"p must lie in 0 .. 1, not {p}")
        for name, x in (("seed", seed), ("offset", offset)):
            if int(x) != x or not 0 <= x < 1 << 64:
                raise ValueError(f"{name} must be a whole number of 64 bits, not {x}")
        if step is not None and (not isinstance(step, _ops.torch.Tensor) or not step.is_cuda
                                 or step.dtype is not _ops.torch.int64 or step.numel() != 1):
            raise TypeError("step must be an int64 device tensor of one number")
        self.p, self.seed, self.offset, self.step = p, int(seed), int(offset), step
        self._c = L.RcDropout(p, 0, self.seed, self.offset, None if step is None else step.data_ptr())


class NormGradients(NamedTuple):
    """layer_norm_backward's results; what was not asked for is None."""

    dx: object
    dtotal: object
    dweight: object
    dbias: object
    din_bias: object


def _rows(t, name):
    """Rows and row stride of a tensor [..., columns]."""
    shape, stride = t.shape, t.stride()
    if not shape:
        raise ValueError(f"{name} must have a dimension of columns")
    if shape[-1] > 1 and stride[-1] != 1:
        raise ValueError(f"{name}: the columns must be contiguous")
    rows, step = 1, None
    for n, s in zip(shape[-2::-1], stride[-2::-1]):
        if n == 1:
            continue
        if step is None:
            step = s
        elif s != step * rows and n and rows:
            raise ValueError(f"{name}: the rows must have one stride between them")
        rows *= n
    return rows, shape[-1] if step is None else step


def _matrix(t, name, like):
    """A matrix that goes with `like`."""
    if t is not like:
        if (not isinstance(t, _ops.torch.Tensor) or t.dtype is not like.dtype
                or t.get_device() != like.get_device()):
            _kind(t, name)
            raise ValueError(f"{name} must have the type and device of the others")
        if t.shape != like.shape:
            raise ValueError(f"{name} must have the shape {tuple(like.shape)}, not {tuple(t.shape)}")
    return L.RcMatrix(t.data_ptr(), _rows(t, name)[1])


def _optional(t, name, like):
    return None if t is None else _ref(_matrix(t, name, like))


def _new(like, columns=None):
    """A contiguous tensor like another one, or with another number of columns."""
    if columns is None:
        return _ops.torch.empty_like(like, memory_format=_ops.torch.contiguous_format)
    return like.new_empty((*like.shape[:-1], columns))


def _output(t, name, like):
    """An output like another tensor (the caller's, or a new one) and its matrix."""
    if t is None:
        t = _new(like)
        return t, L.RcMatrix(t.data_ptr(), t.shape[-1])
    return t, _matrix(t, name, like)


def _vectors(n, like, **vectors):
    """The type of the vectors of parameters that are given, and their addresses."""
    kind, places = None, []
    for name, t in vectors.items():
        if t is None:
            places.append(None)
            continue
        this = _kind(t, name)
        if kind is not None and this != kind:
            raise ValueError(f"{name} must have the type of the other vectors")
        kind = this
        if t.shape != (n,) or not t.is_contiguous() or t.get_device() != like.get_device():
            raise ValueError(f"{name} must be a contiguous vector of {n} on the device of the matrices")
        places.append(t.data_ptr())
    return L.RC_FP32 if kind is None else kind, places


def _gradient(want, name, shape, like):
    """An fp32 gradient of parameters: none (False), a new tensor (True) or the caller's."""
    if want is None or want is False:
        return None
    if want is True:
        return _ops.torch.empty(shape, dtype=_ops.torch.float32, device=like.device)
    if (not isinstance(want, _ops.torch.Tensor) or want.dtype is not _ops.torch.float32
            or want.get_device() != like.get_device()):
        raise TypeError(f"{name} must be True, False or an fp32 tensor on the device of the matrices")
    if want.shape != shape or not want.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of the shape {tuple(shape)}")
    return want


def _accumulates(accumulate, *wants):
    if accumulate and any(w is True for w in wants):
        raise ValueError("accumulate needs the tensors to add to")
    return 1 if accumulate else 0


def _address(t):
    return None if t is None else t.data_ptr()


def _no_graph(**tensors):
    if _ops.torch.is_grad_enabled():
        for name, t in tensors.items():
            if t is not None and getattr(t, "requires_grad", False):
                raise RuntimeError(f"{name} requires gradients, which autograd does not pass through this call; "
                                   "call it under torch.no_grad(), and the operator's backward calls for them")


def _dropout(drop, like, needed):
    if drop is None and not needed:
        return None
    if not isinstance(drop, Dropout):
        raise TypeError("drop must be a Dropout")
    if drop.step is not None and drop.step.get_device() != like.get_device():
        raise ValueError("the dropout's step must be on the device of the matrices")
    return _ref(drop._c)


def _work(size, like):
    return _ops.torch.empty(size, dtype=_ops.torch.uint8, device=like.device) if size else None


@functools.lru_cache(maxsize=256)
def _rows_config(kind, params, rows, cols, operator):
    """Checked sizes, with the bytes of the backward pass's work memory."""
    c = L.RcRows(kind, params, rows, cols)
    size = ctypes.c_size_t()
    L.check(getattr(L.load(), operator + "_memory")(_ref(c), _ref(size)))
    return c, size.value


@functools.lru_cache(maxsize=256)
def _linear_config(kind, bias_kind, rows, fan_in, fan_out, activation, by_out):
    """Checked sizes, with the bytes of the three calls' work memory."""
    c = L.RcLinear(kind, bias_kind, rows, fan_in, fan_out, activation, by_out)
    sizes = [ctypes.c_size_t() for _ in range(3)]
    L.check(L.load().rc_linear_memory(_ref(c), *map(_ref, sizes)))
    return c, *(x.value for x in sizes)


def dropout_forward(x, drop: Dropout, *, bias=None, residual=None, out=None):
    """residual + D(x + bias): D keeps and scales elements as `drop` says, or makes
    them 0.  bias: [columns], residual: like x.  out: a tensor for the result, which
    overlaps no input."""
    _import()
    kind = _kind(x, "x")
    _no_graph(x=x, bias=bias, residual=residual, out=out)
    d = _dropout(drop, x, True)
    rows, step = _rows(x, "x")
    cols = x.shape[-1]
    params, (b,) = _vectors(cols, x, bias=bias)
    c, _ = _rows_config(kind, params, rows, cols, "rc_dropout")
    y, ym = _output(out, "out", x)
    on, stream = _on(x.device)
    _call(on, L.load().rc_dropout_forward, _ref(c), d, _ref(L.RcMatrix(x.data_ptr(), step)), b,
          _optional(residual, "residual", x), _ref(ym), stream)
    return y


def dropout_backward(dy, drop: Dropout, *, derivative=None, bias_grad=False, accumulate: bool = False, out=None):
    """(dx, dbias): dx = D(dy) * derivative, with dropout_forward's `drop`, and the
    column sums of dx before its rounding (None without bias_grad).  derivative:
    what linear_forward stored of an activation that the elements went through
    before the dropout (without a dropout: Dropout(0.0, 0)).  bias_grad: True, or an
    fp32 tensor [columns], which accumulate adds to.  The gradient of the residual is dy."""
    _import()
    kind = _kind(dy, "dy")
    d = _dropout(drop, dy, True)
    rows, step = _rows(dy, "dy")
    cols = dy.shape[-1]
    c, work_bytes = _rows_config(kind, L.RC_FP32, rows, cols, "rc_dropout")
    more = _accumulates(accumulate, bias_grad)
    dbias = _gradient(bias_grad, "bias_grad", (cols,), dy)
    dx, dxm = _output(out, "out", dy)
    work = _work(work_bytes if dbias is not None else 0, dy)
    on, stream = _on(dy.device)
    _call(on, L.load().rc_dropout_backward, _ref(c), d, _ref(L.RcMatrix(dy.data_ptr(), step)),
          _optional(derivative, "derivative", dy), _ref(dxm), _address(dbias), more, _address(work), stream)
    return dx, dbias


def layer_norm_forward(x, weight=None, bias=None, *, eps: float = 1e-5, in_bias=None, drop: Optional[Dropout] = None,
                       residual=None, save: bool = True, out=None, total=None):
    """(y, total, stats): total = residual + D(x + in_bias) in its type (x itself
    where none of the three is given), y = its norm over each row, times weight, plus
    bias (None: 1, 0).  stats: what layer_norm_backward needs, None with save=False.
    out, total: tensors for the results."""
    _import()
    kind = _kind(x, "x")
    _no_graph(x=x, weight=weight, bias=bias, in_bias=in_bias, residual=residual, out=out, total=total)
    d = _dropout(drop, x, False)
    rows, step = _rows(x, "x")
    cols = x.shape[-1]
    params, (w, b, ib) = _vectors(cols, x, weight=weight, bias=bias, in_bias=in_bias)
    c, _ = _rows_config(kind, params, rows, cols, "rc_layer_norm")
    rm = _optional(residual, "residual", x)
    tm = None
    if d is not None or ib is not None or rm is not None:
        total, tm = _output(total, "total", x)
        tm = _ref(tm)
    elif total is not None:
        raise ValueError("total without a residual, a dropout or an in_bias is x")
    else:
        total = x
    y, ym = _output(out, "out", x)
    stats = _ops.torch.empty((2, rows), dtype=_ops.torch.float32, device=x.device) if save else None
    on, stream = _on(x.device)
    _call(on, L.load().rc_layer_norm_forward, _ref(c), float(eps), d, _ref(L.RcMatrix(x.data_ptr(), step)), ib, rm, w,
          b, tm, _ref(ym), _address(stats), stream)
    return y, total, stats


def layer_norm_backward(dy, total, stats, weight=None, *, dtotal=None, drop: Optional[Dropout] = None,
                        input_grad: bool = True, weight_grad=True, bias_grad=True, in_bias_grad=False,
                        accumulate: bool = False):
    """NormGradients from dy and, where total goes on as the next residual, dtotal:
    dtotal, the gradient of total and of residual; dx, that of x (dtotal itself
    without a dropout); dweight, dbias and din_bias.  total and stats are
    layer_norm_forward's, drop the same.  input_grad: whether dx and dtotal are
    formed; weight_grad, bias_grad, in_bias_grad: True, False or fp32 tensors
    [columns], which accumulate adds to.  The parameters' gradients may so be left to
    a later call."""
    _import()
    kind = _kind(dy, "dy")
    d = _dropout(drop, dy, False)
    rows, step = _rows(dy, "dy")
    cols = dy.shape[-1]
    params, (w,) = _vectors(cols, dy, weight=weight)
    c, work_bytes = _rows_config(kind, params, rows, cols, "rc_layer_norm")
    if (not isinstance(stats, _ops.torch.Tensor) or stats.dtype is not _ops.torch.float32 or stats.shape != (2, rows)
            or not stats.is_contiguous() or stats.get_device() != dy.get_device()):
        raise ValueError("stats must be what layer_norm_forward returned for these rows")
    more = _accumulates(accumulate, weight_grad, bias_grad, in_bias_grad)
    sums = [_gradient(want, name, (cols,), dy) for name, want in
            (("weight_grad", weight_grad), ("bias_grad", bias_grad), ("in_bias_grad", in_bias_grad))]
    dt = dx = dtm = dxm = None
    if input_grad:
        dt = _new(dy)
        dtm = _ref(L.RcMatrix(dt.data_ptr(), cols))
        dx = dt
        if d is not None:
            dx = _new(dy)
            dxm = _ref(L.RcMatrix(dx.data_ptr(), cols))
    elif not any(s is not None for s in sums):
        raise ValueError("no gradient is asked for")
    work = _work(work_bytes if any(s is not None for s in sums) else 0, dy)
    on, stream = _on(dy.device)
    _call(on, L.load().rc_layer_norm_backward, _ref(c), d, _ref(L.RcMatrix(dy.data_ptr(), step)),
          _optional(dtotal, "dtotal", dy), _ref(_matrix(total, "total", dy)), stats.data_ptr(), w, dtm, dxm,
          *map(_address, sums), more, _address(work), stream)
    return NormGradients(dx, dt, *sums)


def _weight(weight, like):
    """A weight [in, out], either dimension contiguous: its matrix, and whether it is stored [out, in]."""
    if (not isinstance(weight, _ops.torch.Tensor) or weight.dtype is not like.dtype
            or weight.get_device() != like.get_device()):
        _kind(weight, "weight")
        raise ValueError("weight must have the type and device of the matrices")
    if weight.dim() != 2:
        raise ValueError("weight must be [in, out]")
    s0, s1 = weight.stride()
    if s1 == 1:
        return L.RcMatrix(weight.data_ptr(), s0), 0
    if s0 == 1:
        return L.RcMatrix(weight.data_ptr(), s1), 1
    raise ValueError("weight: one of its dimensions must be contiguous")


def _activation(activation):
    try:
        return _ACTIVATIONS[activation]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be None, 'gelu', 'relu' or 'silu', not {activation!r}") from None


def linear_forward(x, weight, bias=None, *, activation: Optional[str] = None, residual=None, save: bool = True,
                   out=None):
    """(y, derivative): y = act(x weight + bias) + residual.  weight: [in, out],
    either dimension contiguous (the transpose of a matrix stored [out, in] will do).
    activation: None, "gelu" (its tanh form), "relu" or "silu".  derivative: the
    activation's, for the backward calls (None without an activation or with
    save=False).  in and out are multiples of 8, data and row strides of 16 bytes."""
    _import()
    kind = _kind(x, "x")
    _no_graph(x=x, weight=weight, bias=bias, residual=residual, out=out)
    act = _activation(activation)
    rows, step = _rows(x, "x")
    wm, by_out = _weight(weight, x)
    fan_in, fan_out = weight.shape
    if x.shape[-1] != fan_in:
        raise ValueError(f"x must have {fan_in} columns, as weight has rows, not {x.shape[-1]}")
    bias_kind, (b,) = _vectors(fan_out, x, bias=bias)
    c, work_bytes, _, _ = _linear_config(kind, bias_kind, rows, fan_in, fan_out, act, by_out)
    if out is None:
        y = _new(x, fan_out)
        ym = L.RcMatrix(y.data_ptr(), fan_out)
    else:
        y = out
        if not isinstance(y, _ops.torch.Tensor) or y.shape != (*x.shape[:-1], fan_out):
            raise ValueError(f"out must have the shape {(*x.shape[:-1], fan_out)}")
        if y.dtype is not x.dtype or y.get_device() != x.get_device():
            raise ValueError("out must have the type and device of x")
        ym = _matrix(y, "out", y)
    slope = _new(y) if act and save else None
    work = _work(work_bytes, x)
    on, stream = _on(x.device)
    _call(on, L.load().rc_linear_forward, _ref(c), _ref(L.RcMatrix(x.data_ptr(), step)), _ref(wm), b,
          _optional(residual, "residual", y), _ref(ym),
          None if slope is None else _ref(L.RcMatrix(slope.data_ptr(), fan_out)), _address(work), stream)
    return y, slope


def linear_backward_input(dy, weight, *, derivative=None, out=None):
    """dx = (dy weight^T) * derivative.  dy: the gradient at x weight + bias.
    derivative: what linear_forward stored of the activation that made x (dx is then
    the gradient before that activation, which that layer's backward calls take)."""
    _import()
    kind = _kind(dy, "dy")
    rows, step = _rows(dy, "dy")
    wm, by_out = _weight(weight, dy)
    fan_in, fan_out = weight.shape
    if dy.shape[-1] != fan_out:
        raise ValueError(f"dy must have {fan_out} columns, as weight has, not {dy.shape[-1]}")
    c, _, work_bytes, _ = _linear_config(kind, L.RC_FP32, rows, fan_in, fan_out, L.RC_ACT_NONE, by_out)
    shape = (*dy.shape[:-1], fan_in)
    if out is None:
        dx = _new(dy, fan_in)
    elif (not isinstance(out, _ops.torch.Tensor) or out.shape != shape or out.dtype is not dy.dtype
          or out.get_device() != dy.get_device()):
        raise ValueError(f"out must have the shape {shape}, and the type and device of dy")
    else:
        dx = out
    work = _work(work_bytes, dy)
    on, stream = _on(dy.device)
    _call(on, L.load().rc_linear_backward_input, _ref(c), _ref(L.RcMatrix(dy.data_ptr(), step)), _ref(wm),
          _optional(derivative, "derivative", dx), _ref(_matrix(dx, "out", dx)), _address(work), stream)
    return dx


def linear_backward_weight(x, dy, *, by_out: bool = False, weight_grad=True, bias_grad=True, accumulate: bool = False):
    """(dweight, dbias): x^T dy, fp32 [in, out], and the column sums of dy (None
    without bias_grad).  by_out: dweight is the transpose of a contiguous matrix
    [out, in], for weights stored so.  weight_grad, bias_grad: True, or fp32 tensors,
    which accumulate adds to."""
    _import()
    kind = _kind(x, "x")
    rows, step = _rows(x, "x")
    if (not isinstance(dy, _ops.torch.Tensor) or dy.dtype is not x.dtype or dy.get_device() != x.get_device()):
        _kind(dy, "dy")
        raise ValueError("dy must have the type and device of x")
    if dy.shape[:-1] != x.shape[:-1] or not dy.dim():
        raise ValueError(f"dy must have the rows of x, {tuple(x.shape[:-1])}")
    dstep = _rows(dy, "dy")[1]
    fan_in, fan_out = x.shape[-1], dy.shape[-1]
    by_out = 1 if by_out else 0
    c, _, _, work_bytes = _linear_config(kind, L.RC_FP32, rows, fan_in, fan_out, L.RC_ACT_NONE, by_out)
    if weight_grad is None or weight_grad is False:
        raise ValueError("weight_grad must be True or an fp32 tensor")
    more = _accumulates(accumulate, weight_grad, bias_grad)
    shape = (fan_out, fan_in) if by_out else (fan_in, fan_out)
    if weight_grad is not True and by_out:
        weight_grad = weight_grad.t()
    dw = _gradient(weight_grad, "weight_grad", shape, x)
    dbias = _gradient(bias_grad, "bias_grad", (fan_out,), x)
    work = _work(work_bytes, x)
    on, stream = _on(x.device)
    _call(on, L.load().rc_linear_backward_weight, _ref(c), _ref(L.RcMatrix(x.data_ptr(), step)),
          _ref(L.RcMatrix(dy.data_ptr(), dstep)), dw.data_ptr(), _address(dbias), more, _address(work), stream)
    return (dw.t() if by_out else dw), dbias
