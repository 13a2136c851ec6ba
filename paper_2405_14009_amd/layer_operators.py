"""Operators of a layer on the caller's tensors (see include/recycle_stage.h):
dropout, layer norm of a residual sum, and linear layers, each with its
backward pass.

Argument marshalling only, as for the attention operator: every step runs in the
HIP library, on PyTorch's current stream of the tensors' device, with outputs
and work memory from PyTorch, so the calls may be captured into a graph.
Autograd does not record them: a forward pass that it would have to record is
refused, a backward pass is a call of its own, and what one of these calls would
lose of a tangent or of a second derivative is refused as well.

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
from .operators import _kind, _kinds, _no_graph, _no_second_graph

_ACTIVATIONS = {None: L.RC_ACT_NONE, "gelu": L.RC_ACT_GELU, "relu": L.RC_ACT_RELU, "silu": L.RC_ACT_SILU}
_ref, _Matrix = ctypes.byref, L.RcMatrix
torch = _dual = _task = None   # imported with the first call


def _import():
    global torch, _dual, _task
    _ops._import()
    _dual, _task, torch = _ops._dual, _ops._task, _ops.torch


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
        if step is not None and (not isinstance(step, torch.Tensor) or not step.is_cuda
                                 or step.dtype is not torch.int64 or step.numel() != 1):
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
    if len(shape) == 2:
        rows, step = shape[0], stride[0]
    else:
        if not shape:
            raise ValueError(f"{name} must have a dimension of columns")
        rows, step = 1, None
        for n, s in zip(shape[-2::-1], stride[-2::-1]):
            if n == 1:
                continue
            if step is None:
                step = s
            elif s != step * rows and n and rows:
                raise ValueError(f"{name}: the rows must have one stride between them")
            rows *= n
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the columns must be contiguous")
    return rows, shape[-1] if rows == 1 else step


def _tensor(t, name, dtype, device):
    """Refuses what is not a tensor of the type and device (its number) of the others."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != device:
        _kind(t, name)
        raise ValueError(f"{name} must have the type and device of the others")


def _matrix(t, name, shape, dtype, device):
    """A reference to a matrix of this shape."""
    _tensor(t, name, dtype, device)
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    return _ref(_Matrix(t.data_ptr(), _rows(t, name)[1]))


def _output(t, name, like, shape, dtype, device):
    """An output like another tensor (the caller's, or a new one), and a reference to its matrix."""
    if t is None:
        t = torch.empty_like(like, memory_format=torch.contiguous_format)
        return t, _ref(_Matrix(t.data_ptr(), shape[-1]))
    return t, _matrix(t, name, shape, dtype, device)


def _vector(t, name, n, device, kind):
    """The address of a vector of parameters, and its type, which is that of those before it."""
    if t is None:
        return None, kind
    this = _kinds.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if this is None or t.get_device() != device:
        this = _kind(t, name)
        raise ValueError(f"{name} must be on the device of the matrices")
    if kind is not None and this != kind:
        raise ValueError(f"{name} must have the type of the other vectors")
    if t.dim() != 1 or t.numel() != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous vector of {n}")
    return t.data_ptr(), this


def _gradient(want, name, shape, like):
    """An fp32 gradient of parameters: none (False), a new tensor (True) or the caller's."""
    if want is None or want is False:
        return None
    if want is True:
        return torch.empty(shape, dtype=torch.float32, device=like.device)
    if (not isinstance(want, torch.Tensor) or want.dtype is not torch.float32
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


def _dropout(drop, device):
    if not isinstance(drop, Dropout):
        raise TypeError("drop must be a Dropout")
    if drop.step is not None:
        if drop.step.get_device() != device:
            raise ValueError("the dropout's step must be on the device of the matrices")
        drop._c.step = drop.step.data_ptr()
    return _ref(drop._c)


def _work(size, like):
    return torch.empty(size, dtype=torch.uint8, device=like.device)


def _call(function, device, *args):
    """The call on PyTorch's current stream of the device."""
    stream = torch._C._cuda_getCurrentRawStream(device)
    if device == torch._C._cuda_getDevice():
        status = function(*args, stream)
    else:
        with torch.cuda.device(device):
            status = function(*args, stream)
    if status != L.RC_OK:
        L.check(status)


@functools.lru_cache(maxsize=256)
def _rows_config(kind, params, rows, cols, operator):
    """Checked sizes, with the bytes of the backward pass's work memory."""
    c = L.RcRows(kind, L.RC_FP32 if params is None else params, rows, cols)
    size = ctypes.c_size_t()
    L.check(getattr(L.load(), operator + "_memory")(_ref(c), _ref(size)))
    return _ref(c), size.value


@functools.lru_cache(maxsize=256)
def _linear_config(kind, bias_kind, rows, fan_in, fan_out, activation, by_out):
    """Checked sizes, with the bytes of the three calls' work memory."""
    c = L.RcLinear(kind, L.RC_FP32 if bias_kind is None else bias_kind, rows, fan_in, fan_out, activation, by_out)
    sizes = [ctypes.c_size_t() for _ in range(3)]
    L.check(L.load().rc_linear_memory(_ref(c), *map(_ref, sizes)))
    return _ref(c), *(x.value for x in sizes)


def dropout_forward(x, drop: Dropout, *, bias=None, residual=None, out=None):
    """residual + D(x + bias): D keeps and scales elements as `drop` says, or makes
    them 0.  bias: [columns], residual: like x.  out: a tensor for the result, which
    overlaps no input."""
    if torch is None:
        _import()
    kind = _kind(x, "x")
    _no_graph(x, "x", bias, "bias", residual, "residual", out, "out")
    shape, dtype, device = x.shape, x.dtype, x.get_device()
    d = _dropout(drop, device)
    rows, step = _rows(x, "x")
    cols = shape[-1]
    b, params = _vector(bias, "bias", cols, device, None)
    c, _ = _rows_config(kind, params, rows, cols, "rc_dropout")
    r = None if residual is None else _matrix(residual, "residual", shape, dtype, device)
    y, ym = _output(out, "out", x, shape, dtype, device)
    _call(L.load().rc_dropout_forward, device, c, d, _ref(_Matrix(x.data_ptr(), step)), b, r, ym)
    return y


def dropout_backward(dy, drop: Dropout, *, derivative=None, bias_grad=False, accumulate: bool = False, out=None):
    """(dx, dbias): dx = D(dy) * derivative, with dropout_forward's `drop`, and the
    column sums of dx before its rounding (None without bias_grad).  derivative:
    what linear_forward stored of an activation that the elements went through
    before the dropout (without a dropout: Dropout(0.0, 0)).  bias_grad: True, or an
    fp32 tensor [columns], which accumulate adds to.  The gradient of the residual is dy."""
    if torch is None:
        _import()
    kind = _kind(dy, "dy")
    if _task() >= 0 or _dual._current_level >= 0:
        _no_second_graph(dy, "dy", derivative, "derivative")
    shape, dtype, device = dy.shape, dy.dtype, dy.get_device()
    d = _dropout(drop, device)
    rows, step = _rows(dy, "dy")
    cols = shape[-1]
    c, work_bytes = _rows_config(kind, None, rows, cols, "rc_dropout")
    more = _accumulates(accumulate, bias_grad)
    dbias = _gradient(bias_grad, "bias_grad", (cols,), dy)
    m = None if derivative is None else _matrix(derivative, "derivative", shape, dtype, device)
    dx, dxm = _output(out, "out", dy, shape, dtype, device)
    work = _work(work_bytes, dy) if dbias is not None and work_bytes else None
    _call(L.load().rc_dropout_backward, device, c, d, _ref(_Matrix(dy.data_ptr(), step)), m, dxm, _address(dbias), more,
          _address(work))
    return dx, dbias


def layer_norm_forward(x, weight=None, bias=None, *, eps: float = 1e-5, in_bias=None, drop: Optional[Dropout] = None,
                       residual=None, save: bool = True, out=None, total=None):
    """(y, total, stats): total = residual + D(x + in_bias) in its type (x itself
    where none of the three is given), y = its norm over each row, times weight, plus
    bias (None: 1, 0).  stats: what layer_norm_backward needs, None with save=False.
    out, total: tensors for the results."""
    if torch is None:
        _import()
    kind = _kind(x, "x")
    _no_graph(x, "x", weight, "weight", bias, "bias", in_bias, "in_bias", residual, "residual", out, "out", total, "total")
    shape, dtype, device = x.shape, x.dtype, x.get_device()
    d = None if drop is None else _dropout(drop, device)
    rows, step = _rows(x, "x")
    cols = shape[-1]
    w, params = _vector(weight, "weight", cols, device, None)
    b, params = _vector(bias, "bias", cols, device, params)
    ib, params = _vector(in_bias, "in_bias", cols, device, params)
    c, _ = _rows_config(kind, params, rows, cols, "rc_layer_norm")
    r = tm = None
    if residual is not None:
        r = _matrix(residual, "residual", shape, dtype, device)
    if d is not None or ib is not None or r is not None:
        total, tm = _output(total, "total", x, shape, dtype, device)
    elif total is not None:
        raise ValueError("total without a residual, a dropout or an in_bias is x")
    else:
        total = x
    y, ym = _output(out, "out", x, shape, dtype, device)
    stats = torch.empty((2, rows), dtype=torch.float32, device=x.device) if save else None
    _call(L.load().rc_layer_norm_forward, device, c, float(eps), d, _ref(_Matrix(x.data_ptr(), step)), ib, r, w, b, tm,
          ym, _address(stats))
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
    if torch is None:
        _import()
    kind = _kind(dy, "dy")
    if _task() >= 0 or _dual._current_level >= 0:
        _no_second_graph(dy, "dy", total, "total", stats, "stats", weight, "weight", dtotal, "dtotal")
    shape, dtype, device = dy.shape, dy.dtype, dy.get_device()
    d = None if drop is None else _dropout(drop, device)
    rows, step = _rows(dy, "dy")
    cols = shape[-1]
    w, params = _vector(weight, "weight", cols, device, None)
    c, work_bytes = _rows_config(kind, params, rows, cols, "rc_layer_norm")
    if (not isinstance(stats, torch.Tensor) or stats.dtype is not torch.float32 or stats.shape != (2, rows)
            or not stats.is_contiguous() or stats.get_device() != device):
        raise ValueError("stats must be what layer_norm_forward returned for these rows")
    t = _matrix(total, "total", shape, dtype, device)
    din = None if dtotal is None else _matrix(dtotal, "dtotal", shape, dtype, device)
    more = _accumulates(accumulate, weight_grad, bias_grad, in_bias_grad)
    vector = (cols,)
    dw = _gradient(weight_grad, "weight_grad", vector, dy)
    db = _gradient(bias_grad, "bias_grad", vector, dy)
    dib = _gradient(in_bias_grad, "in_bias_grad", vector, dy)
    sums = dw is not None or db is not None or dib is not None
    dt = dx = dtm = dxm = None
    if input_grad:
        dt, dtm = _output(None, "dtotal", dy, shape, dtype, device)
        dx = dt
        if d is not None:
            dx, dxm = _output(None, "dx", dy, shape, dtype, device)
    elif not sums:
        raise ValueError("no gradient is asked for")
    work = _work(work_bytes, dy) if sums and work_bytes else None
    _call(L.load().rc_layer_norm_backward, device, c, d, _ref(_Matrix(dy.data_ptr(), step)), din, t, stats.data_ptr(), w,
          dtm, dxm, _address(dw), _address(db), _address(dib), more, _address(work))
    return NormGradients(dx, dt, dw, db, dib)


def _weight(weight, dtype, device):
    """A weight [in, out], either dimension contiguous: its matrix, and whether it is stored [out, in]."""
    _tensor(weight, "weight", dtype, device)
    if weight.dim() != 2:
        raise ValueError("weight must be [in, out]")
    s0, s1 = weight.stride()
    if s1 == 1:
        return _ref(_Matrix(weight.data_ptr(), s0)), 0
    if s0 == 1:
        return _ref(_Matrix(weight.data_ptr(), s1)), 1
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
    if torch is None:
        _import()
    kind = _kind(x, "x")
    _no_graph(x, "x", weight, "weight", bias, "bias", residual, "residual", out, "out")
    act = _activation(activation)
    dtype, device = x.dtype, x.get_device()
    rows, step = _rows(x, "x")
    wm, by_out = _weight(weight, dtype, device)
    fan_in, fan_out = weight.shape
    if x.shape[-1] != fan_in:
        raise ValueError(f"x must have {fan_in} columns, as weight has rows, not {x.shape[-1]}")
    b, bias_kind = _vector(bias, "bias", fan_out, device, None)
    c, work_bytes, _, _ = _linear_config(kind, bias_kind, rows, fan_in, fan_out, act, by_out)
    shape = (*x.shape[:-1], fan_out)
    r = sm = None
    if residual is not None:
        r = _matrix(residual, "residual", shape, dtype, device)
    if out is None:
        y = x.new_empty(shape)
        ym = _ref(_Matrix(y.data_ptr(), fan_out))
    else:
        y, ym = out, _matrix(out, "out", shape, dtype, device)
    slope = None
    if act and save:
        slope, sm = _output(None, "derivative", y, shape, dtype, device)
    work = _work(work_bytes, x) if work_bytes else None
    _call(L.load().rc_linear_forward, device, c, _ref(_Matrix(x.data_ptr(), step)), wm, b, r, ym, sm, _address(work))
    return y, slope


def linear_backward_input(dy, weight, *, derivative=None, out=None):
    """dx = (dy weight^T) * derivative.  dy: the gradient at x weight + bias.
    derivative: what linear_forward stored of the activation that made x (dx is then
    the gradient before that activation, which that layer's backward calls take)."""
    if torch is None:
        _import()
    kind = _kind(dy, "dy")
    if _task() >= 0 or _dual._current_level >= 0:
        _no_second_graph(dy, "dy", weight, "weight", derivative, "derivative")
    dtype, device = dy.dtype, dy.get_device()
    rows, step = _rows(dy, "dy")
    wm, by_out = _weight(weight, dtype, device)
    fan_in, fan_out = weight.shape
    if dy.shape[-1] != fan_out:
        raise ValueError(f"dy must have {fan_out} columns, as weight has, not {dy.shape[-1]}")
    c, _, work_bytes, _ = _linear_config(kind, None, rows, fan_in, fan_out, L.RC_ACT_NONE, by_out)
    shape = (*dy.shape[:-1], fan_in)
    s = None if derivative is None else _matrix(derivative, "derivative", shape, dtype, device)
    if out is None:
        out = dy.new_empty(shape)
        dxm = _ref(_Matrix(out.data_ptr(), fan_in))
    else:
        dxm = _matrix(out, "out", shape, dtype, device)
    work = _work(work_bytes, dy) if work_bytes else None
    _call(L.load().rc_linear_backward_input, device, c, _ref(_Matrix(dy.data_ptr(), step)), wm, s, dxm, _address(work))
    return out


def linear_backward_weight(x, dy, *, by_out: bool = False, weight_grad=True, bias_grad=True, accumulate: bool = False):
    """(dweight, dbias): x^T dy, fp32 [in, out], and the column sums of dy (None
    without bias_grad).  by_out: dweight is the transpose of a contiguous matrix
    [out, in], for weights stored so.  weight_grad, bias_grad: True, or fp32 tensors,
    which accumulate adds to."""
    if torch is None:
        _import()
    kind = _kind(x, "x")
    if _task() >= 0 or _dual._current_level >= 0:
        _no_second_graph(x, "x", dy, "dy")
    dtype, device = x.dtype, x.get_device()
    rows, step = _rows(x, "x")
    _tensor(dy, "dy", dtype, device)
    if not dy.dim() or dy.shape[:-1] != x.shape[:-1]:
        raise ValueError(f"dy must have the rows of x, {tuple(x.shape[:-1])}")
    dstep = _rows(dy, "dy")[1]
    fan_in, fan_out = x.shape[-1], dy.shape[-1]
    by_out = 1 if by_out else 0
    c, _, _, work_bytes = _linear_config(kind, None, rows, fan_in, fan_out, L.RC_ACT_NONE, by_out)
    if weight_grad is None or weight_grad is False:
        raise ValueError("weight_grad must be True or an fp32 tensor")
    more = _accumulates(accumulate, weight_grad, bias_grad)
    shape = (fan_out, fan_in) if by_out else (fan_in, fan_out)
    if by_out and isinstance(weight_grad, torch.Tensor) and weight_grad.dim() == 2:
        weight_grad = weight_grad.t()
    dw = _gradient(weight_grad, "weight_grad", shape, x)
    dbias = _gradient(bias_grad, "bias_grad", (fan_out,), x)
    work = _work(work_bytes, x) if work_bytes else None
    _call(L.load().rc_linear_backward_weight, device, c, _ref(_Matrix(x.data_ptr(), step)),
          _ref(_Matrix(dy.data_ptr(), dstep)), dw.data_ptr(), _address(dbias), more, _address(work))
    return (dw.t() if by_out else dw), dbias
