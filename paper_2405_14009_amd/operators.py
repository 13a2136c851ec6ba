"""Operators on the caller's tensors (see include/recycle_stage.h): attention
with a sliding window, sinks and a relative position bias, and an AdamW step
over many tensors.

Argument marshalling only: every step runs in the HIP library.  The calls
enqueue on PyTorch's current stream of the tensors' device and take their
outputs and scratch memory from PyTorch, so they may be captured into a graph.
Autograd does not record them: a backward pass is a call of its own, as it is
for a stage.  A forward pass that autograd would have to record is refused, and so
are tangents of forward-mode differentiation and the backward calls of a backward
pass that is itself recorded (create_graph).
"""
from __future__ import annotations

import ctypes
import functools
import math
import operator
from typing import Optional, Sequence

from . import _lib as L


torch = None   # imported with the first call
_dual = None   # torch.autograd.forward_ad
_task = None   # the number of the backward pass that runs, or -1
_kinds = {}    # the library's dtype by PyTorch's


def _import():
    global torch, _dual, _task
    if torch is None:
        import torch as module
        import torch.autograd.forward_ad as _dual
        _task = module._C._current_graph_task_id
        _kinds.update({module.bfloat16: L.RC_BF16, module.float32: L.RC_FP32})
        torch = module


def _kind(t, name):
    """The library's dtype of a tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    kind = _kinds.get(t.dtype)
    if kind is None:
        raise ValueError(f"{name} must be bfloat16 or float32, not {t.dtype}")
    return kind


def _no_graph(*tensors):
    """Refuses (tensor, name, ...) of a forward call that autograd would have to record."""
    if torch.is_grad_enabled():
        for t, name in zip(tensors[::2], tensors[1::2]):
            if t is not None and getattr(t, "requires_grad", False):
                raise RuntimeError(f"{name} requires gradients, which autograd does not pass through this call; "
                                   "call it under torch.no_grad(), and the operator's backward calls for them")
    if _dual._current_level >= 0:
        _no_tangent(tensors)


def _no_second_graph(*tensors):
    """Refuses (tensor, name, ...) of a backward call within a backward pass that autograd
    records (create_graph).  Elsewhere gradients are taken as results, whatever
    their inputs require (a weight's may be left to a later call).  (Callers ask for
    a pass or a tangent themselves first: 0.1 us, where this call takes 0.3.)"""
    if _task() >= 0 and torch.is_grad_enabled():
        for t, name in zip(tensors[::2], tensors[1::2]):
            if t is not None and getattr(t, "requires_grad", False):
                raise RuntimeError(f"{name} requires gradients, which a backward pass with create_graph would take "
                                   "through this call; the operators have no second derivatives")
    if _dual._current_level >= 0:
        _no_tangent(tensors)


def _no_tangent(tensors):
    for t, name in zip(tensors[::2], tensors[1::2]):
        if isinstance(t, torch.Tensor) and _dual.unpack_dual(t).tangent is not None:
            raise RuntimeError(f"{name} has a tangent, which this call would lose; it has no forward-mode derivative")


def _view(t, name, q, shape):
    """A view of a tensor that goes with q."""
    if t is not q:
        if not isinstance(t, torch.Tensor) or t.dtype is not q.dtype or t.get_device() != q.get_device():
            _kind(t, name)
            raise ValueError(f"{name} must have the type and device of q")
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    b, s, h, d = t.stride()
    if d != 1 and shape[3] > 1:
        raise ValueError(f"{name}: the elements of a head must be contiguous")
    # the stride of a dimension of one element says nothing: any will do
    return L.RcView(t.data_ptr(), b if shape[0] > 1 else 0, s if shape[1] > 1 else 0, h if shape[2] > 1 else 0)


def _new(like):
    """A contiguous tensor like another one and its view (half the time of torch.empty)."""
    t = torch.empty_like(like, memory_format=torch.contiguous_format)
    _, s, h, d = like.shape
    return t, L.RcView(t.data_ptr(), s * h * d, h * d, d)


def _on(device):
    """The device as PyTorch's current one (None: it is), and its stream's handle
    (as current_stream does, without the stream's object: 0.1 of 1.1 us)."""
    index = device.index
    current = torch.cuda.current_device()
    if index is None or index == current:
        return None, torch._C._cuda_getCurrentRawStream(current)
    return torch.cuda.device(device), torch._C._cuda_getCurrentRawStream(index)


def _call(on, function, *args):
    if on is None:
        status = function(*args)
    else:
        with on:
            status = function(*args)
    if status != L.RC_OK:
        L.check(status)


@functools.lru_cache(maxsize=256)
def _config(kind, batch, seq, heads, kv, d, causal, window, sinks, buckets, max_distance, bias_kind, scale):
    """A checked configuration, with the bytes of its saved and work memory."""
    names = ("batch", "seq_len", "heads", "kv_heads", "head_dim", "causal", "window", "sinks", "buckets", "max_distance")
    sizes = [L.whole(*x) for x in zip(names, (batch, seq, heads, kv, d, causal, window, sinks, buckets, max_distance))]
    c = L.RcAttention(kind, *sizes, bias_kind, scale)
    saved, work = ctypes.c_size_t(), ctypes.c_size_t()
    L.check(L.load().rc_attention_memory(ctypes.byref(c), ctypes.byref(saved), ctypes.byref(work)))
    return c, saved.value, work.value


class _Call:
    """What a forward and a backward call have in common."""

    __slots__ = ("shape", "kv_shape", "q", "k", "v", "bias", "lengths", "c", "saved_bytes", "work_bytes", "lib")

    def __init__(self, q, k, v, causal, window, sinks, rel_bias, max_distance, lengths, scale):
        _import()
        kind = _kind(q, "q")
        if q.dim() != 4:
            raise ValueError("q must be [batch, tokens, heads, head_dim]")
        self.shape = shape = q.shape
        batch, seq, heads, d = shape
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("k must be [batch, tokens, kv_heads, head_dim]")
        kv = k.shape[2]
        self.kv_shape = (batch, seq, kv, d)
        self.bias = self.lengths = None
        buckets, bias_kind = 0, L.RC_FP32
        if rel_bias is not None:
            bias_kind = _kind(rel_bias, "rel_bias")
            if rel_bias.dim() != 2 or rel_bias.shape[0] != heads or rel_bias.shape[1] < 1:
                raise ValueError(f"rel_bias must be [{heads}, buckets]")
            if not rel_bias.is_contiguous() or rel_bias.device != q.device:
                raise ValueError("rel_bias must be contiguous and on the device of q")
            buckets = rel_bias.shape[1]
            self.bias = rel_bias.data_ptr()
        if lengths is not None:
            if not isinstance(lengths, torch.Tensor) or lengths.device != q.device:
                raise TypeError("lengths must be a tensor on the device of q")
            if lengths.dtype != torch.int32 or lengths.shape != (batch,) or not lengths.is_contiguous():
                raise ValueError(f"lengths must be a contiguous int32 tensor of {batch}")
            self.lengths = lengths.data_ptr()
        if scale is None:
            scale = 1.0 / math.sqrt(d) if d else 0.0
        far = max_distance if buckets else 0
        masks = int(window), int(sinks), int(far)
        if masks != (window, sinks, far):
            raise ValueError("window, sinks and max_distance must be whole numbers")
        self.c, self.saved_bytes, self.work_bytes = _config(
            kind, batch, seq, heads, kv, d, 1 if causal else 0, masks[0], masks[1], buckets, masks[2], bias_kind,
            float(scale))
        self.q = _view(q, "q", q, shape)
        self.k, self.v = _view(k, "k", q, self.kv_shape), _view(v, "v", q, self.kv_shape)
        self.lib = L.load()


def attention_forward(q, k, v, *, causal: bool = True, window: int = 0, sinks: int = 0, rel_bias=None,
                      max_distance: int = 128, lengths=None, scale: Optional[float] = None, save: bool = True,
                      out=None):
    """Attention of sequences over themselves: (o, saved).

    q: [batch, tokens, heads, d], k and v: [batch, tokens, kv_heads, d], bf16 or
    fp32, any strides of 16-byte multiples.  Token j is visible to token i when
    it lies within the sequence's length (lengths: int32 [batch]), does not
    follow i (causal), and is one of the first `sinks` tokens or less than
    `window` away (0: no window).  rel_bias: [heads, buckets], added to the
    scores by the bucket of the distance (the last one from about max_distance
    on).  scale: 1 / sqrt(d) unless given.  saved: what attention_backward needs,
    None with save=False.  out: a tensor for o.

    Tensors that require gradients are taken where autograd is off (no_grad, or
    the forward of an autograd function): o has no graph."""
    _import()
    _no_graph(q, "q", k, "k", v, "v", rel_bias, "rel_bias", out, "out")
    c = _Call(q, k, v, causal, window, sinks, rel_bias, max_distance, lengths, scale)
    on, stream = _on(q.device)
    o, ov = _new(q) if out is None else (out, _view(out, "out", q, c.shape))
    saved = torch.empty(c.saved_bytes, dtype=torch.uint8, device=q.device) if save else None
    ref = ctypes.byref
    _call(on, c.lib.rc_attention_forward, ref(c.c), ref(c.q), ref(c.k), ref(c.v), c.bias, c.lengths, ref(ov),
          saved.data_ptr() if save else None, stream)
    return o, saved


def attention_backward(dout, q, k, v, o, saved, *, causal: bool = True, window: int = 0, sinks: int = 0,
                       rel_bias=None, max_distance: int = 128, lengths=None, scale: Optional[float] = None,
                       dq=None, dk=None, dv=None):
    """Gradients of sum(dout * o): (dq, dk, dv, drel_bias), the last None without
    a bias and of its type otherwise.  o and saved are attention_forward's for the
    same arguments; dq, dk, dv: tensors for the gradients (all of their elements
    are written)."""
    _import()
    if _task() >= 0 or _dual._current_level >= 0:
        _no_second_graph(dout, "dout", q, "q", k, "k", v, "v", rel_bias, "rel_bias", o, "o")
    c = _Call(q, k, v, causal, window, sinks, rel_bias, max_distance, lengths, scale)
    if (not isinstance(saved, torch.Tensor) or saved.numel() != c.saved_bytes or saved.device != q.device
            or saved.dtype is not torch.uint8 or not saved.is_contiguous()):
        raise ValueError("saved must be what attention_forward returned for these arguments")
    ov, dov = _view(o, "o", q, c.shape), _view(dout, "dout", q, c.shape)
    on, stream = _on(q.device)
    dq, dqv = _new(q) if dq is None else (dq, _view(dq, "dq", q, c.shape))
    dk, dkv = _new(k) if dk is None else (dk, _view(dk, "dk", q, c.kv_shape))
    dv, dvv = _new(v) if dv is None else (dv, _view(dv, "dv", q, c.kv_shape))
    dbias = None if rel_bias is None else torch.empty_like(rel_bias)
    work = torch.empty(c.work_bytes, dtype=torch.uint8, device=q.device)
    ref = ctypes.byref
    _call(on, c.lib.rc_attention_backward, ref(c.c), ref(c.q), ref(c.k), ref(c.v), c.bias, c.lengths, ref(ov),
          saved.data_ptr(), ref(dov), ref(dqv), ref(dkv), ref(dvv), None if dbias is None else dbias.data_ptr(),
          work.data_ptr(), stream)
    return dq, dk, dv, dbias


def _blocks(count):
    return -(-count // 128)


class AdamW:
    """AdamW over a fixed set of tensors, all of them in one call.

    params: fp32 tensors; grads: fp32 or bf16 tensors of their sizes, read at each
    step.  decay: whether weight decay applies, by tensor (default: all).
    copies: bf16 tensors that receive the updated parameters, or None, by tensor.
    The moments are exp_avg and exp_avg_sq, by tensor: fp32, or with
    state_bits=8 bytes of codes, with exp_avg_scale and exp_avg_sq_scale a byte
    per 128 elements.  Moments that are not given start at zero (state_bits
    then says which form they have).  Every tensor is contiguous; all are kept
    and updated in place.

    params, grads, copies, decay and the moments are lists whose entries may be
    replaced between steps, and a parameter, gradient or copy may get other memory
    (its `data`): a step that meets another tensor or address than the last one
    checks them all again.  A moment's memory is replaced with its entry only.
    (A graph keeps the addresses that it was captured with.)"""

    def __init__(self, params: Sequence, grads: Sequence, *, decay: Optional[Sequence[bool]] = None,
                 copies: Optional[Sequence] = None, state_bits: Optional[int] = None, exp_avg=None,
                 exp_avg_sq=None, exp_avg_scale=None, exp_avg_sq_scale=None, lr: float = 1e-4,
                 beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, weight_decay: float = 0.1):
        _import()
        self._lib = L.load()
        self.params, self.grads = list(params), list(grads)
        n = len(self.params)
        if state_bits is None:
            state_bits = 32 if exp_avg_scale is None else 8
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.state_bits, self.steps = state_bits, 0
        given = [x is not None for x in (exp_avg, exp_avg_sq)]
        scales = [x is not None for x in (exp_avg_scale, exp_avg_sq_scale)]
        if given[0] != given[1] or scales[0] != scales[1] or scales[0] != (given[0] and state_bits == 8):
            raise ValueError("moments are given with their scales (8 bits) or without (32), or not at all")
        self._check_params()

        def zeros(size):
            kind = torch.uint8 if state_bits == 8 else torch.float32
            return [torch.zeros(size(p.numel()), dtype=kind, device=p.device) for p in self.params]

        self.exp_avg = list(exp_avg) if given[0] else zeros(lambda c: c)
        self.exp_avg_sq = list(exp_avg_sq) if given[0] else zeros(lambda c: c)
        self.exp_avg_scale = self.exp_avg_sq_scale = None
        if state_bits == 8:
            self.exp_avg_scale = list(exp_avg_scale) if given[0] else zeros(_blocks)
            self.exp_avg_sq_scale = list(exp_avg_sq_scale) if given[0] else zeros(_blocks)
        self.copies = [None] * n if copies is None else list(copies)
        self.decay = [True] * n if decay is None else [bool(x) for x in decay]
        self.adam = L.RcAdamConfig(lr, beta1, beta2, eps, weight_decay)
        self._look()

    def _check_params(self) -> None:
        for i, p in enumerate(self.params):
            if not isinstance(p, torch.Tensor) or p.device.type != "cuda":
                raise TypeError(f"params[{i}] must be a device tensor")

    def _moments(self):
        return [*self.exp_avg, *self.exp_avg_sq, *(self.exp_avg_scale or ()), *(self.exp_avg_sq_scale or ())]

    def _others(self):
        return [*self.params, *self.grads, *[c for c in self.copies if c is not None]]

    def _same_moments(self) -> bool:
        """Whether the moments are those of the last look and their storages where they were."""
        moments = self._moments()
        return (self._seen_moments is not None and len(moments) == len(self._seen_moments)
                and all(map(operator.is_, moments, self._seen_moments))
                and list(map(torch.Tensor.data_ptr, self._kept)) == self._kept_at)

    def _refresh(self) -> None:
        """Checks the tensors again if one of them, or its memory, is another one than at the last
        look (15 us of host time for 60 tensors with 8-bit moments)."""
        others, Tensor = self._others(), torch.Tensor
        if not (self._same_moments() and len(others) == len(self._seen) and all(map(operator.is_, others, self._seen))
                and list(map(Tensor.data_ptr, others)) == self._addresses and self.decay == self._decay
                and [c is None for c in self.copies] == self._no_copy
                and list(map(Tensor.numel, self.params)) == self._counts
                and all(map(Tensor.is_contiguous, self.params))):
            self._look()

    def _check_list(self, name, tensors, types, counts, places=None) -> None:
        """Refuses a list that is not one of contiguous tensors of these types and sizes (all of
        them at once, which takes a third of the time of one by one).  places: their numbers."""
        Tensor = torch.Tensor
        if len(tensors) != len(counts):
            raise ValueError(f"{name} must have {len(counts)} entries")
        if (all(issubclass(x, Tensor) for x in set(map(type, tensors)))
                and set(map(Tensor.get_device, tensors)) <= {self._index}
                and {t.dtype for t in tensors} <= set(types) and list(map(Tensor.numel, tensors)) == counts
                and all(map(Tensor.is_contiguous, tensors))):
            return
        for i, t, count in zip(places or range(len(counts)), tensors, counts):
            if not isinstance(t, Tensor) or t.device != self.device:
                raise TypeError(f"{name}[{i}] must be a tensor on {self.device}")
            if t.dtype not in types or t.numel() != count or not t.is_contiguous():
                raise ValueError(f"{name}[{i}] must be a contiguous tensor of {count} elements of "
                                 f"{' or '.join(str(x) for x in types)}")

    def _look(self) -> None:
        """Checks the tensors and writes their addresses down."""
        n, state_bits = len(self.params), self.state_bits
        kind = torch.uint8 if state_bits == 8 else torch.float32
        self._seen_moments = None    # until all of it holds
        self._check_params()
        self.device = self.params[0].device if n else None
        self._index = self.device.index if n else None
        self._counts = [p.numel() for p in self.params]
        if len(self.decay) != n or len(self.copies) != n or len(self.grads) != n:
            raise ValueError(f"grads, decay and copies must have {n} entries")
        f32, bf16 = torch.float32, torch.bfloat16
        each, at = self._counts, [i for i in range(n) if self.copies[i] is not None]
        blocks = [_blocks(count) for count in each] if state_bits == 8 else []
        # per list: tensors, their types and sizes, whether a step writes them
        lists = {"params": (self.params, (f32,), each, True), "grads": (self.grads, (f32, bf16), each, False),
                 "exp_avg": (self.exp_avg, (kind,), each, True), "exp_avg_sq": (self.exp_avg_sq, (kind,), each, True),
                 "copies": ([self.copies[i] for i in at], (bf16,), [each[i] for i in at], True)}
        if state_bits == 8:
            lists["exp_avg_scale"] = (self.exp_avg_scale, (kind,), blocks, True)
            lists["exp_avg_sq_scale"] = (self.exp_avg_sq_scale, (kind,), blocks, True)
        addresses, spans = {}, []
        for name, (tensors, types, counts, w) in lists.items():
            self._check_list(name, tensors, types, counts, at if name == "copies" else None)
            addresses[name] = first = list(map(torch.Tensor.data_ptr, tensors))
            sizes = map(torch.Tensor.element_size, tensors)
            # (first byte, byte behind the last one, whether a step writes them)
            spans += [(x, x + c * e, w) for x, c, e in zip(first, counts, sizes) if c]
        spans.sort()
        end, write_end = 0, 0
        for first, last, w in spans:
            if first < (end if w else write_end):
                raise ValueError("a tensor that a step writes is listed twice or overlaps another one")
            if last > end:
                end = last
            if w and last > write_end:
                write_end = last
        scales = zip(addresses["exp_avg_scale"], addresses["exp_avg_sq_scale"]) if state_bits == 8 else ((None, None),) * n
        copies = dict(zip(at, addresses["copies"]))
        self._tensors = (L.RcAdamwTensor * max(1, n))(*[
            (p, g, m, v, ms, vs, copies.get(i), count, L.RC_BF16 if grad.dtype is bf16 else L.RC_FP32, bool(decay))
            for i, (p, g, m, v, (ms, vs), count, grad, decay) in enumerate(zip(
                addresses["params"], addresses["grads"], addresses["exp_avg"], addresses["exp_avg_sq"], scales, each,
                self.grads, self.decay))])
        self._decay, self._no_copy = list(self.decay), [c is None for c in self.copies]
        self._seen = self._others()
        self._addresses = list(map(torch.Tensor.data_ptr, self._seen))
        # a tensor of our own for each storage that holds moments: it stays while we write to it
        moments = self._moments()
        self._kept = list({t.untyped_storage().data_ptr(): t.detach() for t in moments if t.numel()}.values())
        self._kept_at = list(map(torch.Tensor.data_ptr, self._kept))
        self._seen_moments = moments

    def step(self, grad_scale: float = 1.0, *, step: Optional[int] = None) -> None:
        """One step with grad_scale * grads, as step number `step` (by default one
        more than the last).  A captured step replays its own number."""
        number = self.steps + 1 if step is None else L.whole("step", step, 64)
        self._refresh()
        if not self.params:
            self.steps = number
            return
        on, stream = _on(self.device)
        _call(on, self._lib.rc_adamw_step, self._tensors, len(self.params), ctypes.byref(self.adam),
              self.state_bits, number, float(grad_scale), stream)
        self.steps = number

    def moments(self, out=None):
        """The moments as fp32 values: (exp_avg, exp_avg_sq), lists of tensors, by
        tensor.  out: two such lists to fill (contiguous fp32 tensors of the sizes)."""
        if not self._same_moments():
            self._look()
        if out is None:
            out = [[torch.empty(count, dtype=torch.float32, device=self.device) for count in self._counts]
                   for _ in range(2)]
        n = len(self._counts)
        arrays = []
        for name, tensors in zip(("exp_avg", "exp_avg_sq"), out):
            self._check_list(name, tensors, (torch.float32,), self._counts)
            arrays.append((ctypes.c_void_p * max(1, n))(*map(torch.Tensor.data_ptr, tensors)))
        if n:
            on, stream = _on(self.device)
            _call(on, self._lib.rc_adamw_read, self._tensors, n, self.state_bits, *arrays, stream)
        return out[0], out[1]
