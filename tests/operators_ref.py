"""Plain 64-bit forms of the operators on the caller's tensors (test
infrastructure): attention with a window, sinks and a relative position bias,
with the error that each of its outputs may have, and AdamW with 8-bit moments."""
from __future__ import annotations

import math

import numpy as np
import torch

F64 = torch.float64


# -- attention ----------------------------------------------------------------


def bucket(distance, buckets, max_distance, causal):
    """Bucket of j - i, by its definition in whole numbers."""
    side = buckets if causal else buckets // 2
    n = max(-distance, 0) if causal else abs(distance)
    exact = side // 2
    k = side - exact
    c = n
    if n >= exact:
        c = exact
        while c + 1 < side and n ** k >= exact ** (k - (c + 1 - exact)) * max_distance ** (c + 1 - exact):
            c += 1
    return c + side if not causal and distance > 0 else c


def attention(q, k, v, do=None, *, causal=True, window=0, sinks=0, bias=None, max_distance=128, lengths=None,
              scale=None):
    """Outputs of the operator in 64 bits from tensors of any type, and for each
    the sums of absolute values that bound its error (see bounds)."""
    b, s, h, d = q.shape
    kv = k.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    q, k, v = (t.cpu().to(F64).transpose(1, 2) for t in (q, k, v))
    k, v = (t.repeat_interleave(h // kv, 1) for t in (k, v))
    i, j = torch.arange(s)[:, None], torch.arange(s)[None, :]
    see = torch.ones(s, s, dtype=torch.bool)
    if causal:
        see &= j <= i
    if window:
        see &= ((i - j).abs() < window) | (j < sinks)
    see = see.expand(b, 1, s, s)
    if lengths is not None:
        n = torch.as_tensor(lengths).cpu().clamp(0, s)[:, None, None, None]
        see = see & (j < n) & (i < n)
        dead = (torch.arange(s) >= n[:, :, 0])[..., None]  # rows that are not read
        q, k, v = (t.masked_fill(dead, 0.0) for t in (q, k, v))
    x = scale * (q @ k.transpose(2, 3))
    if bias is not None:
        nb = bias.shape[1]
        of = torch.tensor([bucket(e, nb, max_distance, causal) for e in range(-(s - 1), s)])[j - i + s - 1]
        x = x + bias.cpu().to(F64)[:, of]
    x = torch.where(see, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    back = lambda t: t.transpose(1, 2)                                      # noqa: E731
    shared = lambda t: back(t.reshape(b, kv, h // kv, s, d).sum(2))         # noqa: E731
    out = {"o": back(p @ v)}
    # the sum of absolute values that a score is made of
    size = scale * (q.abs() @ k.abs().transpose(2, 3))
    if bias is not None:
        size = size + x.abs()
    # (what is hidden, or has a bias of -inf, is no part of any sum)
    size = float(torch.where(x > -math.inf, size, 0.0).detach().max())
    mag = {"score": size, "d": d, "o": (back(p @ v.abs()),)}
    if do is None:
        return out, mag
    do = do.cpu().to(F64).transpose(1, 2)
    if lengths is not None:
        do = do.masked_fill(dead, 0.0)
    dp = do @ v.transpose(2, 3)
    D = (p * dp).sum(-1, keepdim=True)
    ds = p * (dp - D)
    out["dq"], out["dk"], out["dv"] = back(scale * (ds @ k)), shared(scale * (ds.transpose(2, 3) @ q)), shared(
        p.transpose(2, 3) @ do)
    # |dS| by its own rounding; P times what D and do.v may be off, per unit of a relative error of P
    off = p * (do.abs() * (p @ v.abs())).sum(-1, keepdim=True)
    ads = ds.abs()
    part = p * (do.abs() @ v.abs().transpose(2, 3) + (do.abs() * (p @ v.abs())).sum(-1, keepdim=True))
    ka, qa = k.abs(), q.abs()
    mag["dq"] = tuple(back(scale * (m @ ka)) for m in (ads, off, part))
    mag["dk"] = tuple(shared(scale * (m.transpose(2, 3) @ qa)) for m in (ads, off, part))
    mag["dv"] = (shared(p.transpose(2, 3) @ do.abs()),)
    if bias is not None:
        def table(m):
            t = torch.zeros(h, nb, dtype=F64)
            return t.index_add_(1, of.reshape(-1), m.sum(0).reshape(h, -1))

        out["dbias"] = table(ds)
        mag["dbias"] = tuple(table(m) for m in (ads, off, part))
    return out, mag


def bounds(out, mag, kind, bias_kind=None, fine=False):
    """How far each element of an output may be from its 64-bit value.

    half: half a step of a type, relative (bf16 2^-8, fp32 2^-24).
    A probability is off by eP, relative: its score, a sum of d products and a
    few more operations in 32 bits, (d + 8) half-steps of the absolute values
    that the score is made of, in the score itself and in the row's reference
    and sum; the exponential and logarithm, 16 half-steps; and, bf16, its
    rounding before the product with v or do.
      o, dv:  eP of the sums of P |v| and P |do|, and the rounding of the result.
      dS = P (do.v - D): eP of itself; D is off by eP of |do| (P |v|) (o's
    probabilities); do.v and D are sums in 32 bits of absolute value
    |do| |v|; and, bf16, dS is rounded before its products.  The sums over
    tokens add 32-bit roundings: under 2^-16 of the absolute values for the up
    to 2^8 in a row of one accumulator here.
    fine: calls whose o takes the probabilities and o itself as two bf16 numbers each
    where D is formed, so that D is off by 2 * 2^-16 in place of eP."""
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
    r = half[kind] if kind == torch.bfloat16 else 0.0
    exact = 2.0 ** -24
    ex = 2 * (mag["d"] + 8) * exact * mag["score"] + 16 * exact
    ep = r + ex
    sums = (mag["d"] + 256) * exact
    got = {}
    for name, ref in out.items():
        last = half[bias_kind or kind] if name == "dbias" else half[kind]
        m = mag[name]
        if name in ("o", "dv"):
            e = (ep + sums) * m[0]
        else:
            e = ((r if name != "dbias" else 0.0) + ex + sums) * m[0] + (2.0 ** -15 + ex if fine else ep) * m[1] + sums * m[2]
        got[name] = (e + last * (ref.abs() + e)) * 1.01 + 1e-30
    return got


def check_attention(got, out, mag, kind, bias_kind=None, fine=False):
    """Every element within its bound; returns the worst share of a bound."""
    worst = {}
    for name, bound in bounds(out, mag, kind, bias_kind, fine).items():
        x = got[name].cpu().to(F64)
        assert x.shape == out[name].shape, name
        assert bool(torch.isfinite(x).all()), f"{name}: not finite"
        share = ((x - out[name]).abs() / bound).max() if x.numel() else torch.tensor(0.0)
        worst[name] = float(share)
    bad = {k: v for k, v in worst.items() if not v <= 1.0}
    assert not bad, f"beyond the bound: {bad} (all: {worst})"
    return worst


# -- AdamW ----------------------------------------------------------------------

M_TABLE = np.array([(c & 7) / 512 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])
V_TABLE = np.array([float(c) if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 1) for c in range(255)])


def _encode(x, table, bias):
    """Codes and block bytes of one tensor's moment (negative codes not offset)."""
    n = x.size
    codes, scales = np.zeros(n, np.int64), np.zeros(-(-n // 128), np.int64)
    for b in range(scales.size):
        a = np.abs(x[128 * b:128 * b + 128])
        fits = a <= np.finfo(np.float32).max
        top = a[fits].max(initial=0.0)
        e = -bias
        if top > 0:
            e = math.frexp(top / table[-1])[1]
            while e > -bias and top <= math.ldexp(table[-1], e - 1):
                e -= 1
            while top > math.ldexp(table[-1], e):
                e += 1
        e = max(e, -bias)
        scales[b] = e + bias
        y = np.ldexp(np.where(fits, a, 0.0), -e)
        hi = np.clip(np.searchsorted(table, y), 1, table.size - 1)
        lo = hi - 1
        down, up = y - table[lo], table[hi] - y
        codes[128 * b:128 * b + 128] = np.where(
            ~fits, -1, np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi))
    return codes, scales


def encode_m(x):
    c, s = _encode(x, M_TABLE, 127)
    return np.where(c < 0, 0x7f, c + np.where(np.signbit(x), 128, 0)).astype(np.uint8), s.astype(np.uint8)


def encode_v(x):
    c, s = _encode(x, V_TABLE, 160)
    c = np.where((c == 0) & (x > 0), 1, c)
    return np.where(c < 0, 255, c).astype(np.uint8), s.astype(np.uint8)


def decode_m(codes, scales):
    t = np.append(M_TABLE, np.nan)
    unit = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 128)[:codes.size]
    return np.where(codes >= 128, -1.0, 1.0) * t[codes & 127] * unit


def decode_v(codes, scales):
    t = np.append(V_TABLE, np.nan)
    return t[codes] * np.repeat(2.0 ** (scales.astype(np.float64) - 160), 128)[:codes.size]


def adamw(p, g, m, v, *, step, decay, grad_scale=1.0, lr=1e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1):
    """(p, m, v) after a step, in 64 bits, with the 32-bit hyperparameters of the call."""
    lr, beta1, beta2, eps, weight_decay, grad_scale = (
        float(np.float32(x)) for x in (lr, beta1, beta2, eps, weight_decay, grad_scale))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    if decay:
        p = p * (1 - lr * weight_decay)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        p = p - lr / (1 - beta1 ** step) * m / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p, m, v
