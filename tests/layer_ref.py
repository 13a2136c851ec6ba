"""Plain 64-bit forms of the operators of a layer, and how far the library's
results may be from them.

Bounds count roundings, by the standard bound of a sum in 32 bits (n terms in any
order: n 2^-24 times the sum of the magnitudes; U below), plus half a step of the
output's type."""
import math

import numpy as np

U = 2.0 ** -24
HALF = {"torch.bfloat16": 2.0 ** -8, "torch.float32": 2.0 ** -24}


def half(t):
    return HALF[str(t.dtype)]


def philox(counter, key):
    """Philox4x32-10 of counters [..., 4] under a key of two words."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [np.uint64(key[0]), np.uint64(key[1])]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ k[0], q & low, (p >> np.uint64(32)) ^ c[3] ^ k[1], p & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return np.stack(c, -1)


def threshold(p):
    """Of the float that the call takes."""
    return int(math.floor(float(np.float32(p)) * 65536 + 0.5))


def factor(rows, cols, p, seed, offset, first=0):
    """D as a factor [rows, cols], of rows first .. first + rows - 1."""
    t = threshold(p)
    if t == 0:
        return np.ones((rows, cols))
    g = -(-cols // 8)
    at = np.zeros((rows, g, 4), dtype=np.uint64)
    at[..., 0] = np.arange(g)
    at[..., 1] = np.arange(first, first + rows)[:, None]
    offset %= 1 << 64
    at[..., 2], at[..., 3] = offset & 0xFFFFFFFF, offset >> 32
    w = philox(at, (seed & 0xFFFFFFFF, seed >> 32))
    n = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(rows, 8 * g)[:, :cols]
    return (n >= t) * (65536.0 / (65536 - t) if t < 65536 else 0.0)


def wide(t):
    return None if t is None else t.detach().double().cpu().numpy()


def close(name, got, ref, bound, kind=None):
    """got within half a step of ref plus bound (finite everywhere)."""
    g = wide(got)
    r = half(got) if kind is None else kind
    lim = r * (np.abs(ref) + bound) + bound + 1e-37
    bad = ~(np.abs(g - ref) <= lim)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(g - ref) / lim, 0)), g.shape)
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} beyond their bounds, at {i}: {g[i]} for {ref[i]} "
                             f"(allowed {lim[i]})")


def sum_rows(x, bias, residual, d):
    """residual + D(x + bias) and the bound of its arithmetic (four roundings)."""
    b = 0.0 if bias is None else bias
    s, mag = (x + b) * d, (np.abs(x) + np.abs(b)) * d
    if residual is not None:
        s, mag = s + residual, mag + np.abs(residual)
    return s, 4 * U * mag


def column_sums(terms, each):
    """Sum over rows of terms whose own bounds are `each`, and its bound."""
    return terms.sum(0), (len(terms) + 2) * U * np.abs(terms).sum(0) + np.broadcast_to(each, terms.shape).sum(0)


class Norm:
    """The norm of rows, with bounds of what the library forms of it."""

    C = 96   # roundings of a row's sums: 16 terms a lane, shuffles, waves, and the few operations around

    def __init__(self, total, eps, w, b):
        n = total.shape[1]
        self.n, self.w = n, 1.0 if w is None else w
        self.mean = total.mean(1, keepdims=True)
        z = total - self.mean
        self.rstd = 1.0 / np.sqrt((z * z).mean(1, keepdims=True) + eps)
        self.xhat = z * self.rstd
        off = self.C * U * np.abs(total).mean(1, keepdims=True)   # of the mean
        rel = self.C * U + (off * self.rstd) ** 2                 # of 1 / deviation
        self.rel = rel
        self.ex = self.rstd * off + np.abs(self.xhat) * (rel + 2 * U)   # of xhat
        self.y = self.xhat * self.w + (0.0 if b is None else b)
        self.ey = np.abs(self.w) * self.ex + 4 * U * (np.abs(self.xhat * self.w) + (0.0 if b is None else np.abs(b)))

    def backward(self, dy, dtotal):
        g = dy * self.w
        m0, m1 = g.mean(1, keepdims=True), (g * self.xhat).mean(1, keepdims=True)
        core = g - m0 - self.xhat * m1
        d = self.rstd * core
        e0 = self.C * U * np.abs(g).mean(1, keepdims=True)
        e1 = self.C * U * np.abs(g * self.xhat).mean(1, keepdims=True) + (np.abs(g) * self.ex).mean(1, keepdims=True)
        mag = np.abs(g) + np.abs(m0) + np.abs(self.xhat * m1)
        bound = self.rstd * (6 * U * mag + e0 + np.abs(self.xhat) * e1 + self.ex * np.abs(m1) + self.rel * np.abs(core))
        if dtotal is not None:
            d, bound = d + dtotal, bound + 2 * U * (np.abs(d) + np.abs(dtotal))
        return d, bound


def act(name, u):
    """act(u) and its derivative."""
    if name == "gelu":
        k = math.sqrt(2 / math.pi)
        t = np.tanh(k * (u + 0.044715 * u ** 3))
        return u * (1 + t) / 2, (1 + t) / 2 + u * (1 - t * t) * k * (1 + 3 * 0.044715 * u * u) / 2
    if name == "silu":
        s = 0.5 * (1 + np.tanh(u / 2))
        return u * s, s * (1 + u * (1 - s))
    if name == "relu":
        return np.maximum(u, 0), (u > 0) * 1.0
    return u, np.ones_like(u)


def product(a, b):
    """a b and the bound of a sum of its products in 32 bits (and of parts of it)."""
    return a @ b, (a.shape[1] + 4) * U * (np.abs(a) @ np.abs(b))
