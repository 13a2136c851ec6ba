"""What the performance of the operators of a layer is judged by: dropout whose
mask is never stored, layer norm over a residual sum, and the linear layer with
its bias, activation and residual, over the sizes and types that a training
program, or one that evaluates single tokens, gives them.

Beside each call stands its plain form: the operator's formulas in elementary
torch operations, in 32 bits whatever the tensors' type, rounded once at the end.

Dropout.  y = residual + D(x + bias).  Element (row, column) is kept when its
16-bit number is at least t = round(65536 p), and then multiplied by
65536 / (65536 - t).  The numbers of columns 8 g .. 8 g + 7 of a row are the
halves of the four words, low ones first, that Philox4x32-10 (Salmon et al.,
"Parallel random numbers: as easy as 1, 2, 3", SC 2011) makes of the counter
(g, row, low and high word of offset) under the key seed.  The gradient takes the
same mask, and may be multiplied by the stored derivative of an activation that
the elements went through before.

Layer norm.  total = residual + D(x + bias), as it is stored in its type (x itself
where there is neither residual, dropout nor bias); y is the norm of total over a
row, times weight, plus bias.

Linear.  u = x W + bias, y = act(u) + residual; the derivative act'(u) is stored
for the backward pass, which starts from the gradient at u.  The input's gradient
is multiplied by the derivative of the activation before, where there is one.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
SEED = 0x9D2C5680A5A5F00D


def _dropout(name, rows, cols, dtype="bf16", params="f32", p=0.1, bias=True, residual=True, derivative=False,
             train=True):
    return dict(name=name, kind="dropout", rows=rows, cols=cols, dtype=dtype, params=params, p=p, bias=bias,
                residual=residual, derivative=derivative, train=train)


def _norm(name, rows, cols, dtype="bf16", params="f32", p=0.0, bias=False, residual=False, train=True):
    return dict(name=name, kind="norm", rows=rows, cols=cols, dtype=dtype, params=params, p=p, bias=bias,
                residual=residual, train=train)


def _linear(name, rows, fan_in, fan_out, dtype="bf16", params="f32", act="none", bias=True, residual=False,
            before=False, by_out=False, train=True):
    return dict(name=name, kind="linear", rows=rows, fan_in=fan_in, fan_out=fan_out, dtype=dtype, params=params,
                act=act, bias=bias, residual=residual, before=before, by_out=by_out, train=train)


def listed():
    return [
        # The smallest workload's residual branch (fp32, 128 tokens of 256): launches are all there is.
        _dropout("dropout_tiny", 128, 256, dtype="f32"),
        # The attention branch of a 6.7B layer, one micro-batch: bias, dropout, residual.
        _dropout("dropout_6.7b", 2048, 4096),
        # After the activation of a 6.7B feed-forward layer, two padded sequences: the backward pass
        # takes the activation's derivative and forms the gradient of the bias before it.
        _dropout("dropout_ffn", 4095, 16384, bias=False, residual=False, derivative=True),
        # One token's final norm: latency.
        _norm("norm_token", 1, 5120, train=False),
        # 1.3B layers' norm over two sequences, alone.
        _norm("norm_1.3b", 4096, 2048),
        # Between the sublayers of a 6.7B layer: bias, dropout, residual and norm in one pass.
        _norm("norm_6.7b", 2048, 4096, p=0.1, bias=True, residual=True),
        # The same of 13B layers over eight sequences, parameters held in bf16.
        _norm("norm_13b", 16384, 5120, params="bf16", p=0.1, bias=True, residual=True),
        # fp32 validation at odd sizes.
        _norm("norm_odd", 1013, 1111, dtype="f32", residual=True),
        # One token through the first product of a 6.7B feed-forward layer: the weight's bytes.
        _linear("linear_token", 1, 4096, 16384, act="gelu", train=False),
        # The smallest workload's feed-forward product (fp32).
        _linear("linear_tiny", 128, 256, 1024, dtype="f32", act="gelu"),
        # 6.7B feed-forward layer, first product: bias and activation.
        _linear("linear_6.7b", 2048, 4096, 16384, act="gelu"),
        # 1.3B feed-forward layer, second product, a ragged number of tokens: residual, the activation
        # before it, weights stored [out, in] with a bf16 bias.
        _linear("linear_down", 4001, 8192, 2048, params="bf16", residual=True, before=True, by_out=True),
    ]


def _log(rng, low, high):
    """A whole number between low and high, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(("dropout", "norm", "linear"))
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    params = rng.choice(("f32", "f32", "bf16"))
    train = rng.random() < 0.75
    if kind == "linear":
        fan_in, fan_out = 8 * _log(rng, 2, 2048), 8 * _log(rng, 2, 2048)
        room = int((1.3e11 if dtype == "bf16" else 1.5e10) / (fan_in * fan_out))   # products of one pass
        rows = min(_log(rng, 1, 16384), max(1, room))
        act = rng.choice(("none", "gelu", "silu"))
        case = _linear("", rows, fan_in, fan_out, dtype=dtype, params=params, act=act, bias=rng.random() < 0.8,
                       residual=rng.random() < 0.5, before=rng.random() < 0.5, by_out=rng.random() < 0.5, train=train)
    else:
        cols = _log(rng, 1, 16384)
        if rng.random() < 0.6:
            cols = max(8, cols // 8 * 8)
        rows = _log(rng, 1, max(1, min(32768, int((6e7 if dtype == "bf16" else 3e7) / cols))))
        p = rng.choice((0.05, 0.1, 0.1, 0.5))
        bias, residual = rng.random() < 0.5, rng.random() < 0.6
        if kind == "dropout":
            case = _dropout("", rows, cols, dtype=dtype, params=params, p=p, bias=bias, residual=residual,
                            derivative=not residual and rng.random() < 0.5, train=train)
        else:
            case = _norm("", rows, cols, dtype=dtype, params=params, p=rng.choice((0.0, p)), bias=bias,
                         residual=residual, train=train)
    del case["name"]
    return case


# -- what a program has before the call ------------------------------------------


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    kind, params = _type(case["dtype"]), _type(case["params"])

    def normal(*shape, std=1.0, mean=0.0, to=kind):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(std).add_(mean).to(to)

    st = {"case": case, "offset": (seed << 20) + 5, "bias": None, "residual": None}
    if case["kind"] == "linear":
        rows, i, o = case["rows"], case["fan_in"], case["fan_out"]
        st["x"] = normal(rows, i)
        # stored [in, out], or [out, in] and seen as its transpose
        st["w"] = normal(o, i, std=i ** -0.5).t() if case["by_out"] else normal(i, o, std=i ** -0.5)
        if case["bias"]:
            st["bias"] = normal(o, std=0.5, to=params)
        if case["residual"]:
            st["residual"] = normal(rows, o)
        if case["train"]:
            st["dy"] = normal(rows, o, std=0.1)
            if case["before"]:
                st["before"] = normal(rows, i, std=0.3, mean=0.5)
        return st
    rows, cols = case["rows"], case["cols"]
    # columns of different sizes and a mean of their own, as activations have them
    st["x"] = normal(rows, cols, mean=0.2) * (1 + normal(cols, std=0.3))
    if case["bias"]:
        st["bias"] = normal(cols, std=0.3, to=params)
    if case["residual"]:
        st["residual"] = normal(rows, cols, std=2.0)
    if case["kind"] == "norm":
        st["weight"], st["shift"] = normal(cols, std=0.2, mean=1.0, to=params), normal(cols, std=0.2, to=params)
    if case["train"]:
        st["dy"] = normal(rows, cols, std=0.1)
        if case.get("derivative"):
            st["before"] = normal(rows, cols, std=0.3, mean=0.5)
        if case["kind"] == "norm" and case["residual"]:
            st["dtotal"] = normal(rows, cols, std=0.1)   # what reaches the residual stream from above
    return st


# -- the plain forms --------------------------------------------------------------


def _threshold(p):
    return int(math.floor(65536 * p + 0.5))


def _kept(rows, cols, p, offset):
    """The mask [rows, cols]: words of 32 bits in 64-bit integers."""
    low = 0xFFFFFFFF
    g = torch.arange((cols + 7) // 8, device="cuda")[None, :]
    r = torch.arange(rows, device="cuda")[:, None]
    c = [(g + 0 * r), (r + 0 * g), torch.full_like(g + r, offset & low), torch.full_like(g + r, (offset >> 32) & low)]
    k0, k1 = SEED & low, SEED >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57      # the low 64 bits, which are all there are
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    halves = torch.stack([x for w in c for x in (w & 0xFFFF, w >> 16)], -1)
    return halves.view(rows, -1)[:, :cols] >= _threshold(p)


def _plain_sum(st):
    """residual + D(x + bias) in 32 bits, and D as a factor (None without dropout)."""
    c = st["case"]
    s = st["x"].float()
    if st["bias"] is not None:
        s = s + st["bias"].float()
    factor = None
    if c["p"]:
        t = _threshold(c["p"])
        factor = torch.where(_kept(c["rows"], c["cols"], c["p"], st["offset"]), 65536 / (65536 - t), 0.0)
        s = s * factor
    if st["residual"] is not None:
        s = s + st["residual"].float()
    return s, factor


def _plain_dropout(st):
    c, kind = st["case"], st["x"].dtype
    s, factor = _plain_sum(st)
    out = {"y": s.to(kind)}
    if c["train"]:
        dx = st["dy"].float() * factor
        if c["derivative"]:
            dx = dx * st["before"].float()
        out["dx"] = dx.to(kind)
        if c["bias"] or c["derivative"]:
            out["dbias"] = dx.sum(0)
    return out


def _plain_norm(st):
    c, kind = st["case"], st["x"].dtype
    s, factor = _plain_sum(st)
    added = c["p"] or c["bias"] or c["residual"]
    total = s.to(kind)
    s = total.float()
    z = s - s.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((z * z).mean(1, keepdim=True) + EPS)
    xhat = z * rstd
    w = st["weight"].float()
    out = {"y": (xhat * w + st["shift"].float()).to(kind)}
    if added:
        out["total"] = total
    if not c["train"]:
        return out
    dy = st["dy"].float()
    g = dy * w
    d = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if c["residual"]:
        d = d + st["dtotal"].float()
    dx = d if factor is None else d * factor
    out["dx"] = dx.to(kind)
    if c["residual"]:
        out["dresidual"] = d.to(kind)
    out["dweight"], out["dshift"] = (dy * xhat).sum(0), dy.sum(0)
    if c["bias"]:
        out["dbias"] = dx.sum(0)
    return out


def _plain_act(act, u):
    """act(u) and its derivative."""
    if act == "gelu":   # the tanh form
        a = math.sqrt(2 / math.pi)
        s = 1.0 / (1.0 + torch.exp(-2 * a * (u + 0.044715 * u * u * u)))
        return u * s, s + 2 * u * s * (1 - s) * a * (1 + 3 * 0.044715 * u * u)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-u))
        return u * s, s * (1 + u * (1 - s))
    raise ValueError(act)


def _plain_linear(st):
    c, kind = st["case"], st["x"].dtype
    x, w = st["x"].float(), st["w"].float()
    y = torch.matmul(x, w)
    if c["bias"]:
        y = y + st["bias"].float()
    out = {}
    if c["act"] != "none":
        y, slope = _plain_act(c["act"], y)
        if c["train"]:
            out["derivative"] = slope.to(kind)
    if c["residual"]:
        y = y + st["residual"].float()
    out["y"] = y.to(kind)
    if not c["train"]:
        return out
    dy = st["dy"].float()
    dx = torch.matmul(dy, w.t())
    if c["before"]:
        dx = dx * st["before"].float()
    out["dx"] = dx.to(kind)
    out["dw"] = torch.matmul(dy.t(), x).t() if c["by_out"] else torch.matmul(x.t(), dy)
    if c["bias"]:
        out["db"] = dy.sum(0)
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"dropout": _own_dropout, "norm": _own_norm, "linear": _own_linear}[kind](state)
    return {"dropout": _plain_dropout, "norm": _plain_norm, "linear": _plain_linear}[kind](state)


# -- the package's calls ------------------------------------------------------------


def _own_dropout(st):
    from paper_2405_14009_amd import Dropout, dropout_backward, dropout_forward
    c = st["case"]
    drop = Dropout(c["p"], SEED, st["offset"])
    out = {"y": dropout_forward(st["x"], drop, bias=st["bias"], residual=st["residual"])}
    if c["train"]:
        wants = c["bias"] or c["derivative"]
        dx, dbias = dropout_backward(st["dy"], drop, derivative=st.get("before"), bias_grad=wants)
        out["dx"] = dx
        if wants:
            out["dbias"] = dbias
    return out


def _own_norm(st):
    from paper_2405_14009_amd import Dropout, layer_norm_backward, layer_norm_forward
    c = st["case"]
    drop = Dropout(c["p"], SEED, st["offset"]) if c["p"] else None
    y, total, stats = layer_norm_forward(st["x"], st["weight"], st["shift"], eps=EPS, in_bias=st["bias"], drop=drop,
                                         residual=st["residual"], save=c["train"])
    out = {"y": y}
    if c["p"] or c["bias"] or c["residual"]:
        out["total"] = total
    if not c["train"]:
        return out
    grads = layer_norm_backward(st["dy"], total, stats, st["weight"], dtotal=st.get("dtotal"), drop=drop,
                                in_bias_grad=c["bias"])
    out["dx"], out["dweight"], out["dshift"] = grads.dx, grads.dweight, grads.dbias
    if c["residual"]:
        out["dresidual"] = grads.dtotal
    if c["bias"]:
        out["dbias"] = grads.din_bias
    return out


def _own_linear(st):
    from paper_2405_14009_amd import linear_backward_input, linear_backward_weight, linear_forward
    c = st["case"]
    act = None if c["act"] == "none" else c["act"]
    y, slope = linear_forward(st["x"], st["w"], st["bias"], activation=act, residual=st["residual"], save=c["train"])
    out = {"y": y}
    if not c["train"]:
        return out
    if act:
        out["derivative"] = slope
    out["dx"] = linear_backward_input(st["dy"], st["w"], derivative=st.get("before"))
    out["dw"], db = linear_backward_weight(st["x"], st["dy"], by_out=c["by_out"], bias_grad=c["bias"])
    if c["bias"]:
        out["db"] = db
    return out


# -- work and exact results -----------------------------------------------------------


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    vector = 4 if case["params"] == "f32" else 2
    if case["kind"] == "linear":
        rows, i, o = case["rows"], case["fan_in"], case["fan_out"]
        nbytes = size * (rows * i + i * o + rows * o * (2 if case["residual"] else 1)) + vector * o * case["bias"]
        flops = 2.0 * rows * i * o
        if case["train"]:
            nbytes += size * rows * o * (2 if case["act"] != "none" else 1)          # derivative out, dy in
            nbytes += size * rows * i * (2 if case["before"] else 1)                 # dx, derivative before
            nbytes += 4 * i * o + 4 * o * case["bias"]
            flops *= 3
        return {"bytes": nbytes, "flops": flops}
    n, cols = case["rows"] * case["cols"], case["cols"]
    if case["kind"] == "dropout":
        nbytes, flops = size * n * (3 if case["residual"] else 2) + vector * cols * case["bias"], 14.0 * n
        if case["train"]:
            nbytes += size * n * (3 if case["derivative"] else 2) + 4 * cols * (case["bias"] or case["derivative"])
            flops += 14.0 * n
        return {"bytes": nbytes, "flops": flops}
    added = bool(case["p"] or case["bias"] or case["residual"])
    nbytes = size * n * (2 + added + case["residual"]) + vector * cols * (2 + case["bias"])
    flops = 8.0 * n + (12.0 * n if case["p"] else 0.0)
    if case["train"]:
        # dy and dtotal in, dx and dresidual out; total counts as written once and kept (x where nothing is added)
        nbytes += size * n * (2 + (2 if case["residual"] else 0)) + 4 * cols * (2 + case["bias"])
        flops += 12.0 * n + (12.0 * n if case["p"] else 0.0)
    return {"bytes": nbytes, "flops": flops}


def _exact_factor(case, offset):
    """D as a factor in 64 bits, from products of 16-bit limbs."""
    def mul(a, m):   # high and low words of the product of 32-bit numbers
        ml, mh = m % 65536, m // 65536
        al, ah = a % 65536, a // 65536
        ll, mid = al * ml, ah * ml
        other = al * mh + mid % 65536 + ll // 65536
        return ah * mh + mid // 65536 + other // 65536, (other % 65536) * 65536 + ll % 65536

    rows, cols = case["rows"], case["cols"]
    groups = -(-cols // 8)
    at = torch.arange(rows * groups, device="cuda")
    x0, x1 = at % groups, torch.div(at, groups, rounding_mode="floor")
    x2 = torch.zeros_like(at) + offset % 2 ** 32
    x3 = torch.zeros_like(at) + offset // 2 ** 32
    for n in range(10):
        key0 = (SEED % 2 ** 32 + n * 0x9E3779B9) % 2 ** 32
        key1 = (SEED // 2 ** 32 + n * 0xBB67AE85) % 2 ** 32
        h0, l0 = mul(x0, 0xD2511F53)
        h1, l1 = mul(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = torch.bitwise_xor(torch.bitwise_xor(h1, x1), key0), l1, \
            torch.bitwise_xor(torch.bitwise_xor(h0, x3), key1), l0
    t = round(case["p"] * 65536)
    out = torch.empty(rows, groups, 8, dtype=torch.float64, device="cuda")
    for j, word in enumerate((x0, x1, x2, x3)):
        out[:, :, 2 * j] = (word % 65536 >= t).view(rows, groups)
        out[:, :, 2 * j + 1] = (torch.div(word, 65536, rounding_mode="floor") >= t).view(rows, groups)
    return out.view(rows, 8 * groups)[:, :cols] * (65536.0 / (65536 - t))


def _exact_rows(case, st):
    factor = _exact_factor(case, st["offset"]) if case["p"] else 1.0
    s = st["x"].double()
    if case["bias"]:
        s += st["bias"].double()
    s = s * factor
    if case["residual"]:
        s += st["residual"].double()
    if case["kind"] == "dropout":
        out = {"y": s}
        if case["train"]:
            dx = st["dy"].double() * factor
            if case["derivative"]:
                dx *= st["before"].double()
            out["dx"] = dx
            if case["bias"] or case["derivative"]:
                out["dbias"] = dx.sum(0)
        return out
    out = {"total": s} if case["p"] or case["bias"] or case["residual"] else {}
    n = case["cols"]
    s = s.to(st["x"].dtype).double()   # the norm is that of the total as it is stored
    var, mean = torch.var_mean(s, 1, correction=0, keepdim=True)
    root = torch.sqrt(var + EPS)
    xhat = (s - mean) / root
    w = st["weight"].double()
    out["y"] = w * xhat + st["shift"].double()
    if not case["train"]:
        return out
    dy = st["dy"].double()
    g = dy * w
    d = (n * g - g.sum(1, keepdim=True) - xhat * (g * xhat).sum(1, keepdim=True)) / (n * root)
    if case["residual"]:
        d += st["dtotal"].double()
        out["dresidual"] = d
    out["dx"] = d * factor
    out["dweight"], out["dshift"] = (xhat * dy).sum(0), dy.sum(0)
    if case["bias"]:
        out["dbias"] = out["dx"].sum(0)
    return out


def _exact_linear(case, st):
    x, w = st["x"].double(), st["w"].double()
    u = x @ w
    if case["bias"]:
        u += st["bias"].double()
    out = {}
    if case["act"] != "none":
        if case["act"] == "gelu":
            k = math.sqrt(2 / math.pi)
            t = torch.tanh(k * (u + 0.044715 * u ** 3))
            y = u * (1 + t) / 2
            slope = (1 + t) / 2 + u * (1 - t * t) * k * (1 + 0.134145 * u ** 2) / 2
        else:   # silu
            e = torch.sigmoid(u)
            y, slope = u * e, e + u * e * torch.sigmoid(-u)
        if case["train"]:
            out["derivative"] = slope
    else:
        y = u
    out["y"] = y + st["residual"].double() if case["residual"] else y
    if not case["train"]:
        return out
    dy = st["dy"].double()
    out["dx"] = dy @ w.T
    if case["before"]:
        out["dx"] *= st["before"].double()
    out["dw"] = (dy.T @ x).T if case["by_out"] else x.T @ dy
    if case["bias"]:
        out["db"] = dy.sum(0)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_linear(case, st) if case["kind"] == "linear" else _exact_rows(case, st)
