"""Dropout, layer norm and linear layers on the caller's tensors against their
plain 64-bit forms, at the sizes and layouts where they can go wrong."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
KINDS = pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
SEED, OFFSET = 0xFEDCBA9876543210, (7 << 32) + 11


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")


def ops():
    import paper_2405_14009_amd as pkg
    return pkg


def normal(seed, *shape, std=1.0, mean=0.0, kind=BF16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std + mean).to(kind).cuda()


def strided(t, left, gap):
    """The same values as columns left .. of a wider matrix."""
    wide = torch.full((t.shape[0], left + t.shape[1] + gap), 9.0, dtype=t.dtype, device="cuda")
    wide[:, left:left + t.shape[1]] = t
    return wide[:, left:left + t.shape[1]]


# -- dropout ---------------------------------------------------------------------

ROWS = [(1, 1), (1, 7), (3, 8), (5, 9), (2, 31), (64, 33), (65, 64), (33, 129), (1, 513), (257, 255), (130, 1025),
        (7, 2048), (19, 2051), (600, 24), (1000, 1), (4099, 3), (3, 16385), (700, 520)]


def check_dropout(rows, cols, kind, p, bias, residual, derivative, params=F32, layout=lambda t: t, seed=3):
    x = layout(normal(seed, rows, cols, kind=kind))
    b = normal(seed + 1, cols, kind=params) if bias else None
    r = layout(normal(seed + 2, rows, cols, std=2.0, kind=kind)) if residual else None
    dy = layout(normal(seed + 3, rows, cols, std=0.1, kind=kind))
    s = layout(normal(seed + 4, rows, cols, mean=0.5, kind=kind)) if derivative else None
    drop = ops().Dropout(p, SEED, OFFSET)
    d = ref.factor(rows, cols, p, SEED, OFFSET)
    y = ops().dropout_forward(x, drop, bias=b, residual=r)
    ref.close("y", y, *ref.sum_rows(ref.wide(x), ref.wide(b), ref.wide(r), d))
    dx, db = ops().dropout_backward(dy, drop, derivative=s, bias_grad=True)
    want = ref.wide(dy) * d * (1.0 if s is None else ref.wide(s))
    ref.close("dx", dx, want, 3 * ref.U * np.abs(want))
    ref.close("dbias", db, *ref.column_sums(want, 3 * ref.U * np.abs(want)))
    alone, none = ops().dropout_backward(dy, drop, derivative=s)
    assert none is None and torch.equal(alone, dx)
    return y, dx, db


@KINDS
@pytest.mark.parametrize("rows,cols", ROWS)
def test_dropout(rows, cols, kind):
    check_dropout(rows, cols, kind, 0.1, True, True, False)
    check_dropout(rows, cols, kind, 0.5, False, False, True)


@KINDS
@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.3, 1 - 2.0 ** -16, 1.0])
def test_dropout_probabilities(p, kind):
    y, dx, _ = check_dropout(37, 203, kind, p, True, False, False)
    if p == 1.0:
        assert not y.any() and not dx.any()


@KINDS
@pytest.mark.parametrize("left,gap", [(0, 1), (1, 0), (3, 8), (8, 16)])
@pytest.mark.parametrize("cols", [40, 43, 5])
def test_dropout_of_columns_of_a_wider_matrix(cols, left, gap, kind):
    check_dropout(21, cols, kind, 0.2, True, True, False, params=BF16, layout=lambda t: strided(t, left, gap))


def test_dropout_keeps_what_lies_around_its_output():
    wide = torch.full((9, 64), 5.0, dtype=BF16, device="cuda")
    for left, cols in ((0, 8), (3, 13), (20, 3), (30, 34)):
        before = wide.clone()
        out = wide[2:7, left:left + cols]
        ops().dropout_forward(normal(1, 5, cols), ops().Dropout(0.5, 1), out=out)
        before[2:7, left:left + cols] = out
        assert torch.equal(wide, before)


def test_dropout_mask_is_that_of_rows_and_columns():
    """Shapes, types and leading dimensions do not matter, only (row, column)."""
    x = torch.ones(4, 6, 77, device="cuda")
    drop = ops().Dropout(0.25, 5, 9)
    a = ops().dropout_forward(x, drop)
    b = ops().dropout_forward(x.view(24, 77)[:11, :50], drop)
    c = ops().dropout_forward(x[0, 0, :].to(BF16), drop)
    assert torch.equal(a.view(24, 77)[:11, :50], b)
    assert torch.equal(a[0, 0] != 0, c != 0)
    for other in (ops().Dropout(0.25, 5, 10), ops().Dropout(0.25, 6, 9), ops().Dropout(0.25, 5 + (1 << 40), 9),
                  ops().Dropout(0.25, 5, 9 + (1 << 40))):
        assert not torch.equal(a, ops().dropout_forward(x, other))


def test_dropped_infinities_and_nan_are_zero():
    d = ref.factor(8, 64, 0.5, SEED, OFFSET)
    x = normal(1, 8, 64)
    x[torch.tensor(d == 0)] = float("nan")
    y = ops().dropout_forward(x, ops().Dropout(0.5, SEED, OFFSET))
    assert torch.isfinite(y).all() and not y[torch.tensor(d == 0)].any()
    x[torch.tensor(d == 0)] = float("inf")
    dx, db = ops().dropout_backward(x, ops().Dropout(0.5, SEED, OFFSET), bias_grad=True)
    assert torch.isfinite(dx).all() and torch.isfinite(db).all()


def test_dropout_takes_its_step_from_the_device():
    x, step = normal(1, 30, 40), torch.tensor([5], dtype=torch.int64, device="cuda")
    drop = ops().Dropout(0.4, SEED, 100, step=step)
    assert torch.equal(ops().dropout_forward(x, drop), ops().dropout_forward(x, ops().Dropout(0.4, SEED, 105)))
    step.fill_(-1)   # modulo 2^64
    assert torch.equal(ops().dropout_forward(x, drop), ops().dropout_forward(x, ops().Dropout(0.4, SEED, 99)))


def test_dropout_beyond_32_bits_of_elements():
    """2^31 + elements, of which the last rows are looked at; all rows of x are one."""
    cols, rows = 32776, 66000
    x = normal(1, 1, cols).expand(rows, cols)
    drop = ops().Dropout(0.1, SEED, OFFSET)
    y = ops().dropout_forward(x, drop)
    d = ref.factor(5, cols, 0.1, SEED, OFFSET, first=rows - 5)
    ref.close("y", y[-5:], *ref.sum_rows(ref.wide(x[-5:]), None, None, d))
    del y
    dx, db = ops().dropout_backward(x, drop, bias_grad=True)
    ref.close("dx", dx[-5:], *ref.sum_rows(ref.wide(x[-5:]), None, None, d))
    # 0.9 rows of x / 0.9 each: eight deviations of the kept ones' number, and the sums' bound
    xs = ref.wide(x[0])
    slack = 8 * np.sqrt(rows * 0.1 / 0.9) + rows * ref.U * rows / 0.9
    assert (np.abs(ref.wide(db) - rows * xs) <= slack * np.abs(xs)).all()


# -- layer norm -------------------------------------------------------------------

NORMS = [(1, 1), (3, 2), (1, 8), (5, 7), (70, 32), (3, 33), (65, 100), (17, 128), (9, 129), (33, 512), (2, 513),
         (40, 1000), (5, 1024), (7, 1025), (600, 1032), (1, 2048), (21, 2049), (3, 4096), (4, 4097), (2, 8192), (5, 8200),
         (3, 16383), (2, 16384), (1300, 200), (2100, 9), (1, 5120)]


def check_norm(rows, cols, kind, p=0.0, bias=False, residual=False, affine=True, params=F32, layout=lambda t: t, seed=3,
               mean=0.2, std=1.0, eps=1e-5):
    x = layout(normal(seed, rows, cols, mean=mean, std=std, kind=kind))
    ib = normal(seed + 1, cols, std=0.3, kind=params) if bias else None
    r = layout(normal(seed + 2, rows, cols, std=2.0, kind=kind)) if residual else None
    w = normal(seed + 3, cols, std=0.2, mean=1.0, kind=params) if affine else None
    b = normal(seed + 4, cols, std=0.2, kind=params) if affine else None
    dy = layout(normal(seed + 5, rows, cols, std=0.1, kind=kind))
    dt = layout(normal(seed + 6, rows, cols, std=0.1, kind=kind)) if residual else None
    drop = ops().Dropout(p, SEED, OFFSET) if p else None
    d = ref.factor(rows, cols, p, SEED, OFFSET)
    y, total, stats = ops().layer_norm_forward(x, w, b, eps=eps, in_bias=ib, drop=drop, residual=r)
    if p or bias or residual:
        ref.close("total", total, *ref.sum_rows(ref.wide(x), ref.wide(ib), ref.wide(r), d))
    else:
        assert total is x
    n = ref.Norm(ref.wide(total), float(np.float32(eps)), ref.wide(w), ref.wide(b))
    ref.close("y", y, n.y, n.ey)
    how = dict(dtotal=dt, drop=drop)
    g = ops().layer_norm_backward(dy, total, stats, w, in_bias_grad=True, **how)
    want, bound = n.backward(ref.wide(dy), ref.wide(dt))
    ref.close("dtotal", g.dtotal, want, bound)
    ref.close("dx", g.dx, want * d, (bound + 2 * ref.U * np.abs(want)) * d)
    ref.close("dweight", g.dweight, *ref.column_sums(ref.wide(dy) * n.xhat, np.abs(ref.wide(dy)) * n.ex))
    ref.close("dbias", g.dbias, *ref.column_sums(ref.wide(dy), 0.0))
    ref.close("din_bias", g.din_bias, *ref.column_sums(want * d, (bound + 2 * ref.U * np.abs(want)) * d))
    # the same in two calls
    a = ops().layer_norm_backward(dy, total, stats, w, weight_grad=False, bias_grad=False, **how)
    assert torch.equal(a.dtotal, g.dtotal) and torch.equal(a.dx, g.dx) and a.dweight is None and a.din_bias is None
    a = ops().layer_norm_backward(dy, total, stats, w, input_grad=False, in_bias_grad=True, **how)
    assert a.dx is None and a.dtotal is None
    for name in ("dweight", "dbias", "din_bias"):
        assert torch.equal(getattr(a, name), getattr(g, name)), name
    return y, total, stats, g


@KINDS
@pytest.mark.parametrize("rows,cols", NORMS)
def test_norm(rows, cols, kind):
    check_norm(rows, cols, kind)
    check_norm(rows, cols, kind, 0.1, True, True, params=BF16)


@KINDS
def test_norm_parts_of_the_sum(kind):
    check_norm(13, 300, kind, residual=True)
    check_norm(13, 300, kind, 0.5)
    check_norm(13, 300, kind, bias=True)
    check_norm(13, 300, kind, affine=False)
    check_norm(13, 300, kind, mean=100.0, std=0.5)   # a mean far above the deviation
    check_norm(13, 300, kind, mean=3.0, std=0.0)     # rows of one value
    check_norm(13, 300, kind, eps=0.5)


@KINDS
@pytest.mark.parametrize("cols,left,gap", [(40, 0, 1), (43, 1, 0), (600, 3, 5), (5, 2, 2), (1030, 8, 2)])
def test_norm_of_columns_of_a_wider_matrix(cols, left, gap, kind):
    check_norm(11, cols, kind, 0.2, True, True, layout=lambda t: strided(t, left, gap))


def test_norm_of_a_large_row_sum_in_bf16():
    """Values whose squares sum beyond bf16 and fp16, and near the end of fp32's squares."""
    check_norm(4, 4096, BF16, std=300.0)
    check_norm(4, 96, F32, std=1e15)


@KINDS
def test_rows_that_share_their_memory(kind):
    """Inputs broadcast over rows, as an expanded tensor has them."""
    x, r = normal(1, 1, 77, kind=kind), normal(2, 9, 77, kind=kind)
    wide = x.expand(9, 77)
    drop = ops().Dropout(0.3, SEED, OFFSET)
    for a, b in ((wide, wide.contiguous()),):
        one = ops().layer_norm_forward(a, drop=drop, residual=r)
        two = ops().layer_norm_forward(b, drop=drop, residual=r)
        assert all(torch.equal(p, q) for p, q in zip(one, two))
        g = ops().layer_norm_backward(a, one[1], one[2], drop=drop)
        h = ops().layer_norm_backward(b, one[1], one[2], drop=drop)
        assert all(torch.equal(p, q) for p, q in zip(g[:4], h[:4]))
    assert torch.equal(ops().dropout_forward(r, drop, residual=wide), ops().dropout_forward(r, drop, residual=wide.contiguous()))


@KINDS
def test_nan_stays_in_its_row(kind):
    x = normal(1, 6, 100, kind=kind)
    x[2, 50] = float("nan")
    x[4, 7] = float("inf")
    y, total, stats = ops().layer_norm_forward(x, None, None)
    g = ops().layer_norm_backward(torch.ones_like(x), total, stats)
    for t in (y, g.dx):
        ok = torch.isfinite(t).all(1).tolist()
        assert ok == [True, True, False, True, False, True]


def test_accumulated_gradients():
    y, total, stats, g = check_norm(50, 300, BF16, 0.1, True, True)
    dy = normal(8, 50, 300)
    old = [torch.full((300,), v, device="cuda") for v in (1.0, 2.0, 3.0)]
    drop = ops().Dropout(0.1, SEED, OFFSET)
    one = ops().layer_norm_backward(dy, total, stats, None, drop=drop, in_bias_grad=True)
    two = ops().layer_norm_backward(dy, total, stats, None, drop=drop, weight_grad=old[0].clone(), bias_grad=old[1].clone(),
                                    in_bias_grad=old[2].clone(), accumulate=True)
    for name, o in zip(("dweight", "dbias", "din_bias"), old):
        assert torch.equal(getattr(two, name), o + getattr(one, name))
    base = torch.full((300,), 4.0, device="cuda")
    _, db = ops().dropout_backward(dy, drop, bias_grad=True)
    ops().dropout_backward(dy, drop, bias_grad=base, accumulate=True)
    assert torch.equal(base, db + 4.0)


@KINDS
def test_no_rows(kind):
    x = torch.empty(0, 40, dtype=kind, device="cuda")
    drop = ops().Dropout(0.1, 1)
    assert ops().dropout_forward(x, drop).shape == (0, 40)
    dx, db = ops().dropout_backward(x, drop, bias_grad=True)
    assert dx.shape == (0, 40) and not db.any()
    y, total, stats = ops().layer_norm_forward(x, residual=x)
    g = ops().layer_norm_backward(x, total, stats, bias_grad=torch.ones(40, device="cuda"),
                                  weight_grad=torch.ones(40, device="cuda"), accumulate=True)
    assert y.shape == (0, 40) and (g.dweight == 1).all() and (g.dbias == 1).all()
    w = normal(1, 40, 16, kind=kind)
    assert ops().linear_forward(x, w)[0].shape == (0, 16)
    dy = torch.empty(0, 16, dtype=kind, device="cuda")
    assert ops().linear_backward_input(dy, w).shape == (0, 40)
    for by_out in (False, True):
        dw, db = ops().linear_backward_weight(x, dy, by_out=by_out)
        assert dw.shape == (40, 16) and not dw.any() and not db.any()
        base, bias = torch.ones_like(dw), torch.ones_like(db)
        ops().linear_backward_weight(x, dy, by_out=by_out, weight_grad=base, bias_grad=bias, accumulate=True)
        assert (base == 1).all() and (bias == 1).all()


# -- linear ------------------------------------------------------------------------

LINEAR = [(1, 8, 8), (1, 256, 1024), (4, 40, 1032), (5, 1032, 40), (8, 24, 2088), (9, 72, 2056), (2, 1024, 64), (3, 64, 200), (7, 520, 24), (17, 72, 1000), (31, 136, 136), (32, 8, 512),
          (33, 64, 64), (65, 1040, 8), (129, 200, 328), (257, 264, 136), (300, 2048, 72), (1000, 24, 16), (70, 8, 4096),
          (513, 520, 520)]


def check_linear(rows, i, o, kind, act, bias=True, residual=True, before=True, by_out=False, params=F32,
                 layout=lambda t: t, seed=3):
    x, dy = layout(normal(seed, rows, i, kind=kind)), layout(normal(seed + 1, rows, o, std=0.1, kind=kind))
    w = normal(seed + 2, i, o, std=i ** -0.5, kind=kind)
    if by_out:
        w = w.t().contiguous().t()
    b = normal(seed + 3, o, std=0.5, kind=params) if bias else None
    r = layout(normal(seed + 4, rows, o, kind=kind)) if residual else None
    s = layout(normal(seed + 5, rows, i, mean=0.5, kind=kind)) if before else None
    X, W, DY = ref.wide(x), ref.wide(w), ref.wide(dy)
    y, slope = ops().linear_forward(x, w, b, activation=act, residual=r)
    u, e = ref.product(X, W)
    if bias:
        u, e = u + ref.wide(b), e + ref.U * (np.abs(u) + np.abs(ref.wide(b)))
    value, d = ref.act(act, u)
    # slopes of the activations and of their derivatives are below 1.2; the logistic in
    # hardware operations is off by 2^-21 of itself per unit of its argument, which counts
    # up to about 16 (beyond, it or its distance from 1 is below 2^-22)
    e = 1.2 * e
    if act in ("gelu", "silu"):
        e = e + (1 + np.abs(u)) * 2.0 ** -19
    total = value if r is None else value + ref.wide(r)
    ref.close("y", y, total, e + 2 * ref.U * (np.abs(value) + np.abs(total)))
    if act is None:
        assert slope is None
    elif act == "relu":
        sure = np.abs(u) > e
        assert np.array_equal(ref.wide(slope)[sure], d[sure])
    else:
        ref.close("derivative", slope, d, e + 8 * ref.U)
    dx = ops().linear_backward_input(dy, w, derivative=s)
    want, e = ref.product(DY, W.T)
    if before:
        want, e = want * ref.wide(s), (e + ref.U * np.abs(want)) * np.abs(ref.wide(s))
    ref.close("dx", dx, want, e)
    dw, db = ops().linear_backward_weight(x, dy, by_out=by_out)
    assert dw.shape == (i, o) and dw.dtype is F32 and (dw.t() if by_out else dw).is_contiguous()
    ref.close("dw", dw, *ref.product(X.T, DY))
    ref.close("db", db, *ref.column_sums(DY, 0.0))
    again, none = ops().linear_backward_weight(x, dy, by_out=by_out, bias_grad=False)
    assert none is None and torch.equal(again, dw)
    # on top of what is there: one addition more
    base = torch.ones_like(dw)
    ops().linear_backward_weight(x, dy, by_out=by_out, weight_grad=base, bias_grad=False, accumulate=True)
    ref.close("accumulated", base, ref.wide(dw) + 1.0, 4 * ref.U * (np.abs(ref.wide(dw)) + 1.0)
              + ref.product(X.T, DY)[1])
    return y, slope


@KINDS
@pytest.mark.parametrize("rows,i,o", LINEAR)
def test_linear(rows, i, o, kind):
    check_linear(rows, i, o, kind, "gelu")
    check_linear(rows, i, o, kind, None, bias=False, residual=False, before=False, by_out=True)
    check_linear(rows, i, o, kind, "silu", residual=False, by_out=True, params=BF16)


@KINDS
@pytest.mark.parametrize("rows,i,o", [(1, 64, 72), (40, 72, 64), (700, 512, 1536), (2100, 264, 1032), (4100, 1032, 264),
                                      (2100, 1032, 2056), (300, 2056, 2312)])
def test_linear_larger_tiles(rows, i, o, kind):
    check_linear(rows, i, o, kind, "relu", params=BF16)
    check_linear(rows, i, o, kind, None, by_out=True)


@pytest.mark.parametrize("by_out", [False, True])
@pytest.mark.parametrize("rows,i,o", [(1, 8192, 4104), (3, 1024, 20480), (64, 4104, 8192), (33, 2048, 8200), (65, 4096, 4096),
                                      (1, 4096, 1024), (32, 1032, 4104), (2, 16384, 2056)])
def test_linear_of_few_rows_and_a_large_weight(rows, i, o, by_out):
    """Plans of few rows: the weight streamed by the whole card, or one launch."""
    x, dy, b = normal(1, rows, i), normal(2, rows, o, std=0.1), normal(3, o, kind=F32)
    w = normal(4, i, o, std=i ** -0.5)
    if by_out:
        w = w.t().contiguous().t()
    X, W, DY = ref.wide(x), ref.wide(w), ref.wide(dy)
    y, _ = ops().linear_forward(x, w, b)
    u, e = ref.product(X, W)
    ref.close("y", y, u + ref.wide(b), e + ref.U * (np.abs(u) + np.abs(ref.wide(b))))
    ref.close("dx", ops().linear_backward_input(dy, w), *ref.product(DY, W.T))


@pytest.mark.parametrize("by_out", [False, True])
@pytest.mark.parametrize("rows,i,o", [(1, 4096, 4096), (100, 256, 200), (640, 1024, 1024), (300, 4096, 4096), (1111, 2048, 8192),
                                      (2048, 4096, 12288), (9001, 4096, 12288), (20000, 512, 512), (5000, 1536, 768),
                                      (40, 64, 16384), (3, 16384, 64)])
def test_bias_gradient_of_every_tile(rows, i, o, by_out):
    """Sums on the way of the product, whatever tile and split the sizes take; the weight's gradient is
    that of a call without them."""
    x, dy = normal(1, rows, i), normal(2, rows, o, std=0.1)
    dw, db = ops().linear_backward_weight(x, dy, by_out=by_out)
    ref.close("db", db, *ref.column_sums(ref.wide(dy), 0.0))
    plain, _ = ops().linear_backward_weight(x, dy, by_out=by_out, bias_grad=False)
    # in another order at most
    mag = (rows + 2) * ref.U * (x.float().abs().t() @ dy.float().abs())
    assert ((dw - plain).abs() <= 2.01 * mag).all()
    old = torch.ones(o, device="cuda")
    _, db2 = ops().linear_backward_weight(x, dy, by_out=by_out, weight_grad=torch.zeros_like(dw), bias_grad=old,
                                          accumulate=True)
    assert torch.equal(db2, db + 1.0)


@KINDS
def test_linear_of_columns_of_a_wider_matrix(kind):
    for rows in (1, 9, 150):
        check_linear(rows, 64, 40, kind, "gelu", layout=lambda t: strided(t, 16, 8))
        check_linear(rows, 64, 40, kind, None, by_out=True, layout=lambda t: strided(t, 8, 24))


def test_linear_weight_with_gaps_between_its_rows():
    wide = normal(1, 80, 128, std=0.1)
    x, dy = normal(2, 30, 64), normal(3, 30, 96)
    w = wide[:64, 16:112]
    y, _ = ops().linear_forward(x, w)
    ref.close("y", y, *ref.product(ref.wide(x), ref.wide(w)))
    ref.close("dx", ops().linear_backward_input(dy, w), *ref.product(ref.wide(dy), ref.wide(w).T))
    w = wide[:64, 16:112].t()    # stored [out, in]
    y, _ = ops().linear_forward(dy, w)
    ref.close("y", y, *ref.product(ref.wide(dy), ref.wide(w)))


@KINDS
def test_activations_of_large_arguments(kind):
    """0, the identity or NaN, never the product of 0 and infinity."""
    inf = float("inf")
    x = torch.zeros(6, 8, dtype=kind, device="cuda")
    x[:, 0] = torch.tensor([-1e30, -60.0, 60.0, 1e30, inf, float("nan")])
    w = torch.eye(8, dtype=kind, device="cuda")
    for act in ("gelu", "silu", "relu"):
        y, s = ops().linear_forward(x[:5].nan_to_num(posinf=3e38), w, activation=act)
        big = x[:5, 0].nan_to_num(posinf=3e38)
        # at 60 silu is off by 60 e^-60, below a step of anything near 60
        assert torch.equal(y[2:, 0], big[2:]) and (y[:2, 0].abs() < 1e-23).all(), act
        assert torch.equal(s[2:, 0], torch.ones_like(s[2:, 0])) and (s[:2, 0].abs() < 1e-23).all(), act
        y, _ = ops().linear_forward(x[5:], w, activation=act)
        assert torch.isnan(y[0, 0])


def test_linear_beyond_a_buffer_s_reach():
    """bf16 activations of more than 2^31 bytes run in parts."""
    rows, i, o = 35000, 32768, 8
    one = normal(1, 1, i)
    x = one.repeat(rows, 1)
    x[-3:] = normal(2, 3, i)
    w = normal(3, i, o, std=i ** -0.5)
    y, _ = ops().linear_forward(x, w)
    want, e = ref.product(ref.wide(x[-3:]), ref.wide(w))
    ref.close("y", y[-3:], want, e)
    assert (y[:-3] == y[0]).all()
    dy = normal(4, rows, o, std=0.1)
    dx = ops().linear_backward_input(dy, w)
    ref.close("dx", dx[-3:], *ref.product(ref.wide(dy[-3:]), ref.wide(w).T))
    del dx
    dw, db = ops().linear_backward_weight(x, dy)
    D = ref.wide(dy)
    want = np.outer(ref.wide(one)[0], D[:-3].sum(0)) + ref.wide(x[-3:]).T @ D[-3:]
    mag = np.outer(np.abs(ref.wide(one)[0]), np.abs(D[:-3]).sum(0)) + np.abs(ref.wide(x[-3:])).T @ np.abs(D[-3:])
    ref.close("dw", dw, want, rows * ref.U * mag)
    ref.close("db", db, *ref.column_sums(D, 0.0))


@KINDS
@pytest.mark.parametrize("i,o", [(65535 * 32, 8), ((1 << 21) - 8, 8), (8, (1 << 21) - 8)])
def test_weight_gradient_of_a_token_and_many_columns(i, o, kind):
    """At both sides of the most rows that few tokens' outer products take."""
    for rows in (1, 3):
        x, dy = normal(1, rows, i, kind=kind), normal(2, rows, o, kind=kind)
        for by_out in (False, True):
            dw, db = ops().linear_backward_weight(x, dy, by_out=by_out)
            ref.close("dw", dw, *ref.product(ref.wide(x).T, ref.wide(dy)))
            ref.close("db", db, *ref.column_sums(ref.wide(dy), 0.0))


@pytest.mark.parametrize("stride", [2200000, 4200000, 4300000])
def test_linear_fp32_weight_of_rows_far_apart(stride):
    """Rows of a weight 2^23 bytes and more apart: 256 of them span more than a copy reaches from a tile's start,
    beyond 4.2 million elements 128 do too."""
    rows, k, n = 16384, 64, 512
    wide = torch.empty(n, stride, device="cuda")
    w = wide[:, 8:8 + k]
    w.copy_(normal(1, n, k, std=0.1, kind=F32))
    x, s = normal(2, rows, k, kind=F32), normal(3, rows, n, mean=0.5, kind=F32)
    W = ref.wide(w)
    want, e = ref.product(ref.wide(x), W.T)
    ref.close("y", ops().linear_forward(x, w.t())[0], want, e)              # stored [out, in]
    ref.close("dx", ops().linear_backward_input(x, w), want, e)             # stored [in, out]
    ref.close("dx", ops().linear_backward_input(x, w, derivative=s), want * ref.wide(s),
              (e + ref.U * np.abs(want)) * np.abs(ref.wide(s)))
    # reduced over the rows far apart
    want, e = ref.product(ref.wide(s), W)
    ref.close("y", ops().linear_forward(s, w)[0], want, e)
    ref.close("dx", ops().linear_backward_input(s, w.t()), want, e)


# -- gradients against differences, together, streams and graphs -----------------------


def test_gradients_against_differences():
    """The library's gradients against differences of the 64-bit forms.

    Central differences of step h along v: off by h^2 / 6 of the third derivative (here below 1e3
    of the inputs' size, h = 1e-4: 2e-6 relative) and by 2^-52 / h of the sums (3e-12)."""
    rows, cols, p, h = 6, 40, 0.3, 1e-4
    x, r = normal(1, rows, cols, kind=F32), normal(2, rows, cols, kind=F32)
    ib, w, b = normal(3, cols, kind=F32), normal(4, cols, kind=F32), normal(5, cols, kind=F32)
    cy, ct = normal(6, rows, cols, kind=F32), normal(7, rows, cols, kind=F32)
    drop, d = ops().Dropout(p, SEED, OFFSET), ref.factor(rows, cols, p, SEED, OFFSET)
    _, total, stats = ops().layer_norm_forward(x, w, b, in_bias=ib, drop=drop, residual=r)
    g = ops().layer_norm_backward(cy, total, stats, w, dtotal=ct, drop=drop, in_bias_grad=True)

    def loss(x, r, ib, w, b):
        t = r + (x + ib) * d
        return (ref.Norm(t, 1e-5, w, b).y * ref.wide(cy)).sum() + (t * ref.wide(ct)).sum()

    at = [ref.wide(t) for t in (x, r, ib, w, b)]
    for k, grad in enumerate((g.dx, g.dtotal, g.din_bias, g.dweight, g.dbias)):
        v = np.random.default_rng(k).standard_normal(at[k].shape)
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + h * v, at[k] - h * v
        slope = (loss(*up) - loss(*down)) / (2 * h)
        got = (ref.wide(grad) * v).sum()
        size = np.abs(ref.wide(grad) * v).sum()
        assert abs(got - slope) <= (1e-5 + 200 * ref.U) * size, (k, got, slope)

    i, o = 24, 16
    for act in ("gelu", "silu"):
        a, wt, bias = normal(8, rows, i, kind=F32), normal(9, i, o, std=0.3, kind=F32), normal(10, o, kind=F32)
        dy = normal(11, rows, o, kind=F32)
        _, slope_ = ops().linear_forward(a, wt, bias, activation=act)
        du, db = ops().dropout_backward(dy, ops().Dropout(0.0, 0), derivative=slope_, bias_grad=True)
        dx = ops().linear_backward_input(du, wt)
        dw, db2 = ops().linear_backward_weight(a, du)
        at = [ref.wide(t) for t in (a, wt, bias)]

        def loss(a, wt, bias):
            return (ref.act(act, a @ wt + bias)[0] * ref.wide(dy)).sum()

        for k, grad in enumerate((dx, dw, db)):
            v = np.random.default_rng(k).standard_normal(at[k].shape)
            up, down = list(at), list(at)
            up[k], down[k] = at[k] + h * v, at[k] - h * v
            slope = (loss(*up) - loss(*down)) / (2 * h)
            got, size = (ref.wide(grad) * v).sum(), np.abs(ref.wide(grad) * v).sum()
            assert abs(got - slope) <= (1e-5 + 200 * ref.U) * size, (act, k, got, slope)
        ref.close("db", db2, ref.wide(db), 2 * (rows + 2) * ref.U * np.abs(ref.wide(du)).sum(0))


def sublayer(t, drop, act="gelu"):
    """A pre-LN layer's feed-forward half and its backward pass: norm of a residual sum, two products
    with an activation and a dropout between them, dropout and residual behind."""
    o = ops()
    y, total, stats = o.layer_norm_forward(t["x"], t["g"], t["b"], in_bias=t["ib"], drop=drop(0), residual=t["r"])
    a, slope = o.linear_forward(y, t["w1"], t["b1"], activation=act)
    a2 = o.dropout_forward(a, drop(1))
    z, _ = o.linear_forward(a2, t["w2"])
    out = o.dropout_forward(z, drop(2), bias=t["b2"], residual=total)
    dz, db2 = o.dropout_backward(t["dy"], drop(2), bias_grad=True)
    da2 = o.linear_backward_input(dz, t["w2"])
    du, db1 = o.dropout_backward(da2, drop(1), derivative=slope, bias_grad=True)
    dn = o.linear_backward_input(du, t["w1"])
    g = o.layer_norm_backward(dn, total, stats, t["g"], dtotal=t["dy"], drop=drop(0), in_bias_grad=True)
    dw2, _ = o.linear_backward_weight(a2, dz, bias_grad=False)
    dw1, db1b = o.linear_backward_weight(y, du)
    return dict(out=out, dx=g.dx, dr=g.dtotal, dg=g.dweight, db=g.dbias, dib=g.din_bias, dw1=dw1, dw2=dw2, db1=db1,
                db1b=db1b, db2=db2)


def sublayer_inputs(rows, h, f, kind, seed=20):
    return dict(x=normal(seed, rows, h, kind=kind), r=normal(seed + 1, rows, h, kind=kind),
                dy=normal(seed + 2, rows, h, std=0.1, kind=kind), g=normal(seed + 3, h, std=0.2, mean=1.0, kind=F32),
                b=normal(seed + 4, h, std=0.2, kind=F32), ib=normal(seed + 5, h, std=0.2, kind=F32),
                w1=normal(seed + 6, h, f, std=h ** -0.5, kind=kind), b1=normal(seed + 7, f, std=0.2, kind=F32),
                w2=normal(seed + 8, f, h, std=f ** -0.5, kind=kind), b2=normal(seed + 9, h, std=0.2, kind=F32))


@KINDS
def test_a_layer_s_feed_forward_half(kind):
    """All of them together against autograd of the formulas in 64 bits.  In bf16 ten roundings of half
    a step follow each other at most, each 2^-8 of what is rounded and independent of the others: the
    norms' distance stays below 10 * 2^-8."""
    rows, h, f, p = 150, 136, 520, 0.2
    t = sublayer_inputs(rows, h, f, kind)
    got = sublayer(t, lambda k: ops().Dropout(p, SEED, OFFSET + k))
    v = {k: x.double().cpu().requires_grad_(k != "dy") for k, x in t.items()}
    d = [torch.tensor(ref.factor(rows, n, p, SEED, OFFSET + k)) for k, n in enumerate((h, f, h))]
    total = v["r"] + (v["x"] + v["ib"]) * d[0]
    n = torch.nn.functional.layer_norm(total, (h,), v["g"], v["b"], 1e-5)
    a = torch.nn.functional.gelu(n @ v["w1"] + v["b1"], approximate="tanh") * d[1]
    out = total + (a @ v["w2"] + v["b2"]) * d[2]
    out.backward(v["dy"])
    want = dict(out=out.detach(), dx=v["x"].grad, dr=v["r"].grad, dg=v["g"].grad, db=v["b"].grad, dib=v["ib"].grad,
                dw1=v["w1"].grad, dw2=v["w2"].grad, db1=v["b1"].grad, db1b=v["b1"].grad, db2=v["b2"].grad)
    tol = 10 * 2.0 ** -8 if kind is BF16 else 1e-5
    for k, x in want.items():
        off = ((got[k].double().cpu() - x).norm() / x.norm()).item()
        assert off <= tol, (k, off)


@KINDS
def test_results_repeat_and_streams(kind):
    t = sublayer_inputs(300, 136, 264, kind)
    make = lambda k: ops().Dropout(0.2, SEED, OFFSET + k)  # noqa: E731
    first = sublayer(t, make)
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    results = []
    for s in side:   # two at once, each on a stream of its own
        with torch.cuda.stream(s):
            results.append(sublayer(t, make))
    torch.cuda.synchronize()
    for got in results:
        for k in first:
            assert torch.equal(got[k], first[k]), k


@KINDS
def test_captured_and_replayed(kind):
    """A graph of all of them, whose masks follow a number on the device; eager work between replays."""
    t = sublayer_inputs(200, 136, 264, kind)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    make = lambda k: ops().Dropout(0.2, SEED, k, step=step)  # noqa: E731
    sublayer(t, make)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(sublayer(t, make))
        graphs.append(g)
    for n in (3, 30, 300, 3):
        step.fill_(n)
        t["x"].copy_(normal(n, 200, 136, kind=kind))
        for g, out in zip(graphs, outs):
            g.replay()
            torch.cuda.synchronize()
            eager = sublayer(t, lambda k: ops().Dropout(0.2, SEED, k + n))
            for k in eager:
                assert torch.equal(out[k], eager[k]), (n, k)


def test_linear_feeds_the_attention_operator():
    """QKV product, attention, output product: what stands around the attention in a layer."""
    b, s, h, n = 2, 70, 128, 2
    x = normal(1, b, s, h)
    w, wo = normal(2, h, 3 * h, std=h ** -0.5), normal(3, h, h, std=h ** -0.5)
    qkv, _ = ops().linear_forward(x, w)
    q, k, v = (t.unflatten(-1, (n, h // n)) for t in qkv.split(h, -1))
    o, saved = ops().attention_forward(q, k, v)
    y, _ = ops().linear_forward(o.flatten(2), wo, residual=x)
    want = x.double().cpu()
    Q = (x.double().cpu() @ w.double().cpu()).unflatten(-1, (3, n, h // n))
    sc = torch.einsum("bihd,bjhd->bhij", Q[:, :, 0], Q[:, :, 1]) / (h // n) ** 0.5
    sc = sc.masked_fill(torch.triu(torch.ones(s, s, dtype=torch.bool), 1), float("-inf"))
    want = want + torch.einsum("bhij,bjhd->bihd", sc.softmax(-1), Q[:, :, 2]).flatten(2) @ wo.double().cpu()
    assert ((y.double().cpu() - want).norm() / want.norm()).item() <= 4 * 2.0 ** -8   # four roundings in a row
    do = ops().linear_backward_input(normal(4, b, s, h, std=0.1), wo).unflatten(-1, (n, h // n))
    dq, dk, dv, _ = ops().attention_backward(do, q, k, v, o, saved)
    dqkv = torch.cat([t.flatten(2) for t in (dq, dk, dv)], -1)
    assert ops().linear_backward_weight(x, dqkv)[0].shape == (h, 3 * h)


def test_refusals_of_device_tensors():
    o, x, w = ops(), normal(1, 6, 64), normal(2, 64, 32)
    drop, v = ops().Dropout(0.1, 1), normal(3, 64, kind=F32)
    need = x.clone().requires_grad_()
    for call in (lambda: o.dropout_forward(need, drop), lambda: o.layer_norm_forward(need),
                 lambda: o.linear_forward(need, w), lambda: o.linear_forward(x, w.clone().requires_grad_())):
        with pytest.raises(RuntimeError, match="requires gradients"):
            call()
        with torch.no_grad():
            call()
    bad = [
        lambda: o.dropout_forward(x.half(), drop), lambda: o.dropout_forward(x.t(), drop),
        lambda: o.dropout_forward(x, None), lambda: o.dropout_forward(x, drop, residual=x.float()),
        lambda: o.dropout_forward(x, drop, residual=x[:3]), lambda: o.dropout_forward(x, drop, bias=v[:8]),
        lambda: o.dropout_forward(x, drop, out=x), lambda: o.dropout_forward(x, drop, bias=v.double()),
        lambda: o.dropout_backward(x, drop, bias_grad=True, accumulate=True),
        lambda: o.dropout_backward(x, drop, bias_grad=v.to(BF16)), lambda: o.dropout_backward(x, drop, bias_grad=v[:9]),
        lambda: o.layer_norm_forward(x, v, v.to(BF16)), lambda: o.layer_norm_forward(x, total=x.clone()),
        lambda: o.layer_norm_backward(x, x, torch.zeros(2, 5, device="cuda")),
        lambda: o.layer_norm_backward(x, x, torch.zeros(2, 6, device="cuda"), input_grad=False, weight_grad=False,
                                      bias_grad=False),
        lambda: o.linear_forward(x, w, activation="tanh"), lambda: o.linear_forward(x, w.float()),
        lambda: o.linear_forward(x, w[:60]), lambda: o.linear_forward(x, w[::2, ::2]),
        lambda: o.linear_forward(x[:, :60], w[:60]), lambda: o.linear_forward(x, w, out=x),
        lambda: o.linear_forward(x[:1].expand(6, 64), w), lambda: o.linear_forward(x, w, residual=x), lambda: o.linear_backward_input(x, w),
        lambda: o.linear_backward_weight(x, x[:3]), lambda: o.linear_backward_weight(x, x, weight_grad=False),
        lambda: o.linear_backward_weight(x, x, accumulate=True),
        lambda: o.linear_backward_weight(x, x, by_out=True, weight_grad=3),
        lambda: o.linear_backward_weight(x, x, by_out=True, weight_grad=v),
        lambda: o.linear_backward_weight(x, x, weight_grad=torch.zeros(64, 32, device="cuda")),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError, ops().RcError)):
            call()
            raise AssertionError(f"case {i} was taken")


def test_no_tangent_or_second_derivative_is_lost():
    """Every call refuses tangents, and the backward calls a pass with create_graph; outside of one they take
    tensors that require gradients, as a deferred weight gradient's."""
    import torch.autograd.forward_ad as dual
    o, x, w, g = ops(), normal(1, 6, 64), normal(2, 64, 64), normal(3, 64, kind=F32)
    drop = ops().Dropout(0.1, 1)
    _, total, stats = o.layer_norm_forward(x, g)
    q = normal(4, 1, 8, 2, 32)
    att, saved = o.attention_forward(q, q, q)
    bare = torch.ones(6, 64, dtype=BF16, device="cuda")
    calls = {   # of an input and of a parameter or stored tensor
        "dropout_backward": [lambda t: o.dropout_backward(t, drop), lambda t: o.dropout_backward(bare, drop, derivative=t)],
        "layer_norm_backward": [lambda t: o.layer_norm_backward(t, total, stats, g),
                                lambda t: o.layer_norm_backward(bare, t, stats, g),
                                lambda t: o.layer_norm_backward(bare, total, stats, g, dtotal=t)],
        "linear_backward_input": [lambda t: o.linear_backward_input(t, w),
                                  lambda t: o.linear_backward_input(bare, w, derivative=t)],
        "linear_backward_weight": [lambda t: o.linear_backward_weight(t, bare), lambda t: o.linear_backward_weight(bare, t)],
    }
    forward = [lambda t: o.dropout_forward(t, drop), lambda t: o.dropout_forward(bare, drop, residual=t),
               lambda t: o.layer_norm_forward(t, g), lambda t: o.layer_norm_forward(bare, residual=t),
               lambda t: o.linear_forward(t, w), lambda t: o.linear_forward(bare, w, residual=t)]
    backward = [c for v in calls.values() for c in v]
    with torch.no_grad(), dual.dual_level():
        t = dual.make_dual(x, x)
        for i, call in enumerate(forward + backward):
            with pytest.raises(RuntimeError, match="tangent"):
                call(t)
                raise AssertionError(f"case {i} was taken")
            call(x)
        t = dual.make_dual(q, q)
        for call in (lambda: o.attention_forward(q, t, q), lambda: o.attention_backward(q, q, t, q, att, saved)):
            with pytest.raises(RuntimeError, match="tangent"):
                call()

    class Through(torch.autograd.Function):
        """y = 2 x, whose backward runs a call of x's on the way."""

        @staticmethod
        def forward(ctx, x, call):
            ctx.save_for_backward(x)
            ctx.call = call
            return 2 * x

        @staticmethod
        def backward(ctx, g):
            ctx.call(ctx.saved_tensors[0])
            return 2 * g, None

    leaf, lq = x.clone().requires_grad_(), q.clone().requires_grad_()
    some = [(leaf, c) for c in backward] + [(lq, lambda t: o.attention_backward(q, t, q, q, att, saved))]
    for i, (t, call) in enumerate(some):
        call(t)
        torch.autograd.grad(Through.apply(t, call).sum(), t)
        with pytest.raises(RuntimeError, match="create_graph"):
            torch.autograd.grad(Through.apply(t, call).sum(), t, create_graph=True)
            raise AssertionError(f"case {i} was taken")
