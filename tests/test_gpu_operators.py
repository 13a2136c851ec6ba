"""The operators on the caller's tensors against their plain 64-bit forms, at
the sizes, masks and layouts where they can go wrong."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import operators_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


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


def inputs(b, s, h, kv, d, kind=BF16, seed=1):
    return dict(q=normal(seed, b, s, h, d, kind=kind), k=normal(seed + 1, b, s, kv, d, kind=kind),
                v=normal(seed + 2, b, s, kv, d, mean=0.3, kind=kind)), normal(seed + 3, b, s, h, d, std=0.1, kind=kind)


def run(t, do, **how):
    o, saved = ops().attention_forward(t["q"], t["k"], t["v"], **how)
    dq, dk, dv, dbias = ops().attention_backward(do, t["q"], t["k"], t["v"], o, saved, **how)
    got = dict(o=o, dq=dq, dk=dk, dv=dv)
    if dbias is not None:
        got["dbias"] = dbias
    return got


def compare(t, do, got, **how):
    bias = how.pop("rel_bias", None)
    out, mag = ref.attention(t["q"], t["k"], t["v"], do, bias=bias, **how)
    return ref.check_attention(got, out, mag, t["q"].dtype, None if bias is None else bias.dtype)


# b, s, heads, kv heads, d, causal, window, sinks, buckets, max_distance, lengths
CASES = [
    (1, 1, 1, 1, 8, True, 0, 0, 0, 0, None),             # one token
    (2, 1, 3, 1, 64, False, 1, 1, 8, 16, None),
    (1, 2, 2, 2, 128, True, 1, 0, 0, 0, None),           # every token sees itself only
    (1, 63, 4, 4, 32, True, 7, 0, 0, 0, None),
    (1, 64, 2, 1, 128, True, 64, 3, 0, 0, None),
    (2, 65, 4, 2, 64, True, 17, 4, 0, 0, None),
    (1, 129, 2, 2, 128, True, 64, 0, 0, 0, None),
    (1, 200, 2, 2, 96, False, 33, 5, 0, 0, None),
    (2, 257, 6, 2, 80, True, 100, 70, 0, 0, None),       # sinks beyond one block of 64
    (1, 700, 2, 1, 64, True, 40, 130, 0, 0, None),       # and of 128
    (1, 1100, 2, 2, 128, True, 65, 4, 0, 0, None),       # sinks' gradients in chunks
    (1, 1300, 2, 2, 40, False, 31, 200, 0, 0, None),     # bidirectional sinks on both sides
    (1, 130, 2, 2, 128, True, 1000, 8, 0, 0, None),      # a window wider than the sequence
    (1, 96, 2, 2, 16, True, 0, 9, 0, 0, None),           # sinks without a window
    (3, 150, 2, 2, 64, False, 20, 3, 0, 0, (150, 0, 77)),  # an empty sequence
    (4, 140, 4, 4, 128, True, 30, 2, 0, 0, (1, 140, 64, 128)),
    (2, 90, 2, 2, 104, False, 0, 0, 0, 0, (-5, 1000)),   # lengths beyond their range
    (1, 33, 2, 2, 64, True, 0, 0, 2, 2, None),           # the fewest buckets
    (1, 150, 2, 2, 64, False, 0, 0, 4, 2, None),
    (1, 300, 3, 3, 64, True, 0, 0, 32, 128, None),
    (2, 333, 4, 2, 128, False, 0, 0, 32, 128, None),
    (1, 400, 2, 2, 32, False, 0, 0, 128, 1024, None),    # the most, none of them far
    (1, 1400, 2, 1, 128, True, 0, 0, 128, 1024, None),
    (2, 260, 2, 1, 96, True, 90, 5, 16, 40, None),       # bias, window and sinks
    (3, 280, 2, 2, 128, False, 70, 6, 32, 100, (280, 31, 0)),
    (1, 900, 2, 2, 64, True, 50, 10, 64, 512, (777,)),
]


# The same on grids of more than 256 blocks of 32 tokens, which take 128 tokens a workgroup.
CASES += [
    (300, 1, 1, 1, 64, True, 0, 0, 0, 0, None),
    (5, 300, 12, 12, 128, True, 70, 4, 0, 0, None),
    (2, 700, 12, 12, 64, True, 40, 130, 0, 0, None),
    (1, 1100, 12, 2, 128, True, 65, 4, 0, 0, None),
    (1, 1300, 9, 9, 40, False, 31, 200, 0, 0, None),
    (6, 260, 8, 8, 96, False, 33, 5, 0, 0, (260, 0, 129, 128, 1, 200)),
    (2, 257, 18, 6, 80, True, 100, 70, 0, 0, None),
    (4, 300, 9, 9, 64, True, 0, 0, 32, 128, (300, 299, 17, 0)),
    (2, 333, 16, 8, 128, False, 0, 0, 32, 128, None),
    (1, 600, 20, 10, 32, False, 0, 0, 128, 1024, None),
    (1, 1400, 8, 2, 128, True, 90, 33, 128, 1024, None),
    (3, 280, 14, 2, 128, False, 70, 6, 32, 100, (280, 31, 0)),
    (1, 2100, 6, 6, 64, True, 50, 10, 64, 512, (1777,)),
    (1, 2200, 1, 1, 16, True, 50, 10, 0, 0, None),   # a small grid, but a long sequence: the sinks' own workgroups
    (1, 2200, 2, 1, 128, False, 50, 40, 8, 20, None),
]


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:10]))
def test_attention(case, kind):
    b, s, h, kv, d, causal, window, sinks, buckets, far, lengths = case
    t, do = inputs(b, s, h, kv, d, kind)
    how = dict(causal=causal, window=window, sinks=sinks, max_distance=far)
    if buckets:
        how["rel_bias"] = normal(9, h, buckets, kind=kind)
    if lengths is not None:
        how["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    compare(t, do, run(t, do, **how), **how)


# Few workgroups of dk and dv, and many heads for each of them: taken in parts.
PARTS = [
    (1, 1100, 8, 1, 40, True, 0, 0, 16, 100, None),       # blocks of 32 keys; 7 parts of 8 heads
    (2, 530, 6, 2, 128, False, 0, 0, 0, 0, (530, 301)),
    (1, 700, 6, 2, 24, True, 100, 40, 8, 30, None),       # with the sinks' own workgroups
    (1, 400, 12, 2, 64, True, 90, 7, 0, 0, (333,)),       # and without
    (6, 1500, 3, 1, 48, True, 300, 40, 8, 20, (1500, 0, 1400, 77, 1, 1000)),   # blocks of 128 keys
    (6, 1500, 3, 1, 72, False, 0, 0, 0, 0, None),
]


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", PARTS, ids=lambda c: "-".join(str(x) for x in c[:10]))
def test_heads_in_parts(case, kind):
    test_attention(case, kind)


# -- layouts, streams, graphs ----------------------------------------------------

MASKED = dict(causal=False, window=40, sinks=3, max_distance=50)


def masked(seed=1, b=2, s=170, h=4, kv=2, d=64, kind=BF16):
    t, do = inputs(b, s, h, kv, d, kind, seed)
    how = dict(MASKED, rel_bias=normal(seed + 9, h, 16, kind=kind),
               lengths=torch.tensor([s - 20 * i for i in range(b)], dtype=torch.int32, device="cuda"))
    return t, do, how


def test_strided_views():
    """Heads as columns of one packed matrix, sequences inside heads, and gradients into such views."""
    b, s, h, d = 2, 170, 4, 64
    packed = normal(1, b, s, 3 * h * d)
    q, k, v = (x.view(b, s, h, d) for x in packed.split(h * d, 2))
    do = normal(4, b, h, s, d, std=0.1).transpose(1, 2)
    t, how = dict(q=q, k=k, v=v), dict(MASKED, rel_bias=normal(9, h, 16))
    grads = torch.full((b, s, 3 * h * d), math.nan, dtype=BF16, device="cuda")
    dq, dk, dv = (x.view(b, s, h, d) for x in grads.split(h * d, 2))
    o = torch.full((s, h, b, d + 8), math.nan, dtype=BF16, device="cuda")
    ov = o[..., :d].permute(2, 0, 1, 3)
    got_o, saved = ops().attention_forward(q, k, v, out=ov, **how)
    assert got_o is ov
    got = ops().attention_backward(do, q, k, v, ov, saved, dq=dq, dk=dk, dv=dv, **how)
    assert got[0] is dq and got[1] is dk and got[2] is dv
    compare(t, do, dict(o=ov, dq=dq, dk=dk, dv=dv, dbias=got[3]), **how)
    assert bool(o[..., d:].isnan().all()), "columns beyond the heads were written"


def test_broadcast_inputs():
    """Inputs that repeat a sequence or a head (stride 0) get a gradient for each use."""
    b, s, h, d = 3, 100, 4, 32
    one = normal(1, 1, s, 1, d)
    t = dict(q=normal(2, b, s, h, d), k=one.expand(b, s, 2, d), v=one.expand(b, s, 2, d))
    do = normal(3, 1, s, 1, d, std=0.1).expand(b, s, h, d)
    compare(t, do, run(t, do, window=30), window=30)


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
def test_results_are_reproducible(kind):
    t, do, how = masked(kind=kind, s=700, b=1)
    first = run(t, do, **how)
    for _ in range(3):
        again = run(t, do, **how)
        assert all(torch.equal(first[n], again[n]) for n in first)


def test_forward_without_saved_is_the_same():
    t, do, how = masked()
    a = ops().attention_forward(t["q"], t["k"], t["v"], **how)[0]
    b, saved = ops().attention_forward(t["q"], t["k"], t["v"], save=False, **how)
    assert saved is None and torch.equal(a, b)


def test_on_another_stream():
    t, do, how = masked()
    want = run(t, do, **how)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(t, do, **how)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(want[n], got[n]) for n in want)


def test_two_captured_graphs():
    """Two graphs captured and replayed in turn, with new inputs and eager work between the replays."""
    calls = [masked(seed=1), masked(seed=30, s=260)]
    graphs, outs = [], []
    for t, do, how in calls:
        run(t, do, **how)
    torch.cuda.synchronize()
    for t, do, how in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(t, do, **how))
        graphs.append(g)
    for turn in range(3):
        for t, do, _ in calls:
            for n, x in enumerate((t["q"], t["k"], t["v"], do)):
                x.copy_(normal(100 * turn + n, *x.shape))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (t, do, how), out in zip(calls, outs):
            want = run(t, do, **how)
            assert all(torch.equal(want[n], out[n]) for n in want), turn


# -- values ------------------------------------------------------------------------


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
def test_padding_is_not_read(kind):
    """NaN and infinities behind a sequence's length reach nothing."""
    t, do, how = masked(kind=kind, b=3)
    want = run(t, do, **how)
    for i, n in enumerate(how["lengths"].tolist()):
        for x, bad in zip((t["q"], t["k"], t["v"], do), (math.nan, math.inf, -math.inf, math.nan)):
            x[i, n:] = bad
    got = run(t, do, **how)
    assert all(torch.equal(want[n], got[n]) for n in want)
    for i, n in enumerate(how["lengths"].tolist()):
        assert all(float(got[x][i, n:].abs().sum()) == 0.0 for x in ("o", "dq", "dk", "dv"))


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
def test_one_visible_token(kind):
    """Where a token sees itself alone, o is its value and no gradient reaches the scores."""
    t, do = inputs(2, 150, 4, 2, 64, kind)
    got = run(t, do, window=1, rel_bias=normal(9, 4, 8, kind=kind), max_distance=16)
    assert torch.equal(got["o"], t["v"].repeat_interleave(2, 2))
    for n in ("dq", "dk", "dbias"):
        assert float(got[n].abs().max()) == 0.0, n


# b, s, heads, kv heads, d, causal, window, lengths
ALONE = [
    (2, 150, 4, 2, 64, True, 1, None),
    (1, 130, 3, 3, 128, False, 1, None),
    (3, 1, 4, 1, 16, True, 0, None),
    (1, 1, 2, 2, 80, False, 0, None),
    (3, 70, 2, 2, 96, False, 0, (1, 0, 1)),              # one token in a padded sequence
    (1, 500, 32, 1, 40, True, 1, None),                  # the heads of dk and dv in parts
    (300, 1, 1, 1, 64, False, 0, None),                  # grids of more than 256 blocks of 32 tokens
    (5, 300, 12, 6, 128, True, 1, (300, 299, 1, 0, 40)),
    (3, 700, 16, 16, 80, False, 1, None),
]


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", ALONE, ids=lambda c: "-".join(str(x) for x in c[:7]))
def test_one_visible_token_without_a_bias(case, kind):
    """The probability is one whatever the score: o is the value, and no gradient reaches the scores."""
    b, s, h, kv, d, causal, window, lengths = case
    t, do = inputs(b, s, h, kv, d, kind)
    how = dict(causal=causal, window=window)
    n = torch.tensor([s] * b if lengths is None else lengths, dtype=torch.int32, device="cuda")
    if lengths is not None:
        how["lengths"] = n
    got = run(t, do, **how)
    real = (torch.arange(s, device="cuda") < n[:, None])[:, :, None, None]
    assert torch.equal(got["o"], torch.where(real, t["v"].repeat_interleave(h // kv, 2), 0.0).to(kind))
    for x in ("dq", "dk"):
        assert int(torch.count_nonzero(got[x])) == 0, (x, float(got[x].abs().max()))


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("b,s,h,kv,d", [(2, 100, 4, 2, 64), (2, 700, 12, 12, 128)])
def test_the_first_token_of_a_causal_sequence(b, s, h, kv, d, kind):
    """The one row that sees a single token, next to rows that see more."""
    t, do = inputs(b, s, h, kv, d, kind)
    got = run(t, do)
    assert torch.equal(got["o"][:, 0], t["v"][:, 0].repeat_interleave(h // kv, 1))
    assert int(torch.count_nonzero(got["dq"][:, 0])) == 0
    assert int(torch.count_nonzero(got["dq"][:, 1])) > 0


@pytest.mark.parametrize("low", [-math.inf, "lowest"])
@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
def test_bias_that_hides(kind, low):
    """A bias of -inf hides its bucket, and a row of such is empty; with the type's
    lowest value a row of such is uniform instead, and a bucket among others hidden."""
    t, do = inputs(1, 200, 2, 2, 64, kind)
    low = torch.finfo(kind).min if low == "lowest" else low
    bias = normal(9, 2, 8, kind=kind)
    bias[0, 2:] = low
    bias[1] = low
    how = dict(rel_bias=bias, max_distance=16)
    got = run(t, do, **how)
    plain = bias.cpu().double()
    out, mag = ref.attention(t["q"], t["k"], t["v"], do, bias=torch.where(plain < -1e38, -math.inf, plain), max_distance=16)
    if math.isfinite(low):  # head 1: the mean over the tokens up to i, whatever the scores
        flat, fmag = ref.attention(t["q"] * 0, t["k"] * 0, t["v"], do, causal=True)
        for n in ("o", "dv"):
            out[n][:, :, 1] = flat[n][:, :, 1]
            mag[n] = tuple(torch.cat((a[:, :, :1], b[:, :, 1:]), 2) for a, b in zip(mag[n], fmag[n]))
        got = {n: got[n] for n in ("o", "dv")}
        out = {n: out[n] for n in ("o", "dv")}
    ref.check_attention(got, out, mag, kind, kind)


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
def test_large_scores(kind):
    """Scores of several thousand: probabilities of nearly one token a row."""
    t, do = inputs(1, 200, 2, 2, 64, kind)
    t["q"], t["k"] = t["q"] * 8, t["k"] * 8
    how = dict(window=60, sinks=2, rel_bias=normal(9, 2, 8, std=30.0, kind=kind), max_distance=16)
    compare(t, do, run(t, do, **how), **how)


@pytest.mark.parametrize("s,buckets", [(1300, 8), (64, 16)])
def test_bias_gradient_of_bf16_tensors_in_32_bits(s, buckets):
    """A bias and its gradient in fp32 next to bf16 tensors (a stage's): the far bucket holds
    most of a long row, and what D is off by sums up there.  D = do.o is formed from
    probabilities and outputs of two bf16 numbers each, so no value that was rounded to bf16
    once enters: the error stays below half of one such rounding, 2^-10 (with
    probabilities of one bf16 number it was 4e-3)."""
    t, do = inputs(1, s, 2, 2, 64)
    how = dict(causal=False, rel_bias=normal(9, 2, buckets, kind=F32), max_distance=128)
    got = run(t, do, **how)
    out, mag = ref.attention(t["q"], t["k"], t["v"], do, causal=False, bias=how["rel_bias"], max_distance=128)
    worst = ref.check_attention({"dbias": got["dbias"]}, {"dbias": out["dbias"]}, mag, BF16, F32, fine=True)
    rel = float((got["dbias"].cpu().double() - out["dbias"]).norm() / out["dbias"].norm())
    print(f"[bias gradient] s {s}: rel-L2 {rel:.1e}, share of the bound {worst}")
    assert rel < 2.0 ** -10


def test_gradients_against_differences():
    """dq, dk, dv and dbias of a small fp32 call against central differences of
    the 64-bit operator.  A difference of step e = 2^-10 is off by e^2 / 6 of a
    third derivative, under 2^-20 * 2^6 of the gradient's size here."""
    t, do = inputs(1, 20, 2, 1, 8, F32)
    bias = normal(9, 2, 8, kind=F32)
    how = dict(causal=False, window=6, sinks=1, max_distance=6, rel_bias=bias)
    got = run(t, do, **how)
    wide = {n: x.cpu().double() for n, x in (("q", t["q"]), ("k", t["k"]), ("v", t["v"]), ("rel_bias", bias))}
    dod, e = do.cpu().double(), 2.0 ** -10

    def total(x):
        o, _ = ref.attention(x["q"], x["k"], x["v"], bias=x["rel_bias"], causal=False, window=6, sinks=1, max_distance=6)
        return float((o["o"] * dod).sum())

    rng = np.random.RandomState(0)
    for n, g in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("rel_bias", "dbias")):
        size = float(got[g].abs().max())
        for at in rng.permutation(wide[n].numel())[:12]:
            flat = wide[n].view(-1)
            was = float(flat[at])
            flat[at] = was + e
            up = total(wide)
            flat[at] = was - e
            down = total(wide)
            flat[at] = was
            assert abs((up - down) / (2 * e) - float(got[g].view(-1)[at])) < 2.0 ** -14 * size + 2.0 ** -20, (n, at)


# -- AdamW ----------------------------------------------------------------------------


def adamw_set(sizes, bits, grad_kind, seed=1, offset=0):
    """Tensors of the given sizes, each `offset` elements into an allocation of its own."""
    rng = np.random.RandomState(seed)
    make = lambda x, kind: torch.cat((torch.zeros(offset), torch.from_numpy(x).float())).to(kind).cuda()[offset:]  # noqa: E731
    p = [make(rng.randn(n) * 0.02, F32) for n in sizes]
    g = [make(rng.randn(n) * np.exp(rng.randn()) * 1e-3, grad_kind) for n in sizes]
    return p, g


def check_adamw(opt, before, grads, scale, step, **hyper):
    """Each tensor's p, m and v after a step against the 64-bit step from its state before.
    fp32: m and v take three half-steps; p a few of p and of the update.  8 bits: the codes
    are those of the 64-bit step."""
    half = 2.0 ** -24
    for i, (p0, m0, v0) in enumerate(before):
        p, m, v = ref.adamw(p0, grads[i], m0, v0, step=step, decay=opt.decay[i], grad_scale=scale, **hyper)
        got = opt.params[i].cpu().double().numpy()
        bound = 4 * half * np.abs(p) + 16 * half * np.abs(p - p0) + 1e-30
        assert np.all(np.abs(got - p) <= bound), (i, np.max(np.abs(got - p) / bound))
        if opt.copies[i] is not None:
            assert torch.equal(opt.copies[i], opt.params[i].to(BF16)), i
        if opt.state_bits == 32:
            gm, gv = opt.exp_avg[i].cpu().double().numpy(), opt.exp_avg_sq[i].cpu().double().numpy()
            parts = 0.9 * np.abs(m0) + 0.1 * np.abs(grads[i] * scale)
            assert np.all(np.abs(gm - m) <= 4 * half * parts + 1e-38), i
            assert np.all(np.abs(gv - v) <= 5 * half * v + 1e-38), i
        else:
            for code, scales, want in ((opt.exp_avg[i], opt.exp_avg_scale[i], ref.encode_m(m)),
                                       (opt.exp_avg_sq[i], opt.exp_avg_sq_scale[i], ref.encode_v(v))):
                assert np.array_equal(scales.cpu().numpy(), want[1]), i
                c, w = code.cpu().numpy(), want[0]
                zero = (c & 127 == 0) & (w & 127 == 0) if want[0] is not None else False  # either sign of zero
                assert np.all((c == w) | zero), (i, np.flatnonzero((c != w) & ~zero)[:5])


def state(opt):
    got = []
    for i, p in enumerate(opt.params):
        m, v = opt.exp_avg[i].cpu().numpy(), opt.exp_avg_sq[i].cpu().numpy()
        if opt.state_bits == 8:
            m = ref.decode_m(m, opt.exp_avg_scale[i].cpu().numpy())
            v = ref.decode_v(v, opt.exp_avg_sq_scale[i].cpu().numpy())
        got.append((p.cpu().double().numpy(), m.astype(np.float64), v.astype(np.float64)))
    return got


SIZES = [1, 2, 127, 128, 129, 4096, 4097, 1000, 8191, 0, 20000]


@pytest.mark.parametrize("offset", [0, 1], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("grad_kind", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits, grad_kind, offset):
    p, g = adamw_set(SIZES, bits, grad_kind, offset=offset)
    copies = [torch.zeros(n, dtype=BF16, device="cuda") if i % 2 else None for i, n in enumerate(SIZES)]
    opt = ops().AdamW(p, g, state_bits=bits, decay=[i % 3 != 0 for i in range(len(SIZES))], copies=copies)
    rng = np.random.RandomState(7)
    for step in range(1, 4):
        for x in g:
            x.mul_(float(rng.rand()) + 0.5)
        grads = [x.cpu().double().numpy() for x in g]
        before = state(opt)
        opt.step(0.5)
        assert opt.steps == step
        check_adamw(opt, before, grads, 0.5, step)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_more_tensors_than_a_launch_takes(bits):
    sizes = [1 + 31 * i % 300 for i in range(131)]
    p, g = adamw_set(sizes, bits, F32)
    opt = ops().AdamW(p, g, state_bits=bits)
    before, grads = state(opt), [x.cpu().double().numpy() for x in g]
    opt.step()
    check_adamw(opt, before, grads, 1.0, 1)


def test_adamw_8_bit_edges():
    """Moments from 2^-75 to 2^60 in one block, blocks of zeros, of equal values at the
    formats' borders, and values that fp32 does not hold: their own codes are NaN, their
    block's others are as if they were not there."""
    g = np.zeros(128 * 8)
    g[:128] = np.ldexp(1.0, np.linspace(-75, 60, 128).astype(int)) * np.where(np.arange(128) % 2, 1, -1)
    g[256:384] = np.ldexp(1.75, 5)                           # both formats' largest code
    g[384:512] = np.ldexp(1.7500002, 5)                      # just beyond: the next power of two
    g[512:640] = np.random.RandomState(0).randn(128)
    g[520], g[530], g[540] = np.nan, np.inf, -np.inf
    g[640:768] = np.random.RandomState(1).randn(128) * 1e30  # squares beyond fp32
    g[768:896] = np.random.RandomState(2).randn(128) * 1e-30
    p = [torch.zeros(g.size, device="cuda")]
    grads = [torch.from_numpy(g).float().cuda()]
    opt = ops().AdamW(p, grads, state_bits=8, weight_decay=0.0)
    before = state(opt)
    wide = grads[0].cpu().double().numpy()
    opt.step()
    b1, b2 = float(np.float32(0.9)), float(np.float32(0.95))
    with np.errstate(invalid="ignore"):
        m, v = (1 - b1) * wide, (1 - b2) * wide * wide
    for code, scales, want in ((opt.exp_avg[0], opt.exp_avg_scale[0], ref.encode_m(m)),
                               (opt.exp_avg_sq[0], opt.exp_avg_sq_scale[0], ref.encode_v(v))):
        assert np.array_equal(scales.cpu().numpy(), want[1])
        c, w = code.cpu().numpy(), want[0]
        assert np.all((c == w) | ((c & 127 == 0) & (w & 127 == 0)) | ((c & 127 == 127) & (w & 127 == 127))), \
            np.flatnonzero(c != w)
    assert before[0][0].sum() == 0 and bool(torch.isfinite(p[0][:512]).all())
    assert int(opt.exp_avg_sq[0][:128].min()) >= 1, "a second moment above zero lost its code"
    # a second step keeps what is not a number where it was
    opt.step()
    m2, v2 = state(opt)[0][1:]
    assert np.array_equal(np.isnan(m2), ~(np.abs(m) < 3.4e38)) and np.isnan(v2[[520, 530, 540]]).all()


def test_adamw_in_a_graph():
    sizes = [3000, 17, 129]
    p, g = adamw_set(sizes, 8, F32)
    opt = ops().AdamW(p, g, state_bits=8)
    opt.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(0.25, step=2)
    for turn in range(3):
        for x in g:
            x.copy_(normal(turn, *x.shape, std=1e-3, kind=F32))
        before, grads = state(opt), [x.cpu().double().numpy() for x in g]
        graph.replay()
        torch.cuda.synchronize()
        check_adamw(opt, before, grads, 0.25, 2)


def test_adamw_steps_as_the_stage_does():
    """32-bit moments: from the same state, the step of a stage's own optimizer.  Both
    are compiled from one formula, but the compiler may join either product of a sum
    with the addition, so each is held to the bounds of its 32-bit roundings."""
    from paper_2405_14009_amd import RC_READ_ADAM_M, RC_READ_ADAM_V, RC_READ_GRAD, RC_READ_PARAM, Stage, param_shape
    stage = Stage(num_layers=1, hidden=64, heads=2, ffn=128, seq_len=32, micro_batch=1, dtype="f32")
    rng = np.random.RandomState(0)
    stage.load_params([[rng.randn(*param_shape(i, 64, 128)) * 0.1 for i in range(12)]])
    flat = lambda what: [torch.from_numpy(x.ravel()).cuda() for x in stage.read_all(what)[0]]  # noqa: E731
    for step in range(1, 4):
        stage.forward((0, 0), normal(step, 1, 32, 64, kind=F32))
        stage.backward((0, 0), normal(step + 9, 1, 32, 64, kind=F32))
        args = dict(decay=[i in (2, 4, 8, 10) for i in range(12)])
        own = ops().AdamW(flat(RC_READ_PARAM), flat(RC_READ_GRAD), exp_avg=flat(RC_READ_ADAM_M),
                          exp_avg_sq=flat(RC_READ_ADAM_V), **args)
        before, grads = state(own), [x.cpu().double().numpy() for x in own.grads]
        own.step(0.5, step=step)
        check_adamw(own, before, grads, 0.5, step)
        stage.optimizer_step(0.5)
        theirs = ops().AdamW(flat(RC_READ_PARAM), flat(RC_READ_GRAD), exp_avg=flat(RC_READ_ADAM_M),
                             exp_avg_sq=flat(RC_READ_ADAM_V), **args)
        check_adamw(theirs, before, grads, 0.5, step)


@pytest.mark.parametrize("offset", [0, 1], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("bits", [32, 8])
def test_moments_as_values(bits, offset):
    p, g = adamw_set(SIZES, bits, F32, offset=offset)
    opt = ops().AdamW(p, g, state_bits=bits)
    for _ in range(2):
        opt.step()
    m, v = opt.moments()
    for i, (_, wm, wv) in enumerate(state(opt)):
        assert np.array_equal(m[i].cpu().numpy(), wm.astype(np.float32)), i
        assert np.array_equal(v[i].cpu().numpy(), wv.astype(np.float32)), i


def test_refusals_of_the_python_calls():
    """What the wrappers refuse before the library sees it; nothing is enqueued."""
    pkg = ops()
    q, k = torch.zeros(2, 40, 4, 64, device="cuda"), torch.zeros(2, 40, 2, 64, device="cuda")
    o, saved = pkg.attention_forward(q, k, k)
    bias = torch.zeros(4, 16, device="cuda")
    for error, call in (
            (TypeError, lambda: pkg.attention_forward(q.cpu(), k, k)),
            (ValueError, lambda: pkg.attention_forward(q.half(), k.half(), k.half())),
            (ValueError, lambda: pkg.attention_forward(q[0], k, k)),
            (ValueError, lambda: pkg.attention_forward(q, k[:, :39], k)),
            (ValueError, lambda: pkg.attention_forward(q, k, k.bfloat16())),
            (ValueError, lambda: pkg.attention_forward(q, k, k.transpose(2, 3).contiguous().transpose(2, 3))),
            (ValueError, lambda: pkg.attention_forward(q, k, k, rel_bias=bias[:3])),
            (ValueError, lambda: pkg.attention_forward(q, k, k, rel_bias=bias.t())),
            (ValueError, lambda: pkg.attention_forward(q, k, k, rel_bias=bias.half())),
            (ValueError, lambda: pkg.attention_forward(q, k, k, lengths=torch.zeros(2, device="cuda"))),
            (TypeError, lambda: pkg.attention_forward(q, k, k, lengths=torch.zeros(2, dtype=torch.int32))),
            (ValueError, lambda: pkg.attention_forward(q, k, k, out=o[:, :39])),
            (pkg.InvalidArgError, lambda: pkg.attention_forward(q, k, k, out=q)),
            (pkg.InvalidArgError, lambda: pkg.attention_forward(q, k, k, out=o[:, :1].expand(q.shape))),
            (ValueError, lambda: pkg.attention_backward(o, q, k, k, o, saved[:-1])),
            (ValueError, lambda: pkg.attention_backward(o, q, k, k, o, None)),
            (pkg.InvalidArgError, lambda: pkg.attention_backward(o, q, k, k, o, saved, dq=q))):
        with pytest.raises(error):
            call()

    x = torch.zeros(300, device="cuda")
    p, g = x[:100], x[100:200]
    half = torch.zeros(100, dtype=BF16, device="cuda")
    for kw in (dict(params=[p, p], grads=[g, g]), dict(params=[p, x[50:150]], grads=[x[200:], x[200:]]),
               dict(params=[p], grads=[p]), dict(params=[p], grads=[x[99:199]]),
               dict(params=[p], grads=[g], exp_avg=[x[200:]], exp_avg_sq=[x[200:]]),
               dict(params=[p, g], grads=[x[200:], x[200:]], copies=[half, half]),
               dict(params=[p], grads=[g[:99]]), dict(params=[half], grads=[g]), dict(params=[p], grads=[]),
               dict(params=[p], grads=[g], decay=[True, False]), dict(params=[p], grads=[g], state_bits=16),
               dict(params=[p], grads=[g], exp_avg=[x[200:]]),
               dict(params=[p], grads=[g], exp_avg=[x[200:]], exp_avg_sq=[x[200:]], state_bits=8)):
        with pytest.raises(ValueError):
            pkg.AdamW(**kw)
    with pytest.raises(TypeError):
        pkg.AdamW([p.cpu()], [g])
    with pytest.raises(TypeError):
        pkg.AdamW([p], [g.cpu()])
    opt = pkg.AdamW([p, x[200:]], [g, g])          # one gradient for two parameters is read only
    for out in ([[p], [p]], [[p, p[:99]], [p, p]], [[p, half], [p, p]]):
        with pytest.raises(ValueError):
            opt.moments(out)
    assert float(x.abs().sum()) == 0.0


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_follows_its_tensors(bits):
    """Parameters and gradients that have other memory, or are other tensors, than at the
    last step: the step takes the new ones and leaves the old ones alone."""
    sizes = [300, 17, 129]
    p, g = adamw_set(sizes, bits, F32)
    opt = ops().AdamW(p, g, state_bits=bits)
    opt.step()
    old = [x.detach() for x in p] + [x.detach() for x in g]    # the same memory
    kept = [x.clone() for x in old]
    p[0].data = p[0].detach() + 1.0
    g[1].data = g[1].detach() * 2.0
    opt.grads[2] = (g[2] * 3.0).bfloat16()
    opt.exp_avg[1] = opt.exp_avg[1].clone()
    opt.decay[0] = False
    before, grads = state(opt), [x.double().cpu().numpy() for x in opt.grads]
    opt.step(0.5)
    check_adamw(opt, before, grads, 0.5, 2)
    changed = [not torch.equal(a, b) for a, b in zip(old, kept)]
    assert changed == [False, True, True, False, False, False]
    # another tensor between the step and the reading of the moments
    opt.exp_avg[0] = opt.exp_avg[0] * 1
    m, v = opt.moments()
    for i, (_, wm, wv) in enumerate(state(opt)):
        assert np.array_equal(m[i].cpu().numpy(), wm.astype(np.float32)), i
        assert np.array_equal(v[i].cpu().numpy(), wv.astype(np.float32)), i


def test_adamw_refuses_what_its_tensors_became():
    """Tensors that no longer fit are refused by the next step, which changes nothing; put right, it runs."""
    p, g = adamw_set([60, 40], 32, F32)
    opt = ops().AdamW(p, g)
    opt.step()
    kept = [x.clone() for x in p]
    p[0].data, was = p[0].detach()[:50], p[0].detach()
    for _ in range(2):
        with pytest.raises(ValueError):
            opt.step()
    p[0].data = was.view(6, 10).t()
    with pytest.raises(ValueError):
        opt.step()
    p[0].data = was
    for lists, error, entry in ((opt.grads, TypeError, None), (opt.grads, ValueError, g[0]), (opt.params, TypeError, p[1].cpu()),
                                (opt.exp_avg, ValueError, opt.exp_avg[0]), (opt.params, ValueError, p[0]),
                                (opt.copies, ValueError, p[1])):
        right, lists[1] = lists[1], entry
        with pytest.raises(error):
            opt.step()
        lists[1] = right
    opt.params.append(p[0])
    for call in (opt.step, opt.moments):
        with pytest.raises(ValueError):
            call()
    opt.params.pop()
    assert opt.steps == 1 and all(torch.equal(a, b) for a, b in zip(p, kept))
    before, grads = state(opt), [x.cpu().double().numpy() for x in g]
    opt.step()
    check_adamw(opt, before, grads, 1.0, 2)


def test_q_itself_as_another_tensor():
    """q given as k and v is read as such; as v next to fewer key heads it has the wrong shape."""
    q, do = normal(1, 2, 40, 4, 64), normal(2, 2, 40, 4, 64, std=0.1)
    t = dict(q=q, k=q, v=q)
    compare(t, do, run(t, do, window=9), window=9)
    k = normal(3, 2, 40, 2, 64)
    for kv in ((k, q), (q, k)):
        with pytest.raises(ValueError):
            ops().attention_forward(q, *kv)


def test_numbers_that_are_not_whole_or_too_large():
    pkg, q = ops(), normal(1, 1, 40, 2, 32)
    for kw in (dict(window=2.5), dict(window=7, sinks=0.5), dict(window=(1 << 32) + 5), dict(window=5, sinks=1 << 32),
               dict(rel_bias=normal(2, 2, 8), max_distance=(1 << 32) + 64),
               dict(rel_bias=normal(2, 2, 8), max_distance=64.5)):
        with pytest.raises(ValueError):
            pkg.attention_forward(q, q, q, **kw)
    p = torch.zeros(8, device="cuda")
    opt = pkg.AdamW([p], [torch.ones_like(p)])
    for step in (2.5, (1 << 64) + 1, 1 << 63):
        with pytest.raises(ValueError):
            opt.step(step=step)
    assert opt.steps == 0 and float(p.abs().sum()) == 0.0


def test_autograd_is_not_cut_silently():
    """A call that autograd would have to record is refused; with autograd off, and in a
    function of its own that calls the backward, it runs."""
    t, do = inputs(1, 40, 2, 2, 32)
    bias = normal(9, 2, 8)
    how = dict(window=9, max_distance=16)
    want = run(t, do, rel_bias=bias, **how)
    leaves = [x.clone().requires_grad_() for x in (t["q"], t["k"], t["v"], bias)]
    for i in range(4):
        x = [leaf if i == j else leaf.detach() for j, leaf in enumerate(leaves)]
        with pytest.raises(RuntimeError, match="gradients"):
            ops().attention_forward(*x[:3], rel_bias=x[3], **how)
    with pytest.raises(RuntimeError, match="out"):
        ops().attention_forward(t["q"], t["k"], t["v"], out=torch.empty_like(t["q"]).requires_grad_())
    with torch.no_grad():
        o, _ = ops().attention_forward(*leaves[:3], rel_bias=leaves[3], **how)
    assert torch.equal(o, want["o"]) and not o.requires_grad

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, b):
            o, saved = ops().attention_forward(q, k, v, rel_bias=b, **how)
            ctx.save_for_backward(q, k, v, b, o, saved)
            return o

        @staticmethod
        def backward(ctx, g):
            q, k, v, b, o, saved = ctx.saved_tensors
            return ops().attention_backward(g, q, k, v, o, saved, rel_bias=b, **how)

    o = Attention.apply(*leaves)
    got = torch.autograd.grad(o, leaves, do)
    assert torch.equal(o, want["o"])
    assert all(torch.equal(a, want[n]) for a, n in zip(got, ("dq", "dk", "dv", "dbias")))


def test_saved_is_what_the_forward_returned():
    """As many elements of another type, or strided ones, are not those bytes."""
    t, do = inputs(1, 40, 2, 2, 32)
    o, saved = ops().attention_forward(t["q"], t["k"], t["v"])
    wide = torch.empty(2 * saved.numel(), dtype=torch.uint8, device="cuda")
    for bad in (saved.bool(), saved[:1].expand(saved.numel()), wide[::2], saved[:-1], saved.cpu()):
        with pytest.raises(ValueError):
            ops().attention_backward(do, t["q"], t["k"], t["v"], o, bad)
    # a copy is (as a checkpointed activation is one)
    a = ops().attention_backward(do, t["q"], t["k"], t["v"], o, saved)
    b = ops().attention_backward(do, t["q"], t["k"], t["v"], o, saved.clone())
    assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


@pytest.mark.parametrize("b,s,h,kv,d,causal,window,buckets", [
    (40, 64, 8, 8, 128, True, 4, 0), (40, 64, 8, 4, 64, False, 2, 0), (3, 300, 16, 16, 80, False, 30, 0),
    (40, 64, 8, 8, 32, True, 9, 0), (40, 64, 8, 8, 128, True, 4, 8), (90, 20, 8, 8, 96, False, 0, 8),
    (2, 64, 2, 2, 128, True, 4, 0)])   # (the last one is a small grid)
def test_rows_of_few_tokens(b, s, h, kv, d, causal, window, buckets):
    """Rows that see at most 64 tokens average no rounding away, so their products take
    probabilities and dS as two bf16 numbers each, whatever the size of the grid: these are off
    by 2^-17 and o, in D, by as much, 2^-8 of the 2^-9 of the results' own rounding.  So the
    errors are that rounding's, within a tenth.  (With one bf16 number each they are 1.4
    to 2 times that.)"""
    t, do = inputs(b, s, h, kv, d)
    how = dict(causal=causal, window=window)
    if buckets:
        how.update(rel_bias=normal(9, h, buckets), max_distance=16)
    got = run(t, do, **how)
    out, _ = ref.attention(t["q"], t["k"], t["v"], do, causal=causal, window=window, bias=how.get("rel_bias"),
                           max_distance=16)
    share = {n: float((got[n].cpu().double() - out[n]).norm() / (out[n].to(BF16).double() - out[n]).norm()) for n in got}
    assert all(x < 1.1 for x in share.values()), share


# Sinks whose workgroups are many: their queries in fewer chunks, or in one.
MANY_SINKS = [
    (7, 600, 8, 8, 32, True, 50, 300, 0, 0, None),
    (2, 1100, 8, 8, 64, True, 70, 700, 8, 30, (1100, 801)),
    (2, 1100, 8, 8, 128, False, 40, 700, 0, 0, None),
    (7, 600, 16, 8, 40, False, 50, 500, 0, 0, (600, 550, 480, 1, 0, 64, 333)),
]


@pytest.mark.parametrize("kind", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", MANY_SINKS, ids=lambda c: "-".join(str(x) for x in c[:10]))
def test_many_sinks(case, kind):
    test_attention(case, kind)


@pytest.mark.parametrize("grad_kind", [F32, BF16], ids=["f32", "bf16"])
def test_adamw_8_bit_codes_bit_by_bit(grad_kind):
    """Every bit of the codes: second moments have no sign, so 0 and 128, or 127 and 255 (not
    a number), are not alike; first moments may differ in the sign of a zero alone."""
    rng = np.random.RandomState(5)
    g = [rng.randn(1000) * 1e-3, np.ldexp(rng.randn(700), rng.randint(-40, 20, 700)), rng.randn(300) * 1e30,
         np.where(rng.rand(500) < 0.5, 0.0, rng.randn(500))]
    g[1][[3, 200, 500]], g[2][7] = (np.nan, np.inf, -np.inf), 0.0
    grads = [torch.from_numpy(x).float().to(grad_kind).cuda() for x in g]
    opt = ops().AdamW([torch.zeros(x.size, device="cuda") for x in g], grads, state_bits=8)
    for step in (1, 2, 3):
        before = state(opt)
        opt.step(step=step)
        for i, (p0, m0, v0) in enumerate(before):
            with np.errstate(invalid="ignore"):
                _, m, v = ref.adamw(p0, grads[i].cpu().double().numpy(), m0, v0, step=step, decay=True)
            (wm, ws), (wv, wvs) = ref.encode_m(m), ref.encode_v(v)
            assert np.array_equal(opt.exp_avg_sq[i].cpu().numpy(), wv), (step, i)
            assert np.array_equal(opt.exp_avg_sq_scale[i].cpu().numpy(), wvs), (step, i)
            assert np.array_equal(opt.exp_avg_scale[i].cpu().numpy(), ws), (step, i)
            c = opt.exp_avg[i].cpu().numpy()
            assert np.all((c == wm) | (c | wm == 128)), (step, i)
