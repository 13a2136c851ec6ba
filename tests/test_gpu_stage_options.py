"""Stages with a windowed or biased attention and with 8-bit Adam moments,
against a 64-bit build of the same layers (torch autograd on the CPU)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from synth import MB, gen_dy, gen_params, gen_x, get_config  # noqa: E402
from tests import operators_ref as ref  # noqa: E402
from tests.conftest import rel_l2  # noqa: E402
from tests.gpu_harness import log, to_device, to_host  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")


def layer(x, P, heads, eps, how):
    """One pre-LN layer in torch; P: its 12 parameters and, with a bias, the 13th."""
    def norm(z, g, b):
        return torch.nn.functional.layer_norm(z, (z.shape[-1],), g, b, eps)

    b, s, h = x.shape
    qkv = norm(x, P[0], P[1]) @ P[2] + P[3]
    q, k, v = (t.reshape(b, s, heads, h // heads) for t in qkv.split(h, -1))
    with_bias = dict(how, bias=P[12]) if len(P) > 12 else how
    o = ref.attention(q, k, v, **with_bias)[0]["o"].reshape(b, s, h)
    y = x + o @ P[4] + P[5]
    u = norm(y, P[6], P[7]) @ P[8] + P[9]
    return y + torch.nn.functional.gelu(u, approximate="tanh") @ P[10] + P[11]


def reference(cfg, params, mbs, how):
    """y and dx by micro-batch, and the gradients summed over them."""
    P = [[torch.tensor(np.asarray(p), dtype=torch.float64, requires_grad=True) for p in lay] for lay in params]
    flat = [p for lay in P for p in lay]
    total = [torch.zeros_like(p) for p in flat]
    y, dx = {}, {}
    for mb in mbs:
        x = torch.tensor(np.asarray(gen_x(cfg, *mb)), dtype=torch.float64, requires_grad=True)
        z = x
        for lay in P:
            z = layer(z, lay, cfg.heads, cfg.ln_eps, how)
        grads = torch.autograd.grad(z, [x] + flat, torch.tensor(np.asarray(gen_dy(cfg, *mb)), dtype=torch.float64))
        y[mb], dx[mb] = z.detach().numpy(), grads[0].numpy()
        total = [t + g for t, g in zip(total, grads[1:])]
    n = len(P[0])
    return y, dx, [[g.numpy() for g in total[l * n:(l + 1) * n]] for l in range(cfg.layers)]


def params_of(cfg, buckets, seed=5):
    rng = np.random.RandomState(seed)
    got = [list(lay) for lay in gen_params(cfg)]
    if buckets:
        for lay in got:
            lay.append(rng.randn(cfg.heads, buckets).astype(np.float32))
    return got


def make(cfg, buckets=0, **kw):
    from paper_2405_14009_amd import Stage
    st = Stage.from_config(cfg, rel_buckets=buckets, **kw)
    st.load_params(params_of(cfg, buckets))
    return st


def train(st, cfg, mbs):
    """F, B and W (one call, then the rest in one batched call) of the micro-batches."""
    y = {mb: to_host(st.forward(mb, to_device(gen_x(cfg, *mb), cfg.dtype))) for mb in mbs}
    dx = {mb: to_host(st.backward_input(mb, to_device(gen_dy(cfg, *mb), cfg.dtype))) for mb in mbs}
    st.backward_weight(mbs[-1])
    if len(mbs) > 1:
        st.backward_weight_many(mbs[:-1])
    from paper_2405_14009_amd import RC_READ_GRAD
    return y, dx, st.read_all(RC_READ_GRAD)


STAGES = [
    # base workload, causal, window, sinks, buckets, max_distance
    ("small_bf16", True, 96, 4, 0, 0),
    ("small_bf16", True, 0, 0, 32, 128),
    ("small_bf16", False, 50, 70, 16, 40),
    ("small_f32", True, 40, 3, 0, 0),
    ("small_f32", False, 0, 0, 32, 64),
    ("small_f32", True, 33, 1, 8, 20),
]


@pytest.mark.parametrize("case", STAGES, ids=lambda c: "-".join(str(x) for x in c))
def test_stage_against_a_64_bit_build(case):
    name, causal, window, sinks, buckets, far = case
    cfg = get_config(name).with_(causal=causal, n_mb=3)
    how = dict(causal=causal, window=window, sinks=sinks)
    if buckets:
        how["max_distance"] = far
    mbs = [(0, 0), (1, 0), (2, 1)]
    want = reference(cfg, params_of(cfg, buckets), mbs, how)
    st = make(cfg, buckets, window=window, sinks=sinks, rel_max_distance=far)
    assert st.attention_kernels() == "operator"
    y, dx, grads = train(st, cfg, mbs)
    t = 1e-5 if cfg.dtype == "f32" else 2e-2
    worst = {("y", mb): rel_l2(y[mb], want[0][mb]) for mb in mbs}
    worst.update({("dx", mb): rel_l2(dx[mb], want[1][mb]) for mb in mbs})
    h = cfg.hidden
    for l in range(cfg.layers):
        for p in range(st.num_params):
            a, b = grads[l][p], want[2][l][p]
            if p == 3:  # the key bias has a zero gradient without a relative bias's help, too
                a, b = np.delete(a, np.s_[h:2 * h]), np.delete(b, np.s_[h:2 * h])
            worst[(l, p)] = rel_l2(a, b)
    log(f"[options] {case}: worst {max(worst.values()):.2e}, bias {[worst.get((l, 12)) for l in range(cfg.layers)]}")
    bad = {k: v for k, v in worst.items() if v > t}
    assert not bad, bad
    st.close()


def test_a_window_as_long_as_the_sequence_is_no_window():
    cfg = get_config("small_bf16").with_(n_mb=1)
    plain, wide = make(cfg), make(cfg, window=cfg.seq, sinks=7)
    assert plain.attention_kernels() == wide.attention_kernels() != "operator"
    a, b = train(plain, cfg, [(0, 0)]), train(wide, cfg, [(0, 0)])
    assert np.array_equal(a[0][(0, 0)], b[0][(0, 0)]) and np.array_equal(a[1][(0, 0)], b[1][(0, 0)])


def test_library_work_memory_gives_the_same():
    cfg = get_config("small_bf16").with_(n_mb=2)
    kw = dict(buckets=16, window=70, sinks=3, rel_max_distance=50, adam_state_bits=8)
    a, b = make(cfg, **kw), make(cfg, static_work=True, **kw)
    ra, rb = train(a, cfg, [(0, 0), (1, 0)]), train(b, cfg, [(0, 0), (1, 0)])
    assert all(np.array_equal(ra[0][m], rb[0][m]) and np.array_equal(ra[1][m], rb[1][m]) for m in ra[0])
    assert all(np.array_equal(x, z) for la, lb in zip(ra[2], rb[2]) for x, z in zip(la, lb))


def moments8(st, what):
    return [[x.astype(np.float64).ravel() for x in lay] for lay in st.read_all(what)]


def check_step8(st, before, grads, scale, step):
    """A stage's 8-bit step, parameter by parameter: the moments are those of the 64-bit step
    after rounding to codes, the parameters a few 32-bit half-steps from it."""
    from paper_2405_14009_amd import RC_READ_ADAM_M, RC_READ_ADAM_V, RC_READ_PARAM
    half = 2.0 ** -24
    m1, v1, p1 = moments8(st, RC_READ_ADAM_M), moments8(st, RC_READ_ADAM_V), st.read_all(RC_READ_PARAM)
    for l, lay in enumerate(p1):
        for i, got in enumerate(lay):
            p0, m0, v0 = (x[l][i] for x in before)
            p, m, v = ref.adamw(p0.astype(np.float64).ravel(), grads[l][i].astype(np.float64).ravel(), m0, v0, step=step,
                                decay=i in (2, 4, 8, 10), grad_scale=scale)
            assert np.array_equal(m1[l][i], ref.decode_m(*ref.encode_m(m)).astype(np.float32)), (l, i)
            assert np.array_equal(v1[l][i], ref.decode_v(*ref.encode_v(v)).astype(np.float32)), (l, i)
            bound = 4 * half * np.abs(p) + 16 * half * np.abs(p - p0.ravel()) + 1e-30
            assert np.all(np.abs(got.ravel() - p) <= bound), (l, i)


def test_8_bit_moments_step_and_rollback():
    """Steps, a rollback and the step again, with everything that a stage can have; next to
    it the tensors that its neighbours hold, in an AdamW of their own."""
    from paper_2405_14009_amd import RC_READ_ADAM_M, RC_READ_ADAM_V, RC_READ_PARAM, AdamW
    cfg = get_config("small_bf16").with_(n_mb=2, layers=1)
    st = make(cfg, 16, window=70, sinks=3, rel_max_distance=50, adam_state_bits=8)
    embedding = torch.randn(333, cfg.hidden, device="cuda") * 0.02
    outer = AdamW([embedding], [torch.zeros_like(embedding)], state_bits=8)
    mbs = [(0, 0), (1, 0)]
    for step in range(1, 4):
        before = (st.read_all(RC_READ_PARAM), moments8(st, RC_READ_ADAM_M), moments8(st, RC_READ_ADAM_V))
        y, dx, grads = train(st, cfg, mbs)
        # the stage's input gradient, as the gradient of the embedding's rows
        rows = torch.from_numpy(dx[(0, 0)].reshape(-1, cfg.hidden)[:333]).float().cuda()
        outer.grads[0].copy_(rows)
        e0 = embedding.cpu().double().numpy().ravel()
        em, ev = (x[0].cpu().double().numpy() for x in outer.moments())
        outer.step(0.5)
        p, m, v = ref.adamw(e0, rows.cpu().double().numpy().ravel(), em, ev, step=step, decay=True, grad_scale=0.5)
        got = [x[0].cpu().numpy() for x in outer.moments()]
        assert np.array_equal(got[0], ref.decode_m(*ref.encode_m(m)).astype(np.float32))
        assert np.array_equal(got[1], ref.decode_v(*ref.encode_v(v)).astype(np.float32))
        st.optimizer_step(0.5)
        check_step8(st, before, grads, 0.5, step)
        if step == 2:  # back, and the same step again
            after = (moments8(st, RC_READ_ADAM_M), moments8(st, RC_READ_ADAM_V))
            st.optimizer_rollback()
            back = (st.read_all(RC_READ_PARAM), moments8(st, RC_READ_ADAM_M), moments8(st, RC_READ_ADAM_V))
            for l in range(cfg.layers):
                for i in range(st.num_params):
                    assert np.array_equal(back[1][l][i], before[1][l][i]) and np.array_equal(back[2][l][i], before[2][l][i])
                    # the update added back and the decay divided out: a few half-steps
                    d = np.abs(back[0][l][i].astype(np.float64) - before[0][l][i])
                    assert np.all(d <= 2.0 ** -21 * (np.abs(before[0][l][i]) + 2e-4)), (l, i)
            train(st, cfg, mbs)
            st.optimizer_step(0.5)
            assert len(after[0]) == cfg.layers
    st.close()


def test_window_stage_in_a_graph():
    """F, B and W of a windowed and biased stage captured and replayed, the eager calls in between."""
    cfg = get_config("small_bf16").with_(n_mb=1, layers=1)
    kw = dict(buckets=16, window=70, sinks=3, rel_max_distance=50)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        st, eager = make(cfg, stream=side, **kw), make(cfg, stream=side, **kw)
        x, dy = to_device(gen_x(cfg, 0), cfg.dtype), to_device(gen_dy(cfg, 0), cfg.dtype)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            st.forward((0, 0), x, y)
            st.backward((0, 0), dy, dx)
        for turn in range(3):
            x.copy_(to_device(gen_x(cfg, 3 + turn), cfg.dtype))
            side.synchronize()
            graph.replay()
            want_y = eager.forward((0, 0), x)
            want_dx = eager.backward((0, 0), dy)
            eager.optimizer_skip()
            side.synchronize()
            assert torch.equal(y, want_y) and torch.equal(dx, want_dx), turn


@pytest.mark.parametrize("bits", [8, 32])
def test_the_step_after_a_rollback(bits):
    """Back from a step, a stage computes with the parameters that it reads out (its bf16 copies
    are theirs), and its next step is that of its state before: the right bank and number."""
    from paper_2405_14009_amd import RC_READ_ADAM_M, RC_READ_ADAM_V, RC_READ_PARAM
    cfg = get_config("small_bf16").with_(n_mb=1, layers=1)
    kw = dict(window=70, sinks=3, rel_max_distance=50, adam_state_bits=bits)
    st, mbs = make(cfg, 16, **kw), [(0, 0)]
    for step in (1, 2, 3):
        train(st, cfg, mbs)
        st.optimizer_step(0.5)
        st.optimizer_rollback()
        before = (st.read_all(RC_READ_PARAM), moments8(st, RC_READ_ADAM_M), moments8(st, RC_READ_ADAM_V))
        y, dx, grads = train(st, cfg, mbs)
        other = make(cfg, 16, **kw)
        other.load_params(before[0])
        y2, dx2, grads2 = train(other, cfg, mbs)
        assert np.array_equal(y[mbs[0]], y2[mbs[0]]) and np.array_equal(dx[mbs[0]], dx2[mbs[0]])
        assert all(np.array_equal(a, b) for a, b in zip(grads[0], grads2[0]))
        other.close()
        st.optimizer_step(0.5)
        if bits == 8:
            check_step8(st, before, grads, 0.5, step)
    st.close()
