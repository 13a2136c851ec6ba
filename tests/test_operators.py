"""CPU checks of the operators on the caller's tensors: memory sizes, refusals
of the C ABI (nothing is enqueued), buckets, and the plain forms that the GPU
tests compare with.  No compute call runs here."""
import ctypes
import math

import numpy as np
import pytest

from tests import operators_ref as ref
from tests.test_abi_cpu import lib_or_skip


def config(**kw):
    L, _ = lib_or_skip()
    base = dict(dtype=L.RC_BF16, batch=2, seq_len=300, heads=4, kv_heads=2, head_dim=64, causal=1, window=0, sinks=0,
                buckets=0, max_distance=0, bias_dtype=L.RC_FP32, scale=0.125)
    base.update(kw)
    return L.RcAttention(**base)


def memory(**kw):
    L, lib = lib_or_skip()
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    st = lib.rc_attention_memory(ctypes.byref(config(**kw)), ctypes.byref(a), ctypes.byref(b))
    return st, a.value, b.value


def up(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("batch,seq,heads,kv,d", [(1, 1, 1, 1, 8), (2, 136, 3, 3, 64), (3, 1000, 8, 2, 128)])
def test_attention_memory_holds_every_part(bf16, batch, seq, heads, kv, d):
    L, _ = lib_or_skip()
    size = dict(dtype=L.RC_BF16 if bf16 else L.RC_FP32, batch=batch, seq_len=seq, heads=heads, kv_heads=kv, head_dim=d)
    rows = batch * heads * (-(-seq // 64) * 64)
    blocks = -(-seq // 128)
    st, saved, work = memory(**size)
    assert st == 0
    # two statistics a row, rows padded to blocks of 64, and what o's rounding drops
    assert saved >= 2 * 4 * rows + (2 * batch * seq * heads * d if bf16 else 0)
    assert work >= 4 * rows
    # with a bias: a sum per bucket of each block of 32 queries
    blocks = -(-seq // 32)
    assert memory(**size, buckets=32, max_distance=128)[2] >= up(4 * rows) + 4 * batch * heads * blocks * 32
    # with sinks in a window: shares of 32 rows of dk and dv, of the window and each chunk of queries
    if seq > 512:
        chunks = -(-seq // 512)
        got = memory(**size, window=40, sinks=4, buckets=32, max_distance=128)[2]
        assert got >= up(4 * rows) + 4 * batch * heads * blocks * 32 + 4 * batch * kv * (1 + chunks) * 2 * 32 * d


BAD_ATTENTION = [
    (dict(dtype=7), "INVALID_ARG", b"dtype"),
    (dict(batch=0), "INVALID_ARG", b"positive"),
    (dict(seq_len=0), "INVALID_ARG", b"positive"),
    (dict(heads=4, kv_heads=3), "INVALID_ARG", b"multiple"),
    (dict(causal=2), "INVALID_ARG", b"causal"),
    (dict(window=-1), "INVALID_ARG", b"negative"),
    (dict(sinks=-1), "INVALID_ARG", b"negative"),
    (dict(scale=0.0), "INVALID_ARG", b"scale"),
    (dict(scale=-1.0), "INVALID_ARG", b"scale"),
    (dict(scale=math.nan), "INVALID_ARG", b"scale"),
    (dict(scale=math.inf), "INVALID_ARG", b"scale"),
    (dict(scale=3e38), "INVALID_ARG", b"scale"),
    (dict(buckets=-4), "INVALID_ARG", b"buckets"),
    (dict(buckets=1, max_distance=8), "INVALID_ARG", b"buckets"),
    (dict(buckets=7, max_distance=8, causal=0), "INVALID_ARG", b"even"),
    (dict(buckets=2, max_distance=8, causal=0), "INVALID_ARG", b"buckets"),
    (dict(buckets=32, max_distance=16), "INVALID_ARG", b"max_distance"),
    (dict(buckets=32, max_distance=128, bias_dtype=5), "INVALID_ARG", b"bias_dtype"),
    (dict(buckets=256, max_distance=1000), "UNSUPPORTED", b"buckets"),
    (dict(buckets=32, max_distance=2000), "UNSUPPORTED", b"max_distance"),
    (dict(head_dim=60), "UNSUPPORTED", b"head_dim"),
    (dict(head_dim=136), "UNSUPPORTED", b"head_dim"),
    (dict(seq_len=(1 << 24) + 1), "UNSUPPORTED", b"seq_len"),
    (dict(seq_len=1, batch=1 << 24, heads=1, kv_heads=1), "UNSUPPORTED", b"blocks"),
    (dict(seq_len=129, batch=1 << 20, heads=8, kv_heads=1), "UNSUPPORTED", b"blocks"),
    (dict(seq_len=128, batch=1 << 20, heads=4, kv_heads=4, window=2, sinks=128), "UNSUPPORTED", b"blocks"),
    (dict(seq_len=1 << 24, batch=1 << 12, heads=8, kv_heads=8), "UNSUPPORTED", b"blocks"),
]


@pytest.mark.parametrize("kw,status,word", BAD_ATTENTION, ids=lambda x: str(x)[:40])
def test_attention_refusals(kw, status, word):
    L, lib = lib_or_skip()
    assert memory(**kw)[0] == getattr(L, "RC_ERR_" + status)
    assert word in lib.rc_last_error()


@pytest.mark.parametrize("bf16,sinks", [(True, 0), (False, 0), (True, 9), (False, 9)])
def test_attention_memory_holds_the_shares_of_parts(bf16, sinks):
    """4 heads a key head and 16 blocks of 32 keys: four parts, of the keys and of the sinks' chunks."""
    L, _ = lib_or_skip()
    size = dict(dtype=L.RC_BF16 if bf16 else L.RC_FP32, batch=1, seq_len=500, heads=4, kv_heads=1, head_dim=72)
    if sinks:
        size.update(window=300, sinks=sinks)
    shares = 4 * 2 * 500 + (4 * 2 * 32 if sinks else 0)
    assert memory(**size)[2] >= up(4 * 4 * 512) + 4 * 96 * shares


def test_attention_takes_the_most_blocks_of_a_launch():
    assert memory(seq_len=128, batch=(1 << 24) - 2, heads=1, kv_heads=1)[0] == 0


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("batch,seq,heads,kv,d", [(1, 8192, 32, 32, 128), (1, 8192, 32, 8, 128), (16, 2048, 16, 16, 64)])
def test_attention_memory_of_many_sinks(bf16, batch, seq, heads, kv, d):
    """The shares of the sinks' rows: two of each row, or as many as 1024 workgroups of 32 rows write."""
    L, _ = lib_or_skip()
    size = dict(dtype=L.RC_BF16 if bf16 else L.RC_FP32, batch=batch, seq_len=seq, heads=heads, kv_heads=kv, head_dim=d,
                window=512)
    plain = memory(**size)[2]
    for sinks in (1, 4, 33, 512, 1500, seq - 192):
        rows = -(-sinks // 32) * 32
        share = memory(**size, sinks=sinks)[2] - plain
        assert 0 < share <= 4 * 2 * d * (batch * kv * rows + max(1024 * 32, batch * heads * rows)) + 256, (sinks, share)


@pytest.mark.parametrize("seq,heads,batch,masks", [
    (1, 1, (1 << 24) - 2, {}),
    (32, 2, (1 << 23) - 2, {}),      # a launch may have a workgroup more per head (the bias gradient)
    (33, 1, (1 << 23) - 1, {}),
    (64, 1, (1 << 23) - 1, {}),
    (128, 1, (1 << 22) - 1, {}),
    (128, 4, (1 << 20) - 1, dict(window=8)),
    (1 << 24, 31, 1, dict(window=16)),
])
def test_fp32_attention_takes_the_most_blocks_of_a_launch(seq, heads, batch, masks):
    """fp32 kernels take 32 tokens a workgroup: the largest batches whose launches are
    below 2^24 workgroups, and the next ones, which are refused up front."""
    L, lib = lib_or_skip()
    size = dict(dtype=L.RC_FP32, seq_len=seq, heads=heads, kv_heads=heads, head_dim=8, **masks)
    assert memory(**size, batch=batch)[0] == L.RC_OK
    more = dict(heads=heads + 1, kv_heads=heads + 1, batch=batch) if batch == 1 else dict(batch=batch + 1)
    assert memory(**{**size, **more})[0] == L.RC_ERR_UNSUPPORTED and b"blocks" in lib.rc_last_error()


def test_a_stage_refuses_launches_beyond_the_most_blocks():
    L, lib = lib_or_skip()
    cfg = dict(hidden=8, heads=1, ffn=8, seq_len=64, micro_batch=1 << 23, dtype=L.RC_FP32)
    assert stage_memory(cfg, window=2)[0] == L.RC_ERR_UNSUPPORTED and b"blocks" in lib.rc_last_error()


def test_attention_refuses_tensors_before_any_device_work():
    """Null, misaligned, overlapping and oversized tensors (host addresses that are
    never touched)."""
    L, lib = lib_or_skip()
    c = config()
    at = 1 << 20

    def view(data=at, b=300 * 256, t=256, h=64):
        return L.RcView(data, b, t, h)

    def forward(c=c, q=None, k=None, v=None, bias=None, lengths=None, o=None, saved=None):
        q, o = q or view(), o or view(8 * at)
        k, v = k or view(2 * at, b=300 * 128, t=128), v or view(3 * at, b=300 * 128, t=128)
        r = ctypes.byref
        return lib.rc_attention_forward(r(c), r(q), r(k), r(v), bias, lengths, r(o), saved, None)

    def backward(dq=None, dk=None, dv=None, dbias=None, saved=256, work=512, c=c, bias=None):
        r = ctypes.byref
        q, o, do = view(), view(8 * at), view(9 * at)
        k, v = view(2 * at, b=300 * 128, t=128), view(3 * at, b=300 * 128, t=128)
        dq, dk = dq or view(4 * at), dk or view(5 * at, b=300 * 128, t=128)
        dv = dv or view(6 * at, b=300 * 128, t=128)
        return lib.rc_attention_backward(r(c), r(q), r(k), r(v), bias, None, r(o), saved, r(do), r(dq), r(dk), r(dv),
                                         dbias, work, None)

    bad = L.RC_ERR_INVALID_ARG
    assert lib.rc_attention_forward(None, None, None, None, None, None, None, None, None) == bad
    assert lib.rc_attention_memory(None, None, None) == bad
    assert forward(q=view(0)) == bad and b"null q" in lib.rc_last_error()
    assert forward(q=view(at + 8)) == bad and b"16 bytes" in lib.rc_last_error()
    assert forward(k=view(2 * at, t=132)) == bad and b"16 bytes" in lib.rc_last_error()
    assert forward(v=view(2 * at, h=-64)) == bad and b"negative" in lib.rc_last_error()
    assert forward(o=view(8 * at, t=0)) == bad and b"overlap" in lib.rc_last_error()
    assert forward(o=view(8 * at, h=56)) == bad and b"overlap" in lib.rc_last_error()
    assert forward(o=view(at)) == bad and b"inputs" in lib.rc_last_error()
    assert forward(bias=64) == bad and b"bias" in lib.rc_last_error()
    assert forward(c=config(buckets=8, max_distance=16)) == bad and b"bias" in lib.rc_last_error()
    assert forward(lengths=66) == bad and b"aligned" in lib.rc_last_error()
    assert forward(saved=128) == bad and b"256" in lib.rc_last_error()
    big = 8 * ((2 ** 31 // 2) // 299 // 8 + 1)
    assert forward(q=view(b=0, t=big)) == L.RC_ERR_UNSUPPORTED and b"2^31" in lib.rc_last_error()
    f32 = config(dtype=L.RC_FP32)
    assert forward(c=f32, q=view(b=0, t=1 << 24)) == L.RC_ERR_UNSUPPORTED and b"token_stride" in lib.rc_last_error()
    assert backward(dq=view(at)) == bad and b"inputs" in lib.rc_last_error()
    assert backward(dk=view(6 * at, b=300 * 128, t=128)) == bad and b"share" in lib.rc_last_error()
    assert backward(dq=view(4 * at, b=8)) == bad and b"overlap" in lib.rc_last_error()
    assert backward(saved=None) == bad and backward(work=None) == bad and backward(work=8) == bad
    assert backward(c=config(buckets=8, max_distance=16), bias=64) == bad and b"dbias" in lib.rc_last_error()


def test_adamw_refusals():
    L, lib = lib_or_skip()
    adam = L.RcAdamConfig(1e-4, 0.9, 0.95, 1e-8, 0.1)

    def step(bits=32, n=1, number=1, adam=adam, **kw):
        base = dict(param=4096, grad=8192, exp_avg=12288, exp_avg_sq=16384, count=7, grad_dtype=L.RC_FP32, decay=1)
        base.update(kw)
        t = (L.RcAdamwTensor * 1)(L.RcAdamwTensor(**base))
        return lib.rc_adamw_step(t, n, ctypes.byref(adam) if adam else None, bits, number, 1.0, None)

    bad = L.RC_ERR_INVALID_ARG
    for kw, word in ((dict(bits=16), b"state_bits"), (dict(number=0), b"step"), (dict(n=-1), b"negative"),
                     (dict(adam=None), b"null"), (dict(count=-1), b"count"), (dict(count=1 << 50), b"count"),
                     (dict(count=(1 << 34) - 1023), b"count"),
                     (dict(grad_dtype=3), b"grad_dtype"), (dict(param=None), b"null"), (dict(exp_avg=None), b"null"),
                     (dict(bits=8), b"scales"), (dict(exp_avg_scale=64), b"scales"),
                     (dict(bits=8, exp_avg_scale=64), b"scales"), (dict(param=4098), b"aligned"),
                     (dict(exp_avg=4098), b"aligned"), (dict(copy=4097), b"aligned"),
                     (dict(adam=L.RcAdamConfig(1e-4, 1.0, 0.95, 1e-8, 0.1)), b"beta"),
                     (dict(adam=L.RcAdamConfig(1e-4, 0.9, math.nan, 1e-8, 0.1)), b"beta")):
        assert step(**kw) == bad, kw
        assert word in lib.rc_last_error(), (kw, lib.rc_last_error())
    assert lib.rc_adamw_step(None, 1, ctypes.byref(adam), 32, 1, 1.0, None) == bad
    assert lib.rc_adamw_step(None, 0, ctypes.byref(adam), 32, 1, 1.0, None) == L.RC_OK   # nothing to do
    assert step(count=0, param=None) == L.RC_OK
    t = (L.RcAdamwTensor * 1)(L.RcAdamwTensor(exp_avg=4096, exp_avg_sq=8192, count=4))
    out = (ctypes.c_void_p * 1)(64)
    assert lib.rc_adamw_read(t, 1, 32, out, (ctypes.c_void_p * 1)(None), None) == bad
    assert lib.rc_adamw_read(t, 1, 8, out, out, None) == bad and b"scales" in lib.rc_last_error()
    assert lib.rc_adamw_read(t, 1, 32, out, None, None) == bad


def test_adamw_read_refuses_destinations_that_overlap():
    """Two destinations in one place, partly so, or a destination among the moments (host
    addresses that are never touched); empty tensors have none."""
    L, lib = lib_or_skip()

    def read(m, v, bits=32, counts=(100, 50)):
        kw = [dict(exp_avg=4096, exp_avg_sq=8192), dict(exp_avg=12288, exp_avg_sq=16384)]
        if bits == 8:
            kw = [dict(k, exp_avg_scale=20480 + 64 * i, exp_avg_sq_scale=24576 + 64 * i) for i, k in enumerate(kw)]
        t = (L.RcAdamwTensor * 2)(*[L.RcAdamwTensor(count=c, **k) for c, k in zip(counts, kw)])
        P = ctypes.c_void_p * 2
        return lib.rc_adamw_read(t, 2, bits, P(*m), P(*v), None)

    at = 1 << 20
    for bits in (32, 8):
        for m, v in (((at, 2 * at), (at, 3 * at)), ((at, 2 * at), (3 * at, 2 * at + 196)), ((at, at + 396), (2 * at, 3 * at)),
                     ((at, 2 * at), (2 * at - 396, 3 * at)), ((at, 4096), (2 * at, 3 * at)), ((4096, at), (2 * at, 3 * at)),
                     ((at, 2 * at), (16384 - 396, 3 * at))):
            assert read(m, v, bits) == L.RC_ERR_INVALID_ARG, (bits, m, v)
            assert b"overlap" in lib.rc_last_error()
    for m, v in (((24576, at), (2 * at, 3 * at)), ((at, 20480 + 64), (2 * at, 3 * at))):
        assert read(m, v, 8) == L.RC_ERR_INVALID_ARG and b"overlap" in lib.rc_last_error()
    assert read((at, 4096), (2 * at, 4096), counts=(0, 0)) == L.RC_OK


def stage_memory(cfg_kw=None, **options):
    L, lib = lib_or_skip()
    base = dict(num_layers=2, hidden=256, heads=4, ffn=1024, seq_len=128, micro_batch=2, causal=1, dtype=L.RC_BF16,
                ln_eps=1e-5, max_stashed_mb=2, max_inflight_mb=1)
    base.update(cfg_kw or {})
    o = L.RcStageOptions(**options)
    a, b, c = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    st = lib.rc_stage_memory_requirements_with(ctypes.byref(L.RcStageConfig(**base)), ctypes.byref(o), ctypes.byref(a),
                                               ctypes.byref(b), ctypes.byref(c))
    return st, a.value, b.value, c.value


def test_stage_options():
    L, lib = lib_or_skip()
    plain = stage_memory()
    assert plain[0] == L.RC_OK
    assert stage_memory(window=128, sinks=5) == plain          # a window as long as the sequence is none
    assert stage_memory(adam_state_bits=32) == plain
    for options, word in ((dict(window=-1), b"negative"), (dict(buckets=-2), b"negative"),
                          (dict(adam_state_bits=16), b"adam_state_bits"), (dict(static_work=2), b"static_work"),
                          (dict(buckets=1, max_distance=8), b"buckets"), (dict(buckets=32), b"max_distance")):
        assert stage_memory(**options)[0] == L.RC_ERR_INVALID_ARG, options
        assert word in lib.rc_last_error(), (options, lib.rc_last_error())
    assert stage_memory(buckets=32, max_distance=5000)[0] == L.RC_ERR_UNSUPPORTED
    assert stage_memory(dict(hidden=1024), window=8)[0] == L.RC_ERR_UNSUPPORTED   # heads of 256
    n = 2 * (4 * 256 * 256 + 2 * 256 * 1024 + 9 * 256 + 1024)
    # 8-bit moments: two banks of a byte a moment and two per 128, in place of 4 + 4 bytes
    small = stage_memory(adam_state_bits=8)
    assert abs((plain[1] - small[1]) - (8 * n - 4 * n * 129 / 128)) < 16384
    # the probabilities of a windowed stage are not kept, only statistics and what o's rounding drops
    assert stage_memory(window=40)[2] < plain[2]


def test_stage_options_on_a_dry_run():
    from paper_2405_14009_amd import RC_READ_PARAM, InvalidArgError, Stage
    kw = dict(num_layers=2, hidden=256, heads=4, ffn=1024, seq_len=128, micro_batch=2, max_stashed_mb=2, dry_run=True)
    st = Stage(**kw, window=40, sinks=2, rel_buckets=16, rel_max_distance=50, adam_state_bits=8)
    assert st.attention_kernels() == "operator" and st.num_params == 13
    T, rows = 256, 2 * 4 * 128
    a = st.stash_account()
    assert a["a_f"] == 2 * (2 * (8 * T * 256 + 2 * T * 1024) + 16 * T + 8 * rows + 2 * T * 256)
    assert a["s_w"] == 2 * (2 * (12 * T * 256 + 2 * T * 1024) + 16 * T + 4 * 4 * 16)
    st.forward((0, 0))
    st.backward((0, 0))
    st.optimizer_step()
    st.optimizer_rollback()
    assert [r[1] for r in st.op_log()] == [0, 1, 2, 3, 5]
    with pytest.raises(InvalidArgError):
        st.read(RC_READ_PARAM, 0, 12)       # a dry run has no device memory
    plain = Stage(**kw)
    assert plain.num_params == 12
    with pytest.raises((InvalidArgError, IndexError)):
        plain.read(RC_READ_PARAM, 0, 12)


@pytest.mark.parametrize("option", ["window", "sinks", "rel_buckets", "rel_max_distance", "adam_state_bits"])
@pytest.mark.parametrize("beyond", [1 << 32, -(1 << 32), 1 << 31])
def test_numbers_beyond_32_bits_are_refused(option, beyond):
    """A number that the library's 32 bits would hold as another one."""
    from paper_2405_14009_amd import Stage
    kw = dict(num_layers=1, hidden=256, heads=4, ffn=1024, seq_len=128, micro_batch=2, dry_run=True)
    good = dict(window=40, sinks=2, rel_buckets=16, rel_max_distance=50, adam_state_bits=8)
    Stage(**kw, **good)
    with pytest.raises(ValueError, match=option):
        Stage(**kw, **{**good, option: good[option] + beyond})


def test_attention_sizes_beyond_32_bits_are_refused():
    from paper_2405_14009_amd import operators
    L, _ = lib_or_skip()
    names = ("batch", "seq_len", "heads", "kv_heads", "head_dim", "causal", "window", "sinks", "buckets", "max_distance")
    good = (2, 300, 4, 2, 64, 1, 40, 3, 16, 50)
    call = lambda sizes: operators._config(L.RC_BF16, *sizes, L.RC_FP32, 0.125)   # noqa: E731
    assert call(good)[1] > 0
    for i, name in enumerate(names):
        with pytest.raises(ValueError, match=name):
            call(good[:i] + (good[i] + (1 << 32),) + good[i + 1:])


def test_buckets_by_their_definition():
    """The test's own bucket against the logarithms, away from their ties, and at the ties."""
    for causal, buckets, far in ((True, 32, 128), (False, 32, 128), (True, 16, 40), (False, 64, 512), (True, 2, 2)):
        side = buckets if causal else buckets // 2
        exact = side // 2
        for n in range(0, 600):
            c = ref.bucket(-n, buckets, far, causal)
            assert 0 <= c < side and (n >= exact or c == n)
            if n >= exact:
                x = exact + math.log(n / exact) / math.log(far / exact) * (side - exact)
                if abs(x - round(x)) > 1e-6:
                    assert c == min(int(x), side - 1), (n, c, x)
                else:
                    assert c == min(round(x), side - 1), (n, c, x)
            if not causal and n:
                assert ref.bucket(n, buckets, far, causal) == c + side


def test_moment_formats():
    """Codes and values of the 8-bit moments: every code back to itself, ties to even, borders."""
    for encode, decode, table, bias in ((ref.encode_m, ref.decode_m, ref.M_TABLE, 127),
                                        (ref.encode_v, ref.decode_v, ref.V_TABLE, 160)):
        codes = np.arange(table.size)
        codes = np.append(codes, [table.size - 1] * (-codes.size % 128))
        values = table[codes] * 2.0 ** -20
        for at in range(0, codes.size, 128):   # with the largest code in each block its power of two is known
            block = values[at:at + 128].copy()
            block[0] = table[-1] * 2.0 ** -20
            c, s = encode(block)
            assert s[0] == bias - 20 and np.array_equal(c[1:], codes[at + 1:at + 128])
            assert np.array_equal(decode(c, s), block)
        mid = (table[:-1] + table[1:]) / 2
        for i in range(0, mid.size, 127):
            block = np.concatenate((mid[i:i + 127], [table[-1]]))
            c, _ = encode(block)
            want = np.arange(i, i + block.size - 1)
            want = want + want % 2
            if encode is ref.encode_v:
                want[:1] = np.where(want[:1] == 0, 1, want[:1])
            assert np.array_equal(c[:-1], want)
    assert ref.encode_v(np.array([1e-30, 1.0]))[0][0] == 1 and ref.encode_v(np.array([0.0, 1.0]))[0][0] == 0


@pytest.mark.parametrize("name,cls", [
    ("void (anonymous namespace)::attn_op_fwd_k<(anonymous namespace)::TileB16<128>, true>(AttnOpArgs)", "attn_fwd"),
    ("void (anonymous namespace)::attn_op_fwd32_k<(anonymous namespace)::TileF32<64>, false>(AttnOpArgs)", "attn_fwd"),
    ("void (anonymous namespace)::attn_op_dq_k<(anonymous namespace)::TileB16<64>, true>(AttnOpArgs)", "attn_bwd"),
    ("void (anonymous namespace)::attn_op_dkv32_k<(anonymous namespace)::TileB16<64>, true>(AttnOpArgs)", "attn_bwd"),
    ("void (anonymous namespace)::attn_op_sum_k<(anonymous namespace)::TileB16<64> >(AttnOpArgs)", "attn_bwd"),
    ("(anonymous namespace)::attn_op_add_dbias_k(AttnOpShares, int, long, float*, int)", "reduce"),
    ("void (anonymous namespace)::adamw_tensors_k<8, 1>((anonymous namespace)::Args)", "adamw"),
])
def test_profile_classes_of_the_operators(name, cls):
    from paper_2405_14009_amd.profile_summary import kernel_class
    assert kernel_class(name) == cls
