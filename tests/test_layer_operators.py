"""CPU checks of the operators of a layer: work memory, refusals of the C ABI
(nothing is enqueued), and the plain forms that the GPU tests compare with.  No
compute call runs here."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from tests import layer_ref as ref
from tests.test_abi_cpu import lib_or_skip

REF = ctypes.byref
BASE = 1 << 20      # addresses that no call gets to read


def status(name):
    L, _ = lib_or_skip()
    return getattr(L, "RC_ERR_" + name)


def refused(st, name, word):
    _, lib = lib_or_skip()
    assert st == status(name), (st, lib.rc_last_error())
    assert word in lib.rc_last_error(), lib.rc_last_error()


def rows(**kw):
    L, _ = lib_or_skip()
    base = dict(dtype=L.RC_BF16, param_dtype=L.RC_FP32, rows=10, cols=64)
    base.update(kw)
    return L.RcRows(**base)


def drop(**kw):
    L, _ = lib_or_skip()
    base = dict(p=0.1, reserved=0, seed=1, offset=2, step=None)
    base.update(kw)
    return L.RcDropout(**base)


def at(slot, stride=64, shift=0):
    """A matrix in a place of its own."""
    L, _ = lib_or_skip()
    return REF(L.RcMatrix(BASE + slot * (1 << 16) + shift, stride))


def linear(**kw):
    L, _ = lib_or_skip()
    base = dict(dtype=L.RC_BF16, bias_dtype=L.RC_FP32, rows=10, in_=64, out=64, activation=0, by_out=0)
    base.update(kw)
    return L.RcLinear(**base)


def place(slot):
    return BASE + slot * (1 << 16)


# -- the generator ---------------------------------------------------------------

KNOWN = [   # the generator's published answers
    ([0] * 4, [0, 0], [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
     [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]),
]


@pytest.mark.parametrize("counter,key,words", KNOWN)
def test_philox_known_answers(counter, key, words):
    assert ref.philox(np.array(counter, dtype=np.uint64), key).tolist() == words


def test_mask_counts():
    """Kept elements of 400000: within five deviations of their expected number, in every column of eight."""
    for p in (0.1, 0.5, 0.9):
        d = ref.factor(1000, 400, p, 1234567890123456789, 3) != 0
        q = 1 - ref.threshold(p) / 65536
        assert abs(d.sum() - q * d.size) <= 5 * math.sqrt(d.size * q * (1 - q))
        each = d.reshape(1000, 50, 8).sum((0, 1))
        assert (np.abs(each - q * 50000) <= 5 * np.sqrt(50000 * q * (1 - q))).all()
        pairs = (d[:, 1:] & d[:, :-1]).mean()
        assert abs(pairs - q * q) <= 5 / math.sqrt(399000)
    assert ref.threshold(2.0 ** -18) == 0 and ref.threshold(2.0 ** -16) == 1 and ref.threshold(1.0) == 65536


def test_plain_norm_against_autograd():
    torch = pytest.importorskip("torch")
    g = np.random.default_rng(1)
    x, w, b, dy, dt = (g.standard_normal(s) for s in ((5, 33), 33, 33, (5, 33), (5, 33)))
    t = [torch.tensor(v, requires_grad=True) for v in (x, w, b)]
    y = torch.nn.functional.layer_norm(t[0], (33,), t[1], t[2], 1e-5)
    ((y * torch.tensor(dy)).sum() + (t[0] * torch.tensor(dt)).sum()).backward()
    n = ref.Norm(x, 1e-5, w, b)
    assert np.allclose(n.y, y.detach().numpy(), atol=1e-12)
    assert np.allclose(n.backward(dy, dt)[0], t[0].grad.numpy(), atol=1e-12)
    assert np.allclose((dy * n.xhat).sum(0), t[1].grad.numpy(), atol=1e-12)


@pytest.mark.parametrize("name", ["gelu", "silu", "relu", None])
def test_plain_activations_against_differences(name):
    u = np.linspace(-6, 6, 240) + 0.01
    h = 1e-5
    slope = (ref.act(name, u + h)[0] - ref.act(name, u - h)[0]) / (2 * h)
    assert np.allclose(ref.act(name, u)[1], slope, atol=1e-8)
    assert np.abs(ref.act(name, u)[1]).max() < 1.2   # what the bounds of the GPU tests count on
    assert np.abs(np.diff(ref.act(name, u)[1]) / np.diff(u)).max() < 1.2 or name == "relu"


# -- sizes of work memory ------------------------------------------------------------


@pytest.mark.parametrize("r,c", [(0, 1), (1, 1), (1000, 7), (5000, 4096), (3, 16384), (1 << 30, 8)])
def test_rows_memory(r, c):
    L, lib = lib_or_skip()
    n = ctypes.c_size_t()
    pad = 4 * (-(-c // 8) * 8)
    for call, vectors in ((lib.rc_dropout_memory, 1), (lib.rc_layer_norm_memory, 3)):
        assert call(REF(rows(rows=r, cols=c)), REF(n)) == 0
        assert n.value % (vectors * pad) == 0 and n.value <= vectors * pad * 2048
        # several workgroups leave partial sums, one (few rows) none
        assert (n.value > vectors * pad) == (r > 512) or r == 1000


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("r,i,o", [(0, 8, 8), (1, 4096, 16384), (300, 2048, 72), (4001, 8192, 2048), (1 << 22, 64, 64)])
def test_linear_memory(r, i, o, dtype):
    L, lib = lib_or_skip()
    for by_out in (0, 1):
        n = [ctypes.c_size_t() for _ in range(3)]
        assert lib.rc_linear_memory(REF(linear(dtype=dtype, rows=r, in_=i, out=o, by_out=by_out)), *map(REF, n)) == 0
        # a row of the bias gradient's sums at least, where they take more than one workgroup
        assert n[2].value >= 4 * o or (0 < r <= 8 if dtype else r <= 512)
        assert lib.rc_linear_memory(REF(linear(dtype=dtype, rows=r, in_=i, out=o)), None, None, None) == 0


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("by_out", [0, 1])
def test_few_tokens_fit_a_grid(dtype, by_out):
    """Weight gradients of few tokens take no work memory: up to 65535 blocks of 32 rows, which a grid's
    second dimension holds."""
    L, lib = lib_or_skip()
    n = ctypes.c_size_t()
    for rows_of, few in ((65535 * 32, True), (65535 * 32 + 8, False), ((1 << 21) - 8, False)):
        i, o = (8, rows_of) if by_out else (rows_of, 8)
        assert lib.rc_linear_memory(REF(linear(dtype=dtype, rows=1, in_=i, out=o, by_out=by_out)), None, None, REF(n)) == 0
        # (other products of one token sum dy's columns on their way: bf16)
        assert n.value == 0 if few else n.value > 0 or dtype == 0, (rows_of, n.value)


PLAN = r"""
#include <cstdio>
#include "gemm_plan.h"
int main() {
  const long dims[] = {8, 24, 40, 64, 136, 256, 264, 640, 1024, 1288, 5120, 16384};
  const long depths[] = {8, 72, 512, 2048, 6000, 65536};
  for (long M : dims) for (long N : dims) for (long K : depths) for (long room : {0L, 1L << 20, 16L << 20})
    for (int cus : {64, 256, 304}) {
      const long least = (N + 255) / 256 * M;   // what a caller provides at least
      for (long sums : {least, 4 * least}) {
        const GemmPlan p = plan_bf16(M, N, K, true, 1, room, sums, cus, true);
        if (p.colsum_a_rows(N) != (N + p.bn - 1) / p.bn * p.splits || p.colsum_a_rows(N) * M > sums) {
          std::printf("M %ld N %ld K %ld room %ld cus %d\n", M, N, K, room, cus);
          return 1;
        }
      }
    }
  for (long M : {1L, 16L, 64L}) for (long N : dims) for (long K : depths) for (long room : {0L, 1L << 16, 16L << 20})
    for (int cus : {64, 256, 304}) {
      const GemmPlan p = plan_stream(M, N, K, room, cus);
      if (p.tiles != (M + 63) / 64 * ((N + 63) / 64) || p.split_k % 64 || p.splits * (long)p.split_k < K ||
          (p.splits - 1) * (long)p.split_k >= K || p.split_floats > room || (p.splits > 1) != (p.split_floats > 0)) {
        std::printf("stream M %ld N %ld K %ld room %ld cus %d\n", M, N, K, room, cus);
        return 1;
      }
    }
  for (long M : dims) for (long N : dims) for (long K : depths) for (long room : {0L, 1L << 20, 16L << 20})
    for (int cus : {64, 256, 304}) {
      const F32Plan p = plan_f32(M, N, 1, K, 1, room, cus, true);
      if (p.tiles != (M + p.bm - 1) / p.bm * ((N + p.bn - 1) / p.bn) || p.split_k % 32 || p.splits * (long)p.split_k < K ||
          (p.splits - 1) * (long)p.split_k >= K || p.split_floats > room || (p.splits > 1) != (p.split_floats > 0) ||
          (p.bn != p.bm && (p.bm != 128 || p.bn != 256))) {
        std::printf("fp32 M %ld N %ld K %ld room %ld cus %d\n", M, N, K, room, cus);
        return 1;
      }
    }
  return 0;
}
"""


def test_plans_leave_room_for_the_left_operand_s_sums(tmp_path):
    """The choice of tile and split where a product sums its left operand's columns, and of few rows."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_14009_amd", "csrc")
    (tmp_path / "main.cpp").write_text(PLAN)
    exe = str(tmp_path / "main")
    subprocess.run([cxx, "-std=c++17", "-O2", "-I", csrc, str(tmp_path / "main.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


REACH = r"""
#include <cstdio>
#include "gemm_plan.h"
int main() {
  const long strides[] = {512, 2100000, 2105372, 2105376, 2105380, 2105384, 2200000, 4194304, 4226948, 4227192, 4227196, 5000000};
  int wide = 0;
  for (long M : {64L, 2048L, 4096L, 8192L, 16384L}) for (long N : {256L, 512L, 4096L}) for (long K : {64L, 512L, 4096L})
    for (long room : {0L, 16L << 20}) for (long lda : strides) for (long ldb : strides) for (bool kcontig : {false, true}) {
      if (f32_wide(lda, ldb)) continue;   // copied from 64-bit addresses
      const F32Plan p = plan_f32(M, N, 1, K, 1, room, 256, true, kcontig ? ldb : 0);
      // the last chunk of a tile's last row, k-contiguous (else its rows are the k-tile's 32)
      const long a = (p.bm - 1) * 4 * lda + 4 * 32, b = ((kcontig ? p.bn : 32) - 1) * 4 * ldb + 4 * (kcontig ? 32 : p.bn);
      if (a > 0x7fffffffL || b > 0x7fffffffL) {
        std::printf("M %ld N %ld K %ld lda %ld ldb %ld: tile %d x %d\n", M, N, K, lda, ldb, p.bm, p.bn);
        return 1;
      }
      wide += p.bn == 256;
      // no effect where the rows are in reach (255 * 4 * 2105376 + 128 is 2^31)
      const F32Plan q = plan_f32(M, N, 1, K, 1, room, 256, true);
      if (ldb < 2105376 && (q.bn != p.bn || q.bm != p.bm || q.splits != p.splits)) return 2;
    }
  return wide > 0 ? 0 : 3;
}
"""


def run_host(tmp_path, text):
    """The exit status and output of a host program over the launchers' headers."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_14009_amd", "csrc")
    (tmp_path / "main.cpp").write_text(text)
    exe = str(tmp_path / "main")
    subprocess.run([cxx, "-std=c++17", "-O2", "-I", csrc, str(tmp_path / "main.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    return r.returncode, r.stdout


def test_fp32_tiles_stay_in_reach_of_their_copies(tmp_path):
    """Copies reach 2^31 - 1 bytes from a tile's start (beyond, they deposit zeros): the rows of every tile that
    the plan takes lie within, whatever the row strides."""
    status, out = run_host(tmp_path, REACH)
    assert status == 0, (status, out)


# -- refusals ------------------------------------------------------------------------

BAD_ROWS = [(dict(dtype=9), "INVALID_ARG", b"dtype"), (dict(param_dtype=2), "INVALID_ARG", b"param_dtype"),
            (dict(rows=-1), "INVALID_ARG", b"rows"), (dict(rows=1 << 31), "INVALID_ARG", b"rows"),
            (dict(cols=0), "INVALID_ARG", b"cols"), (dict(cols=(1 << 29) + 1), "INVALID_ARG", b"cols")]


@pytest.mark.parametrize("kw,st,word", BAD_ROWS, ids=str)
def test_bad_sizes(kw, st, word):
    L, lib = lib_or_skip()
    n = ctypes.c_size_t()
    refused(lib.rc_dropout_memory(REF(rows(**kw)), REF(n)), st, word)
    refused(lib.rc_layer_norm_memory(REF(rows(**kw)), REF(n)), st, word)
    refused(lib.rc_dropout_forward(REF(rows(**kw)), REF(drop()), at(0), None, None, at(1), None), st, word)
    refused(lib.rc_dropout_backward(REF(rows(**kw)), REF(drop()), at(0), None, at(1), None, 0, None, None), st, word)
    refused(lib.rc_layer_norm_forward(REF(rows(**kw)), 1e-5, None, at(0), None, None, None, None, None, at(1), None,
                                      None), st, word)


@pytest.mark.parametrize("kw,word", [(dict(p=-0.1), b"p must"), (dict(p=1.5), b"p must"), (dict(p=math.nan), b"p must"),
                                     (dict(reserved=1), b"reserved"), (dict(step=place(9) + 4), b"step")], ids=str)
def test_bad_dropout(kw, word):
    L, lib = lib_or_skip()
    d = REF(drop(**kw))
    refused(lib.rc_dropout_forward(REF(rows()), d, at(0), None, None, at(1), None), "INVALID_ARG", word)
    refused(lib.rc_dropout_backward(REF(rows()), d, at(0), None, at(1), None, 0, None, None), "INVALID_ARG", word)
    refused(lib.rc_layer_norm_forward(REF(rows()), 1e-5, d, at(0), None, None, None, None, at(2), at(1), None, None),
            "INVALID_ARG", word)


def test_dropout_refusals():
    L, lib = lib_or_skip()
    r, d, many = REF(rows()), REF(drop()), REF(rows(rows=600))
    fwd = lambda x=at(0), b=None, res=None, y=at(1): lib.rc_dropout_forward(r, d, x, b, res, y, None)  # noqa: E731
    refused(lib.rc_dropout_forward(None, d, at(0), None, None, at(1), None), "INVALID_ARG", b"null sizes")
    refused(lib.rc_dropout_forward(r, None, at(0), None, None, at(1), None), "INVALID_ARG", b"null dropout")
    refused(fwd(x=None), "INVALID_ARG", b"null x")
    refused(fwd(y=None), "INVALID_ARG", b"null y")
    refused(fwd(x=at(0, shift=1)), "INVALID_ARG", b"multiples of 2 bytes")
    refused(fwd(b=place(3) + 2), "INVALID_ARG", b"bias: not aligned")
    refused(fwd(x=at(0, stride=-64)), "INVALID_ARG", b"row_stride")
    refused(fwd(x=at(0, stride=1 << 46)), "INVALID_ARG", b"row_stride")
    refused(fwd(y=at(1, stride=63)), "INVALID_ARG", b"rows of the output overlap")
    refused(fwd(y=at(1, stride=0)), "INVALID_ARG", b"rows of the output overlap")
    # in place, beside each other in one matrix, into a row of the input, over the bias
    refused(fwd(y=at(0)), "INVALID_ARG", b"y overlaps x")
    refused(fwd(res=at(1)), "INVALID_ARG", b"y overlaps residual")
    refused(fwd(x=at(0, stride=200), y=at(0, stride=200, shift=126)), "INVALID_ARG", b"y overlaps x")
    refused(fwd(x=at(0, stride=200), y=at(0, stride=200, shift=400 * 3 + 274)), "INVALID_ARG", b"y overlaps x")
    refused(fwd(y=at(0, shift=64 * 9 * 2)), "INVALID_ARG", b"y overlaps x")
    refused(fwd(b=place(1)), "INVALID_ARG", b"y overlaps bias")
    bwd = lambda dx=at(1), db=None, acc=0, w=place(5), s=None: lib.rc_dropout_backward(  # noqa: E731
        r, d, at(0), s, dx, db, acc, w, None)
    refused(bwd(dx=None), "INVALID_ARG", b"null dx")
    refused(bwd(acc=2), "INVALID_ARG", b"accumulate")
    large = lambda w: lib.rc_dropout_backward(many, d, at(0), None, at(2), place(4), 0, w, None)  # noqa: E731
    refused(large(None), "INVALID_ARG", b"work")
    refused(large(place(8) + 16), "INVALID_ARG", b"work")
    refused(large(place(4)), "INVALID_ARG", b"overlaps")
    refused(bwd(db=place(3) + 2), "INVALID_ARG", b"dbias")
    refused(bwd(db=place(1)), "INVALID_ARG", b"overlaps")
    refused(bwd(s=at(1)), "INVALID_ARG", b"dx overlaps derivative")


def test_layer_norm_refusals():
    L, lib = lib_or_skip()
    r = REF(rows())

    def fwd(r=r, eps=1e-5, d=None, x=at(0), ib=None, res=None, w=None, b=None, total=None, y=at(1), stats=None):
        return lib.rc_layer_norm_forward(r, eps, d, x, ib, res, w, b, total, y, stats, None)

    def bwd(r=r, dy=at(0), din=None, total=at(2), stats=place(3), w=None, dt=at(4), dx=None, dw=None, db=None, dib=None,
            acc=0, work=place(9)):
        return lib.rc_layer_norm_backward(r, None, dy, din, total, stats, w, dt, dx, dw, db, dib, acc, work, None)

    refused(fwd(r=REF(rows(cols=16392))), "UNSUPPORTED", b"columns")
    refused(bwd(r=REF(rows(cols=16392))), "UNSUPPORTED", b"columns")
    for eps in (-1.0, math.nan, math.inf):
        refused(fwd(eps=eps), "INVALID_ARG", b"eps")
    refused(fwd(total=at(2)), "INVALID_ARG", b"is x")
    refused(fwd(res=at(5)), "INVALID_ARG", b"null total")
    refused(fwd(ib=place(5)), "INVALID_ARG", b"null total")
    refused(fwd(d=REF(drop())), "INVALID_ARG", b"null total")
    refused(fwd(res=at(5), total=at(5)), "INVALID_ARG", b"overlaps")
    refused(fwd(res=at(5), total=at(1)), "INVALID_ARG", b"overlaps")
    refused(fwd(stats=place(1)), "INVALID_ARG", b"overlaps")
    refused(fwd(stats=place(4) + 2), "INVALID_ARG", b"stats")
    refused(fwd(w=place(4) + 2), "INVALID_ARG", b"weight")
    refused(bwd(total=None), "INVALID_ARG", b"null total")
    refused(bwd(stats=None), "INVALID_ARG", b"null stats")
    refused(bwd(dt=None), "INVALID_ARG", b"no gradient")
    refused(bwd(dx=at(4)), "INVALID_ARG", b"overlaps")
    refused(bwd(dt=at(2)), "INVALID_ARG", b"dtotal overlaps total")
    refused(bwd(din=at(4)), "INVALID_ARG", b"overlaps dtotal_in")
    refused(bwd(dw=place(5), db=place(5) + 16), "INVALID_ARG", b"overlaps")
    many = REF(rows(rows=600))
    refused(bwd(r=many, total=at(2), dt=at(6), stats=place(8), dw=place(20), work=None), "INVALID_ARG", b"work")
    refused(bwd(acc=3), "INVALID_ARG", b"accumulate")


BAD_LINEAR = [(dict(dtype=5), "INVALID_ARG", b"dtype"), (dict(bias_dtype=5), "INVALID_ARG", b"bias_dtype"),
              (dict(rows=-1), "INVALID_ARG", b"rows"), (dict(rows=1 << 31), "INVALID_ARG", b"rows"),
              (dict(in_=0), "INVALID_ARG", b"positive"), (dict(out=-8), "INVALID_ARG", b"positive"),
              (dict(activation=4), "INVALID_ARG", b"activation"), (dict(activation=-1), "INVALID_ARG", b"activation"),
              (dict(by_out=2), "INVALID_ARG", b"by_out"), (dict(in_=60), "UNSUPPORTED", b"multiples of 8"),
              (dict(out=4), "UNSUPPORTED", b"multiples of 8"), (dict(in_=32768, out=32768), "UNSUPPORTED", b"2^31"),
              (dict(dtype=0, in_=1 << 20, out=1 << 20), "UNSUPPORTED", b"2^40")]


@pytest.mark.parametrize("kw,st,word", BAD_LINEAR, ids=str)
def test_bad_linear(kw, st, word):
    L, lib = lib_or_skip()
    n = ctypes.c_size_t()
    l = REF(linear(**kw))
    refused(lib.rc_linear_memory(l, REF(n), None, None), st, word)
    refused(lib.rc_linear_forward(l, at(0), at(1), None, None, at(2), None, None, None), st, word)
    refused(lib.rc_linear_backward_input(l, at(0), at(1), None, at(2), None, None), st, word)
    refused(lib.rc_linear_backward_weight(l, at(0), at(1), place(4), None, 0, place(5), None), st, word)


@pytest.mark.parametrize("kw", [dict(in_=(1 << 30) + 8, out=8), dict(in_=8, out=(1 << 30) + 8),
                                dict(in_=8, out=(1 << 31) - 8)], ids=str)
def test_linear_widths_that_32_bits_do_not_count(kw):
    """fp32 weights of 2^33 elements would fit a card; a tile past the last column, or the bytes of a row, would
    not fit the kernels' 32 bits."""
    test_bad_linear(dict(kw, dtype=0), "UNSUPPORTED", b"2^30")
    L, lib = lib_or_skip()
    assert lib.rc_linear_memory(REF(linear(dtype=0, in_=8, out=1 << 30)), None, None, None) == 0


def test_linear_refusals():
    L, lib = lib_or_skip()
    W = place(9)

    def fwd(l=linear(), x=at(0), w=at(1), b=None, res=None, y=at(2), s=None, work=W):
        return lib.rc_linear_forward(REF(l), x, w, b, res, y, s, work, None)

    refused(lib.rc_linear_forward(None, at(0), at(1), None, None, at(2), None, W, None), "INVALID_ARG", b"null linear")
    refused(fwd(x=None), "INVALID_ARG", b"null x")
    refused(fwd(w=None), "INVALID_ARG", b"null weight")
    refused(fwd(y=None), "INVALID_ARG", b"null y")
    refused(fwd(x=at(0, shift=8)), "INVALID_ARG", b"16 bytes")
    refused(fwd(x=at(0, stride=68)), "INVALID_ARG", b"16 bytes")
    refused(fwd(y=at(2, stride=56)), "INVALID_ARG", b"rows of the output overlap")
    refused(fwd(x=at(0, stride=1 << 21)), "UNSUPPORTED", b"row_stride")
    refused(fwd(w=at(1, stride=56)), "INVALID_ARG", b"weight: rows overlap")
    refused(fwd(x=at(0, stride=0)), "INVALID_ARG", b"x: rows overlap")
    refused(fwd(res=at(3, stride=56)), "INVALID_ARG", b"residual: rows overlap")
    refused(fwd(w=at(1, stride=1 << 24)), "UNSUPPORTED", b"weight: spans")
    refused(fwd(s=at(3)), "INVALID_ARG", b"without an activation")
    refused(fwd(y=at(0)), "INVALID_ARG", b"y overlaps x")
    refused(fwd(y=at(1)), "INVALID_ARG", b"y overlaps weight")
    refused(fwd(l=linear(activation=1), s=at(2)), "INVALID_ARG", b"overlaps")
    refused(fwd(b=place(4) + 2), "INVALID_ARG", b"bias")
    n = [ctypes.c_size_t() for _ in range(3)]
    big = linear(rows=64, in_=8192, out=64)     # few tiles over a long reduction: split, with partial sums
    lib.rc_linear_memory(REF(big), *map(REF, n))
    if n[0].value:
        refused(fwd(l=big, x=at(0, 8192), work=None), "INVALID_ARG", b"work")
    refused(lib.rc_linear_backward_input(REF(linear()), at(0), at(1), at(2), at(2), W, None), "INVALID_ARG", b"overlaps")
    wt = lambda dw=place(4), db=None, acc=0, work=W: lib.rc_linear_backward_weight(  # noqa: E731
        REF(linear(rows=40)), at(0), at(1), dw, db, acc, work, None)
    refused(wt(dw=None), "INVALID_ARG", b"null dweight")
    refused(wt(dw=place(4) + 4), "INVALID_ARG", b"16 bytes")
    refused(wt(acc=2), "INVALID_ARG", b"accumulate")
    refused(wt(db=place(5), work=None), "INVALID_ARG", b"work")
    refused(wt(dw=place(0)), "INVALID_ARG", b"dweight overlaps x")
    refused(wt(db=place(4) + 64), "INVALID_ARG", b"overlaps")


def test_python_refusals():
    """What the Python calls refuse before they reach the library (device tensors: the GPU tests)."""
    torch = pytest.importorskip("torch")
    import paper_2405_14009_amd as pkg
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError, match="x must be a device tensor"):
        pkg.dropout_forward(x, pkg.Dropout(0.1, 1))
    with pytest.raises(TypeError, match="dy must be a device tensor"):
        pkg.layer_norm_backward(x, x, x)
    with pytest.raises(TypeError, match="x must be a device tensor"):
        pkg.linear_forward(x, x)
    for kw in (dict(p=-0.1, seed=1), dict(p=1.1, seed=1), dict(p=math.nan, seed=1), dict(p=0.1, seed=-1),
               dict(p=0.1, seed=1 << 64), dict(p=0.1, seed=1, offset=0.5), dict(p=0.1, seed=1, offset=-3)):
        with pytest.raises(ValueError):
            pkg.Dropout(**kw)
    with pytest.raises(TypeError, match="step"):
        pkg.Dropout(0.1, 1, step=torch.zeros(1, dtype=torch.int64))


@pytest.mark.parametrize("shape,stride,want", [
    ((5,), (1,), (1, 5)), ((3, 5), (5, 1), (3, 5)), ((3, 5), (9, 1), (3, 9)), ((2, 3, 5), (27, 9, 1), (6, 9)),
    ((2, 3, 5), (30, 9, 1), None), ((2, 1, 5), (30, 9, 1), (2, 30)), ((1, 3, 5), (7, 9, 1), (3, 9)),
    ((4, 5), (0, 1), (4, 0)), ((2, 4, 5), (0, 0, 1), (8, 0)), ((2, 4, 5), (0, 5, 1), None), ((3, 1), (4, 9), (3, 4)),
    ((3, 5), (1, 3), None), ((0, 5), (5, 1), (0, 5)), ((2, 0, 5), (5, 5, 1), (0, 5)), ((1, 1, 5), (3, 2, 1), (1, 5)),
])
def test_rows_of_a_view(shape, stride, want):
    torch = pytest.importorskip("torch")
    from paper_2405_14009_amd.layer_operators import _rows
    t = torch.zeros(200).as_strided(shape, stride)
    if want is None:
        with pytest.raises(ValueError):
            _rows(t, "t")
    else:
        assert _rows(t, "t") == want


@pytest.mark.parametrize("name,cls", [
    ("gemm_bf16_persist_kernel<5, false, false, true, false>(GemmParams)", "gemm_wgrad"),
    ("gemm_bf16_pp_kernel<128, 2, 3, 4, true, true, 0, false>(GemmParams)", "gemm_dgrad"),
    ("gemm_bf16_pp_kernel<128, 2, 3, 4, true, false, 2, false>(GemmParams)", "gemm_fwd"),
    ("gemm_bf16_pp_kernel<128, 2, 3, 4, false, false, 5, true>(GemmParams)", "gemm_wgrad"),
    ("gemm_bf16_tile_kernel<128, 128, 2, true, true, 7, false>(GemmParams)", "gemm_fwd"),
    ("gemm_bf16_tile_kernel<128, 128, 2, true, false, 4, false>(GemmParams)", "gemm_dgrad"),
    ("gemm_bf16_kernel<256, 256, 8, 1, 64, 2, true, false, 6, false>(GemmParams)", "gemm_other"),
    ("gemm_small_kernel<float, true, false, 7, true, false>(GemmParams)", "gemm_f32"),
    ("_ZN12_GLOBAL__N_117gemm_small_kernelIDF16bLb1ELb0ELi7ELb0ELb0EEEv10GemmParams", "gemm_fwd"),
    ("_ZN12_GLOBAL__N_117gemm_small_kernelIDF16bLb0ELb0ELi5ELb0ELb1EEEv10GemmParams", "gemm_wgrad"),
    ("_ZN12_GLOBAL__N_115splitk_finish_kILi7EDF16bEEv10GemmParams", "gemm_fwd"),
    ("_ZN12_GLOBAL__N_110norm_bwd_kIDF16bLi64ELi1ELb1ELi256EEEv8NormArgsii", "layernorm"),
    ("_ZN12_GLOBAL__N_19dropout_kIDF16bLb0ELb1EEEv11DropoutArgsili", "dropout"),
    ("(anonymous namespace)::rows_finish_k(Finish)", "reduce"),
    ("_ZN12_GLOBAL__N_112few_tokens_kIDF16bLi8EEEv9FewTokens", "gemm_wgrad"),
])
def test_profile_classes(name, cls):
    from paper_2405_14009_amd.profile_summary import kernel_class
    assert kernel_class(name) == cls


@pytest.mark.parametrize("name", [
    "gemm_bf16_kernel<256, 256, 8, 1, 64, 2, true, false, 0, false>(GemmParams)",
    "gemm_bf16_tile_kernel<64, 64, 4, true, false, 0>(GemmParams)",
    "_ZN12_GLOBAL__N_117gemm_small_kernelIDF16bLb1ELb0ELi0ELb0ELb0EEEv10GemmParams",
])
def test_profile_class_of_materialised_attention(name):
    """P V and dS K, forward and backward, are no input gradient of a linear layer."""
    from paper_2405_14009_amd.profile_summary import kernel_class
    assert kernel_class(name) == "gemm_other"


def test_what_autograd_would_lose():
    """The guards that every call goes through: forward calls under autograd, backward calls of a pass with
    create_graph, tangents in either, whatever the grad mode."""
    torch = pytest.importorskip("torch")
    import torch.autograd.forward_ad as dual
    from paper_2405_14009_amd import operators as o
    o._import()
    leaf, plain = torch.ones(2, requires_grad=True), torch.ones(2)
    with pytest.raises(RuntimeError, match="b requires gradients"):
        o._no_graph(plain, "a", leaf, "b")
    with torch.no_grad():
        o._no_graph(plain, "a", leaf, "b", None, "c")
    o._no_second_graph(leaf, "a")   # a call of its own, as a deferred weight gradient is
    for guard in (o._no_graph, o._no_second_graph):
        with dual.dual_level(), torch.no_grad():
            guard(plain, "a", leaf, "b", None, "c", True, "d")
            with pytest.raises(RuntimeError, match="b has a tangent"):
                guard(plain, "a", dual.make_dual(plain, plain), "b")

    class Twice(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            ctx.save_for_backward(x)
            return 2 * x

        @staticmethod
        def backward(ctx, g):
            o._no_second_graph(g, "g", *ctx.saved_tensors, "x")
            return 2 * g

    torch.autograd.grad(Twice.apply(leaf).sum(), leaf)
    with pytest.raises(RuntimeError, match="x requires gradients.*create_graph"):
        torch.autograd.grad(Twice.apply(leaf).sum(), leaf, create_graph=True)
