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
    # with a bias: a sum per bucket of each block of 128 queries
    assert memory(**size, buckets=32, max_distance=128)[2] >= up(4 * rows) + 4 * batch * heads * blocks * 32
    # with sinks in a window: shares of 128 rows of dk and dv from each chunk of queries
    if seq > 512:
        chunks = -(-seq // 512)
        got = memory(**size, window=40, sinks=4, buckets=32, max_distance=128)[2]
        assert got >= up(4 * rows) + 4 * batch * heads * blocks * 32 + 4 * batch * kv * chunks * 2 * 128 * d
