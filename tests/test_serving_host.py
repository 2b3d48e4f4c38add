"""The operators around a round, without a GPU: their refusals, and pins of their float64 statement."""

import ctypes
import math

import numpy as np
import pytest

from oracle import serving_oracle as ref
from paper_2608_29748_gb300 import build as libbuild

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16 = 0, 1
P, I64, F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    L = ctypes.CDLL(libbuild.build())
    L.retrace_last_error.restype = ctypes.c_char_p
    L.retrace_attend_workspace_bytes.restype = ctypes.c_size_t
    return L


class Cache(ctypes.Structure):
    _fields_ = [("k", P), ("v", P), ("page_stride", I64), ("slot_stride", I64), ("head_stride", I64), ("num_pages", ctypes.c_int),
                ("page_size", ctypes.c_int), ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("page_table", P),
                ("table_stride", I64), ("max_pages", ctypes.c_int), ("dtype", ctypes.c_int)]


def cache(**kw):
    c = dict(k=16, v=16, page_stride=4096, slot_stride=256, head_stride=128, num_pages=9, page_size=16, kv_heads=2, head_dim=128,
             page_table=16, table_stride=4, max_pages=4, dtype=BF16)
    c.update(kw)
    return Cache(**c)


def append(lib, c=None, q=16, k=16, v=16, out=16, Hq=4, B=2, T=4, lens=16, rope=16, positions=64, rot=128, stride=512, start=None):
    c = cache() if c is None else c
    return lib.retrace_kv_append(P(q), I64(stride), I64(128), Hq, P(k), I64(256), I64(128), P(v), I64(256), I64(128), P(start), P(lens),
                                 B, T, P(rope), positions, rot, 0, ctypes.byref(c) if c else None, P(out), I64(512), I64(128), None)


def attend(lib, c=None, q=16, out=16, Hq=4, B=2, T=4, lens=16, scale=0.1, window=0, sinks=0, ws=256, nbytes=1 << 30, stride=512,
           start=None):
    c = cache() if c is None else c
    return lib.retrace_attend(P(q), I64(stride), I64(128), Hq, P(start), P(lens), B, T, F(scale), window, sinks, 1,
                              ctypes.byref(c) if c else None, P(out), I64(512), I64(128), P(ws), ctypes.c_size_t(nbytes), None)


def sample(lib, logits=16, dtype=BF16, B=2, R=3, V=10, rs=10, bs=30, u=16, tokens=16):
    return lib.retrace_sample(P(logits), dtype, B, R, V, I64(rs), I64(bs), P(u), None, None, None, None, P(tokens), None, None)


@pytest.mark.parametrize("call", [append, attend])
def test_cache_arguments(lib, call):
    assert call(lib, c=False) == INVALID and b"cache" in lib.retrace_last_error()
    for kw in (dict(dtype=5), dict(kv_heads=0), dict(head_dim=0), dict(page_size=0), dict(num_pages=-1), dict(max_pages=-1),
               dict(head_stride=-1), dict(slot_stride=-1), dict(page_stride=-1), dict(table_stride=3), dict(k=0), dict(v=0),
               dict(page_table=0), dict(kv_heads=3)):
        assert call(lib, c=cache(**kw)) == INVALID, kw
        assert lib.retrace_last_error()
    assert call(lib, c=cache(head_dim=257)) == UNSUPPORTED
    assert call(lib, c=cache(max_pages=1 << 28, table_stride=1 << 28)) == UNSUPPORTED
    assert call(lib, B=-1) == INVALID and call(lib, T=-1) == INVALID and call(lib, B=0) == INVALID
    assert call(lib, T=5) == INVALID  # no q_start, 5 tokens of 2 sequences
    assert call(lib, T=(1 << 30) + 2) == UNSUPPORTED
    assert call(lib, lens=0) == INVALID and call(lib, q=16, out=0) == INVALID
    assert call(lib, stride=-1) == INVALID
    assert call(lib, Hq=0) == INVALID and call(lib, Hq=3) == INVALID
    assert call(lib, T=0, q=0, out=0, lens=0) == OK  # nothing to do


def test_append_arguments(lib):
    assert append(lib, k=0) == INVALID and append(lib, v=0) == INVALID
    assert append(lib, rot=7) == INVALID and append(lib, rot=130) == INVALID and append(lib, rot=-2) == INVALID
    assert append(lib, positions=-1) == INVALID


def test_attend_arguments(lib):
    assert attend(lib, q=0) == INVALID
    assert attend(lib, window=-1) == INVALID and attend(lib, sinks=-1) == INVALID
    assert attend(lib, scale=math.nan) == INVALID and attend(lib, scale=math.inf) == INVALID
    assert attend(lib, ws=0) == WORKSPACE and attend(lib, ws=264) == WORKSPACE and attend(lib, nbytes=1000) == WORKSPACE
    size = lib.retrace_attend_workspace_bytes
    assert size(4, 3, 128, BF16) == 0 and size(4, 2, 257, BF16) == 0 and size(0, 1, 64, BF16) == 0 and size(4, 2, 64, 9) == 0
    assert 0 < size(4, 2, 64, BF16) <= size(4, 2, 128, BF16) < 1 << 28


def test_sample_arguments(lib):
    assert sample(lib, logits=0) == INVALID and sample(lib, u=0) == INVALID and sample(lib, tokens=0) == INVALID
    assert sample(lib, dtype=3) == INVALID and sample(lib, V=0) == INVALID and sample(lib, B=-1) == INVALID
    assert sample(lib, rs=-1) == INVALID and sample(lib, V=(1 << 24) + 1) == UNSUPPORTED
    assert sample(lib, B=1 << 20, R=1 << 20) == UNSUPPORTED
    assert sample(lib, B=0, logits=0) == OK and sample(lib, R=0, u=0) == OK


def test_rotation_by_complex_numbers():
    rng = np.random.default_rng(0)
    x, t = rng.normal(size=10), rng.normal(size=3)
    cs = np.stack([np.cos(t), np.sin(t)], -1)
    for interleaved in (False, True):
        i = np.arange(0, 6, 2) if interleaved else np.arange(3)
        j = i + 1 if interleaved else i + 3
        z = (x[i] + 1j * x[j]) * np.exp(1j * t)
        y = ref.rotate(x, cs, interleaved)
        assert np.allclose(y[i], z.real) and np.allclose(y[j], z.imag) and np.array_equal(y[6:], x[6:])


def test_attention_by_hand():
    """One head of size one: values are weighted averages that can be written down."""
    k = np.zeros((2, 2, 1, 1))
    v = np.array([1.0, 2.0, 3.0, 4.0]).reshape(2, 2, 1, 1)
    table, q = np.array([[1, 0]]), np.ones((2, 1, 1))
    out = lambda **m: ref.attend(q, k, v, table, [0, 2], [1], 1.0, **m)[0].ravel()  # noqa: E731  (values by position: 3 4 1 2)
    assert np.allclose(out(), [3.5, 8 / 3])
    assert np.allclose(out(causal=False), [8 / 3, 8 / 3])
    assert np.allclose(out(window=1), [4, 1]) and np.allclose(out(window=1, sinks=1), [3.5, 2])
    k[0, 0] = math.log(2)  # position 2 weighs twice
    assert np.allclose(out(), [3.5, 9 / 4])
    assert np.allclose(ref.attend(q, k, v, np.array([[5, 0]]), [0, 2], [1], 1.0)[0].ravel(), [0, 1])


def test_sampling_by_hand():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    kept = lambda *s: sorted(ref.kept_tokens(x, *s)[0].tolist())  # noqa: E731
    assert kept(1, 0, 1, 0) == [0, 1, 2, 3] and kept(1, 2, 1, 0) == [1, 3] and kept(1, 0, 0.71, 0) == [1, 2, 3]
    assert kept(1, 0, 0.69, 0) == [1, 3] and kept(1, 0, 1, 0.49) == [1, 2, 3] and kept(0, 0, 1, 0) == [1] and kept(1, 3, 0.5, 0) == [1, 3]
    assert ref.sample(x, 0.55, 1, 2, 1, 0)[0] == 1 and ref.sample(x, 0.6, 1, 2, 1, 0)[0] == 3
    assert np.isclose(ref.sample(x, 0.6, 1, 2, 1, 0)[1], 3 / 7)
    assert ref.sample([-np.inf, np.nan], 0.5, 1, 0, 1, 0) == (-1, 0.0)
