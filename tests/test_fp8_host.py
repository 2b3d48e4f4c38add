"""The cache in 8 bits and its pages, without a GPU: refusals, and pins of their float64 statement."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from paper_2608_29748_gb300 import build as libbuild
from test_serving_host import Cache, cache

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16, E4M3 = 0, 1, 2
P, I64, F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    L = ctypes.CDLL(libbuild.build())
    L.retrace_last_error.restype = ctypes.c_char_p
    L.retrace_attend_workspace_bytes.restype = ctypes.c_size_t
    return L


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


class Cache8(ctypes.Structure):
    _fields_ = [("pages", Cache), ("k_exp", P), ("v_exp", P), ("exp_page_stride", I64), ("exp_head_stride", I64)]


def cache8(k_exp=16, v_exp=16, exp_page_stride=2, exp_head_stride=1, **kw):
    return Cache8(cache(**dict(dict(dtype=E4M3), **kw)), k_exp, v_exp, exp_page_stride, exp_head_stride)


def append(lib, c=None, q=16, k=16, v=16, out=16, Hq=4, B=2, T=4, lens=16, rope=16, positions=64, rot=128, stride=512, start=None,
           dtype=BF16):
    c = cache8() if c is None else c
    return lib.retrace_kv_append_fp8(P(q), I64(stride), I64(128), Hq, P(k), I64(256), I64(128), P(v), I64(256), I64(128), dtype, P(start),
                                     P(lens), B, T, P(rope), positions, rot, 0, ctypes.byref(c) if c else None, P(out), I64(512), I64(128),
                                     None)


def attend(lib, c=None, q=16, out=16, Hq=4, B=2, T=4, lens=16, scale=0.1, window=0, sinks=0, ws=256, nbytes=1 << 30, stride=512,
           start=None, dtype=BF16):
    c = cache8() if c is None else c
    return lib.retrace_attend_fp8(P(q), I64(stride), I64(128), Hq, dtype, P(start), P(lens), B, T, F(scale), window, sinks, 1,
                                  ctypes.byref(c) if c else None, P(out), I64(512), I64(128), P(ws), ctypes.c_size_t(nbytes), None)


@pytest.mark.parametrize("call", [append, attend])
def test_cache_arguments(lib, call):
    assert call(lib, c=False) == INVALID and b"cache" in lib.retrace_last_error()
    for kw in (dict(dtype=BF16), dict(dtype=F32), dict(kv_heads=0), dict(head_dim=0), dict(page_size=0), dict(num_pages=-1),
               dict(max_pages=-1), dict(head_stride=-1), dict(slot_stride=-1), dict(page_stride=-1), dict(table_stride=3), dict(k=0),
               dict(v=0), dict(page_table=0), dict(kv_heads=3), dict(k_exp=0), dict(v_exp=0), dict(exp_page_stride=-1),
               dict(exp_head_stride=-1)):
        assert call(lib, c=cache8(**kw)) == INVALID, kw
        assert lib.retrace_last_error()
    assert call(lib, c=cache8(head_dim=257)) == UNSUPPORTED
    assert call(lib, c=cache8(max_pages=1 << 28, table_stride=1 << 28)) == UNSUPPORTED
    assert call(lib, c=cache8(max_pages=1, page_size=1 << 24)) == UNSUPPORTED  # a page of 2^31 elements
    assert call(lib, dtype=E4M3) == INVALID and call(lib, dtype=7) == INVALID
    assert call(lib, B=-1) == INVALID and call(lib, T=-1) == INVALID and call(lib, B=0) == INVALID
    assert call(lib, T=5) == INVALID and call(lib, T=(1 << 30) + 2) == UNSUPPORTED
    assert call(lib, lens=0) == INVALID and call(lib, q=16, out=0) == INVALID
    assert call(lib, stride=-1) == INVALID
    assert call(lib, Hq=0) == INVALID and call(lib, Hq=3) == INVALID
    assert call(lib, T=0, q=0, out=0, lens=0) == OK


def test_append_arguments(lib):
    assert append(lib, k=0) == INVALID and append(lib, v=0) == INVALID
    assert append(lib, rot=7) == INVALID and append(lib, rot=130) == INVALID and append(lib, positions=-1) == INVALID


def test_attend_arguments(lib):
    assert attend(lib, q=0) == INVALID
    assert attend(lib, window=-1) == INVALID and attend(lib, sinks=-1) == INVALID
    assert attend(lib, scale=math.nan) == INVALID and attend(lib, scale=math.inf) == INVALID
    assert attend(lib, ws=0) == WORKSPACE and attend(lib, ws=264) == WORKSPACE and attend(lib, nbytes=1000) == WORKSPACE
    assert 0 < lib.retrace_attend_workspace_bytes(4, 2, 64, E4M3) <= lib.retrace_attend_workspace_bytes(4, 2, 128, E4M3) < 1 << 28


def reserve(lib, lens=16, new=16, B=2, page=16, table=16, stride=4, width=4, held=16, free=16, pages=9, counts=16, start=16, slots=16, T=4):
    return lib.retrace_kv_reserve(P(lens), P(new), B, page, P(table), I64(stride), width, P(held), P(free), pages, P(counts), P(start),
                                  P(slots), T, None)


def test_reserve_arguments(lib):
    for kw in (dict(lens=0), dict(new=0), dict(B=-1), dict(page=0), dict(table=0), dict(stride=3), dict(width=-1), dict(held=0),
               dict(free=0), dict(pages=-1), dict(counts=0), dict(start=0), dict(T=-1)):
        assert reserve(lib, **kw) == INVALID, kw
        assert lib.retrace_last_error()
    assert reserve(lib, width=1 << 28, stride=1 << 28) == UNSUPPORTED and reserve(lib, B=(1 << 30) + 1) == UNSUPPORTED


def test_the_other_cache_operators_refuse_eight_bits(lib):
    import test_serving_host as plain

    assert plain.append(lib, c=cache(dtype=E4M3)) == INVALID and plain.attend(lib, c=cache(dtype=E4M3)) == INVALID


def test_binding_refusals(rt):
    k8 = torch.zeros((12, 8, 2, 16)).to(torch.float8_e4m3fn)
    exps, table = torch.zeros((12, 2), dtype=torch.int8), torch.arange(12, dtype=torch.int32).view(3, 4)
    with pytest.raises(TypeError, match="8 bits|float8"):
        rt.KvCacheFp8._code(k8.float())
    with pytest.raises(ValueError, match="CUDA"):
        rt.KvCacheFp8(k8, k8.clone(), table, exps, exps.clone())
    pool = lambda **kw: rt.PagePool(**dict(dict(page_table=table, page_size=8, free_pages=torch.zeros(5, dtype=torch.int32),  # noqa: E731
                                                counts=torch.zeros(2, dtype=torch.int32), held=torch.zeros(3, dtype=torch.int32)), **kw))
    for kw in (dict(held=torch.zeros(4, dtype=torch.int32)), dict(counts=torch.zeros(3, dtype=torch.int32)),
               dict(page_table=table[:1].expand(3, -1)), dict(free_pages=torch.zeros((5, 2), dtype=torch.int32))):
        with pytest.raises(ValueError):
            pool(**kw)
    with pytest.raises(TypeError):
        pool(held=torch.zeros(3))
    with pytest.raises(ValueError, match="CUDA"):
        pool()


def test_every_e4m3_number_and_the_places_between():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    finite = np.unique(codes[np.isfinite(codes)])
    assert finite.size == 253 and finite[-1] == 448  # 256 less two NaN and the second zero
    assert np.array_equal(ref.e4m3(finite), finite)
    mid = ((finite[1:] + finite[:-1]) / 2).astype(np.float32)  # exact; torch takes fp32 to e4m3, to the nearest even
    x = np.concatenate([mid, np.nextafter(mid, np.float32(np.inf)), np.nextafter(mid, np.float32(-np.inf))])
    assert np.array_equal(ref.e4m3(x), torch.tensor(x).to(torch.float8_e4m3fn).double().numpy())
    assert ref.e4m3(1e9) == 448 and ref.e4m3(-np.inf) == -448 and np.isnan(ref.e4m3(np.nan))


def test_exponents_by_hand():
    assert ref.page_exponent([448.0]) == 0 and ref.page_exponent([448.1]) == 1 and ref.page_exponent([-224.0, np.nan]) == -1
    assert ref.page_exponent([0.0]) == -40 and ref.page_exponent([np.inf]) == 40 and ref.page_exponent([1.0]) == -8


def test_append_by_hand():
    """One head of one element; the second append raises the page's exponent."""
    k = np.zeros((2, 4, 1, 1))
    e = np.full((2, 1), 9)
    call = lambda x, codes, exps, at: ref.append_fp8(np.zeros((len(x), 1, 1)), np.reshape(x, (-1, 1, 1)), np.reshape(x, (-1, 1, 1)), codes,  # noqa: E731
                                                     codes, exps, exps, np.array([[1, 0]]), [0, len(x)], [at], None, False)
    _, c, _, x, _ = call([1.0, 7.0], k, e, 0)
    assert x[1, 0] == -6 and c[1, :2, 0, 0].tolist() == [64, 448] and x[0, 0] == 9  # 7 = 448 / 64
    _, c, _, x, _ = call([100.0, -3.0, 5.0], c, x, 2)
    assert x[1, 0] == -2 and c[1, :, 0, 0].tolist() == [4, 28, 384, -12]  # 400 lies between 384 and 416: the even one
    assert x[0, 0] == -6 and c[0, 0, 0, 0] == 320


def test_reserve_by_hand():
    table = np.full((3, 3), -1)
    table, held, free, missing, starts, slots = ref.reserve([0, 0, 0], [5, 0, 9], 4, table, [0, 0, 0], [9, 8, 7, 6, 5], 16)
    assert table.tolist() == [[5, 6, -1], [-1] * 3, [7, 8, 9]] and held == [2, 0, 3] and free == [] and missing == 0
    assert starts == [0, 5, 5, 14] and slots == [20, 21, 22, 23, 24, 28, 29, 30, 31, 32, 33, 34, 35, 36, -1, -1]
    table, held, free, missing, starts, slots = ref.reserve([5, 0, 3], [0, 6, 0], 4, table, held, free, 7)
    assert missing == 2 and table.tolist() == [[5, 6, -1], [-1] * 3, [7, -1, -1]] and held == [2, 0, 1] and free == [9, 8]
    assert starts == [0, 0, 6, 6] and slots == [-1] * 7
    table, held, free, missing, _, slots = ref.reserve([5, 0, 3], [0, 6, 0], 4, table, held, free, 6)
    assert missing == 0 and table[1].tolist() == [8, 9, -1] and slots == [32, 33, 34, 35, 36, 37]
