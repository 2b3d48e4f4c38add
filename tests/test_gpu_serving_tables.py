"""Page tables of unusual layouts: refused, or read as they are.

Tolerance, in fp32: a score of 64 products has an error of about 8 * 2^-24 of their
absolute sum (20 to 40 here), so a weight one of 2e-5 of it.
"""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from serving import Batch, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def test_tables_with_equal_rows(rt):
    """Three sequences over the same pages: refused as an expanded row, right as rows of their own."""
    x = Batch([(2, 60)] * 3, 4, 2, 64, 16, torch.float32, seed=1)
    shared = x.table[:1].expand(3, -1)
    with pytest.raises(ValueError, match="page_table"):
        rt.KvCache(x.k, x.v, shared)
    x.table = shared.contiguous()
    ws = rt.AttendWorkspace(4, 2, 64, x.dtype)
    rt.retrace_attend(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start)
    want, spread = ref.attend(f64(x.q), f64(x.k), f64(x.v), x.table.cpu().numpy(), x.starts, x.cached, 0.125)
    assert np.all(np.abs(f64(x.out) - want) <= 2e-5 * spread) and ws.check() == 0


def test_tables_with_rows_apart(rt):
    """A part of a wider table, and a single row of any stride."""
    for lens in ([(2, 60), (1, 31), (5, 0)], [(3, 40)]):
        x = Batch(lens, 4, 2, 64, 16, torch.float32, seed=2)
        wide = torch.full((len(lens), x.table.shape[1] + 3), 10**6, dtype=torch.int32, device="cuda")
        wide[:, 1:-2] = x.table
        tables = [wide[:, 1:-2]]
        if len(lens) == 1:
            tables.append(x.table.as_strided(x.table.shape, (0, 1)))
        for table in tables:
            x.table = table
            ws = rt.AttendWorkspace(4, 2, 64, x.dtype)
            rt.retrace_attend(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start)
            want, spread = ref.attend(f64(x.q), f64(x.k), f64(x.v), x.table.cpu().numpy(), x.starts, x.cached, 0.125)
            assert np.all(np.abs(f64(x.out) - want) <= 2e-5 * spread) and ws.check() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_windows_and_sinks_past_32_bits(rt, dtype):
    """More than any sequence is long: everything is seen, as with 2^31 - 1."""
    x = Batch([(2, 300), (9, 40)], 4, 2, 64, 16, dtype, seed=3)
    ws, cache = rt.AttendWorkspace(4, 2, 64, dtype), x.cache(rt)
    call = lambda **mask: (rt.retrace_attend(x.q, cache, x.cache_len, x.out, ws, q_start=x.q_start, **mask), x.out.clone())[1]  # noqa: E731
    want = call()
    for far in (2**31 - 1, 2**31, 2**32, 2**32 + 7, 2**63 - 1):
        assert torch.equal(call(window=far), want)
        assert torch.equal(call(window=5, sinks=far), want)
    with pytest.raises(rt.RetraceError):
        call(window=-(2**33))
    with pytest.raises(rt.RetraceError):
        call(window=5, sinks=-1)


def test_queries_without_a_place_to_go(rt):
    """Refused by name, before anything is enqueued."""
    x = Batch([(2, 20)], 4, 2, 64, 16, torch.float32, seed=4)
    before = x.k.clone()
    with pytest.raises(ValueError, match="q_out"):
        rt.retrace_kv_append(x.q, x.nk, x.nv, x.cache(rt), x.cache_len, None)
    torch.cuda.synchronize()
    assert torch.equal(x.k, before)
