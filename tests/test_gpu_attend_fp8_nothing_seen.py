"""retrace_attend_fp8: a row that sees no key is zero, whatever its query is."""

import numpy as np
import pytest
import torch

from serving import f64
from serving_fp8 import E4M3, Batch8

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", [[(1, 300)], [(3, 40), (17, 700)], [(150, 20)], [(2, 9000)]])
@pytest.mark.parametrize("number", [float("nan"), float("inf"), -float("inf")])
def test_queries_that_are_no_numbers_meet_no_keys(rt, dtype, lens, number):
    """The pages of every position are missing: nothing is visible."""
    x = Batch8(lens, 4, 2, 64, 16, dtype, seed=3)
    x.table.fill_(-1)
    x.q[::2, 1, 5] = number
    ws = rt.AttendWorkspace(4, 2, 64, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start)
    assert ws.check() == 0 and not f64(x.out).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_some_pages_are_missing(rt, dtype):
    """Only the rows that meet a key are numbers no more: the first tokens' pages are gone, later ones' are there."""
    x = Batch8([(40, 0)], 4, 2, 64, 8, dtype, seed=4)
    x.table[0, :2] = -1
    x.q[:, 1, 5] = float("nan")
    ws = rt.AttendWorkspace(4, 2, 64, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start)
    assert ws.check() == 0
    got = f64(x.out)
    assert not got[:16].any() and np.isnan(got[16:, 1]).all() and np.isfinite(got[:, [0, 2, 3]]).all()
