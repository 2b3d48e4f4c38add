"""retrace_attend_fp8 with queries and scales near the end of fp32, where the scores are zero all the same.

All keys of a row weigh the same then, and the result is the mean of the values: within 2^-8 of the mean of |v| and of
itself in bf16, 2e-5 of the mean of |v| in fp32.
"""

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
@pytest.mark.parametrize("lens", [(1, 300), (4, 100), (17, 700), (2, 9000)])
@pytest.mark.parametrize("size, scale", [(2.0**110, 0.125), (2.0**127, 0.125), (2.0**127, -512.0), (1.0, 2.9e38), (2.0**-20, 2.9e38), (2.0**30, 2.9e38)])
@pytest.mark.parametrize("exponent", [40, 0, -40])
def test_scores_of_zero(rt, dtype, lens, size, scale, exponent):
    """The queries' one element meets keys of zero, in the largest unit and others; the second token's query is small."""
    x = Batch8([lens], 4, 2, 64, 16, dtype, seed=5)
    x.q.zero_()
    x.q[..., 0] = size
    x.q[1::2, :, 0] = 2.0**-100
    x.k_exp.fill_(exponent)
    x.k[..., 0] = torch.zeros((), device="cuda").to(E4M3)
    ws = rt.AttendWorkspace(4, 2, 64, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start, causal=False, scale=scale)
    assert ws.check() == 0
    n, c = lens
    _, v = x.values()
    table = x.table[0].cpu().numpy()
    rows = v[table[table >= 0]].reshape(-1, 2, 64)[: n + c]
    want, mean = rows.mean(0), np.abs(rows).mean(0)
    tol = 2.0**-8 * (mean + np.abs(want)) if dtype == BF16 else 2e-5 * mean
    for h in range(4):
        assert np.all(np.abs(f64(x.out)[:, h] - want[h // 2]) <= tol[h // 2])
