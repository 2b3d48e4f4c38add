"""retrace_attend_fp8 with queries of different sizes in one call: a row's result is its own.

Tolerance.  A row's largest element is 256, its others are whole multiples of 2^-9 below a half, 8 bits
each: in the row's own unit the two e4m3 parts hold them exactly (4 bits, and what is left, a multiple of
2^-9 of at most 4 bits).  The largest element meets keys of zero.  So scores are off by fp32's sums alone, some
2^-20 here, and the result by what any bf16 call's is: 2^-8 of sum p |v| and of the result.
"""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from serving import f64
from serving_fp8 import E4M3, Batch8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq, n", [(2, 2), (4, 3), (4, 8), (4, 17), (1, 71)])
@pytest.mark.parametrize("distance", [1, 3, 6, 9])
def test_larger_rows_beside_it_do_not_matter(rt, D, Hq, n, distance):
    x = Batch8([(n, 700)], Hq, 1, D, 16, torch.bfloat16, seed=D + n, exps=(-6, -5))
    x.k[..., 0] = torch.zeros((), device="cuda").to(E4M3)
    g = torch.Generator().manual_seed(n)
    x.q.copy_(torch.randint(-255, 256, x.q.shape, generator=g) * 2.0**-9)
    x.q[..., 0] = 256.0
    rows = x.q.reshape(n * Hq, D).clone()
    rows[::2] *= 2.0**distance
    x.q.copy_(rows.view(n, Hq, D))
    scale = D**-0.5 * 8
    ws = rt.AttendWorkspace(Hq, 1, D, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start, scale=scale)
    assert ws.check() == 0
    want, spread = ref.attend(f64(x.q), *x.values(), x.table.cpu().numpy(), x.starts, x.cached, scale)
    tol, err = 2.0**-8 * (spread + np.abs(want)), np.abs(f64(x.out) - want)
    assert np.all(err <= tol), float((err / tol).max())
