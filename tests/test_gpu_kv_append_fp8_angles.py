"""retrace_kv_append_fp8 with a rotation table that is empty: tokens beyond its positions are cached nowhere."""

import pytest
import torch

from serving_fp8 import Batch8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 33])
@pytest.mark.parametrize("shape", [(0, 16, 2), (0, 0, 2), (6, 0, 2)])
def test_tables_without_positions_or_pairs(dtype, D, shape):
    """Positions 3 to 8 of one sequence: with six positions and nothing to turn, the first three have a place."""
    from paper_2608_29748_gb300 import binding as rt

    x, y = (Batch8([(6, 3)], 4, 2, D, 16, dtype) for _ in range(2))
    rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, x.cache(rt), x.cache_len, torch.zeros(shape, device="cuda"), x.out, q_start=x.q_start)
    there = max(shape[0] - 3, 0)
    if there:  # as without a table, of the tokens that have a position
        start = torch.tensor([0, there], dtype=torch.int32, device="cuda")
        rt.retrace_kv_append_fp8(y.q[:there], y.nk[:there], y.nv[:there], y.cache(rt), y.cache_len, None, y.out[:there], q_start=start)
    for a, b in ((x.k.view(torch.uint8), y.k.view(torch.uint8)), (x.v.view(torch.uint8), y.v.view(torch.uint8)), (x.k_exp, y.k_exp), (x.v_exp, y.v_exp)):
        assert torch.equal(a, b)
    assert torch.equal(x.out[:there], x.q[:there]) and not x.out[there:].any()
