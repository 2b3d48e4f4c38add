"""retrace_kv_append_fp8's rotation, bit for bit: each product is rounded to fp32 before the sum, whatever the layout.

What is stored follows from that in one rounding (bf16 queries, e4m3 codes in the page's unit), so a token's codes do not
depend on the strides and types that decide which code path it takes.
"""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from serving import f64, rope_table
from serving_fp8 import Batch8

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def turned(x, cs, interleaved):
    """x [n, heads, D] by the angles of its n tokens, in fp32."""
    x, rot = x.float().cpu().numpy().copy(), 2 * cs.shape[1]
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    v, w = x[..., a], x[..., b]
    x[..., a], x[..., b] = v * c - w * s, w * c + v * s
    return x


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D, rot, pad", [(128, 128, 0), (64, 32, 0), (96, 48, 0), (64, 64, 1), (40, 6, 0), (256, 256, 0)])
def test_products_are_rounded(dtype, interleaved, D, rot, pad):
    from paper_2608_29748_gb300 import binding as rt

    n = 301
    x = Batch8([(n, 0), (n, 16)], 8, 4, D, 16, dtype, seed=D + rot, pad=pad)
    rope = rope_table(400, rot)
    rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, x.cache(rt), x.cache_len, rope, x.out, q_start=x.q_start, interleaved=interleaved)
    pos = np.concatenate([np.arange(n), 16 + np.arange(n)])
    cs = rope.cpu().numpy()[pos]
    want = torch.from_numpy(turned(x.q, cs, interleaved)).to(dtype)
    assert torch.equal(x.out.cpu(), want)
    k, codes, exps, table = turned(x.nk, cs, interleaved), f64(x.k), x.k_exp.cpu().numpy(), x.table.cpu().numpy()
    for b in range(2):
        at = np.flatnonzero(np.arange(2 * n) // n == b)
        for p0 in range(0, 320, 16):
            of = at[(pos[at] >= p0) & (pos[at] < p0 + 16)]
            if of.size:
                page = table[b, p0 // 16]
                for h in range(4):
                    e = ref.page_exponent(k[of, h])
                    assert exps[page, h] == e
                    assert np.array_equal(codes[page, pos[of] - p0, h], ref.e4m3(k[of, h].astype(np.float64) * 2.0**-e))
