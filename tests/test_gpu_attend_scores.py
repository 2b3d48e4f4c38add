"""retrace_attend where scores are far from zero.

The scores here are exact in fp32 (few bits each), so the only errors are those of the weights
and of the result.  In bf16 the weights are rounded before the product with v (at
most 2^-8 each, so 2^-8 of sum p |v|) and the result once (at most 2^-8 of it).  In fp32 an
exponent of up to 20 and its exponential have a few 2^-24 of it: 1e-5 of sum p |v|.
"""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from serving import Batch, f64

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def check(x, rt, scale, **mask):
    ws = rt.AttendWorkspace(x.Hq, x.Hkv, x.D, x.dtype)
    rt.retrace_attend(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start, scale=scale, **mask)
    torch.cuda.synchronize()
    assert ws.check() == 0
    want, spread = ref.attend(f64(x.q), f64(x.k), f64(x.v), x.table.cpu().numpy(), x.starts, x.cached, scale, **mask)
    tol = 2.0**-8 * (spread + np.abs(want)) if x.dtype == BF16 else 1e-5 * spread
    err = np.abs(f64(x.out) - want)
    assert np.all(err <= tol + 1e-30), (float(err.max()), np.argwhere(err > tol)[:4])


def batch(dtype, lens, D=64):
    """Queries e_0, keys 0."""
    x = Batch(lens, 2, 1, D, 16, dtype, seed=D)
    x.q.zero_()
    x.q[..., 0] = 1.0
    x.k.zero_()
    return x


def put(x, b, values):
    """The first element of the keys of sequence b, by position."""
    p = torch.arange(len(values), device="cuda")
    x.k[x.table[b, p // x.page].long(), p % x.page, 0, 0] = torch.as_tensor(values, dtype=x.dtype, device="cuda")


ORDERS = {"rising": lambda n, rng: np.arange(n) * 128 // n, "falling": lambda n, rng: np.arange(n)[::-1] * 128 // n,
          "any": lambda n, rng: rng.integers(0, 128, n)}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("exponent", [10, 16, 20, 24, 27, 28, 29, 30, 31, 32, 33, 40, 64, 100, 120])
def test_scores_of_any_size(rt, dtype, order, exponent):
    """Scores from 2^e to 2^(e + 1): those equal to the largest share the weight."""
    rng = np.random.default_rng(exponent)
    lens = [(3, 700), (1, 40), (150, 100)]
    for scale in (0.125, -0.25, 2.0**-6 * 1.5):
        x = batch(dtype, lens)
        x.q[..., 0] = 2.0 ** (exponent // 2)
        for b, (n, c) in enumerate(lens):
            put(x, b, 2.0 ** (exponent - exponent // 2) * (1 + ORDERS[order](n + c, rng) / 128))
        check(x, rt, scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("base", [-(2**18), 2**13, 2**18])
def test_scores_close_together_far_from_zero(rt, dtype, D, base):
    """Scores within a few units of one large number, some rows with small scores beside them, over
    one part and over many."""
    rng = np.random.default_rng(D)
    for lens in ([(3, 700), (150, 100)], [(2, 9000)]):
        x = batch(dtype, lens, D)
        for b, (n, c) in enumerate(lens):
            put(x, b, np.full(n + c, base / 64))
        x.k[..., 1] = torch.tensor(rng.integers(-16, 17, x.k.shape[:3]) / 4, dtype=dtype, device="cuda")
        x.q[..., 0] = 64.0
        x.q[::2, 1, 0] = 0.0
        x.q[..., 1] = 1.0
        check(x, rt, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_jumps_between_tiles(rt, dtype):
    """From zero to far and back, in both directions, within a tile and from tile to tile."""
    for far in (2.0**12, 2.0**20, 2.0**31, -(2.0**31)):
        x = batch(dtype, [(2, 1000), (140, 500)])
        for b, n in ((0, 1002), (1, 640)):
            values = np.zeros(n)
            values[n // 3 : n // 3 + 70] = far
            values[n // 2 + 1] = 2 * far
            put(x, b, values)
        check(x, rt, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("low, high", [(3.5, 11.75), (3.5, 11.0), (3.484375, 10.3125), (3.59375, 9.75), (2.234375, 10.5), (5.15625, 10.625)])
def test_weights_are_rounded_once(rt, dtype, low, high):
    """A maximum that appears in the second half of a tile rescales the weights of the first
    half, which are rounded already.  These scores lose most if that rounds them again."""
    n, c = 140, 244
    x = Batch([(n, c)], 1, 1, 64, 16, dtype)
    x.q.zero_()
    x.q[..., 0] = 1.0
    x.k.zero_()
    x.v.zero_()
    values = np.full(n + c, -120.0)
    values[:128], values[128:192], values[197] = 0.0, low, high
    put(x, 0, values)
    p = torch.arange(128, 192, device="cuda")
    x.v[x.table[0, p // 16].long(), p % 16, 0] = (1 + torch.arange(64, device="cuda") / 64).to(dtype)
    check(x, rt, 1.0, causal=False)
    x.v[x.table[0, p // 16].long(), p % 16, 0] = (1 + 1 / 128 + torch.arange(64, device="cuda") / 64).to(dtype)
    check(x, rt, 1.0, causal=False)
