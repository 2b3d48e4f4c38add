"""retrace_attend_fp8 where scores are far from zero, and where numbers are none.

The scores here are exact in fp32 (few bits each), so the only errors are those of the weights
and of the result: as for any scores, 2^-8 of sum p |v| and of the result in bf16.  In fp32 an
exponent of up to 20 and its exponential have a few 2^-24 of it: 1e-5 of sum p |v|.
"""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from serving import f64
from serving_fp8 import E4M3, Batch8

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def attend(x, rt, scale, **mask):
    ws = rt.AttendWorkspace(x.Hq, x.Hkv, x.D, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start, scale=scale, **mask)
    torch.cuda.synchronize()
    assert ws.check() == 0
    return f64(x.out)


def check(x, rt, scale, **mask):
    got = attend(x, rt, scale, **mask)
    want, spread = ref.attend(f64(x.q), *x.values(), x.table.cpu().numpy(), x.starts, x.cached, scale, **mask)
    tol = 2.0**-8 * (spread + np.abs(want)) if x.dtype == BF16 else 1e-5 * spread
    err = np.abs(got - want)
    assert np.all(err <= tol + 1e-30), (float(err.max()), np.argwhere(err > tol)[:4])


def batch(dtype, lens, D=64):
    """Queries e_0, keys 0 in units of 1."""
    x = Batch8(lens, 2, 1, D, 16, dtype, seed=D)
    x.q.zero_()
    x.q[..., 0] = 1.0
    x.k.copy_(torch.zeros(x.k.shape).to(E4M3))
    x.k_exp.zero_()
    return x


def put(x, b, values, element=0):
    """An element of the keys of sequence b, by position."""
    p = torch.arange(len(values), device="cuda")
    codes = torch.as_tensor(np.asarray(values, np.float32)).to(E4M3)
    assert np.array_equal(f64(codes), np.asarray(values, np.float64))
    x.k[x.table[b, p // x.page].long(), p % x.page, 0, element] = codes.cuda()


ORDERS = {"rising": lambda n, rng: np.arange(n) * 8 // n, "falling": lambda n, rng: np.arange(n)[::-1] * 8 // n,
          "any": lambda n, rng: rng.integers(0, 8, n)}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("exponent", [10, 16, 20, 24, 27, 28, 29, 30, 31, 32, 33, 40, 64, 100, 120])
def test_scores_of_any_size(rt, dtype, order, exponent):
    """Scores from 2^e to 2^(e + 1): those equal to the largest share the weight."""
    rng = np.random.default_rng(exponent)
    for lens in ([(3, 700), (1, 40), (150, 100)], [(1, 40), (2, 500)]):
        for scale in (0.125, -0.25, 2.0**-6 * 1.5):
            x = batch(dtype, lens)
            unit = min(exponent // 2, 40)
            x.q[..., 0] = 2.0 ** (exponent - unit)
            x.k_exp.fill_(unit)
            for b, (n, c) in enumerate(lens):
                put(x, b, 1 + ORDERS[order](n + c, rng) / 8)
            check(x, rt, scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("base", [-(2**18), 2**13, 2**18])
def test_scores_close_together_far_from_zero(rt, dtype, D, base):
    """Scores within a few units of one large number, some rows with small scores beside them, over
    one part and over many."""
    rng = np.random.default_rng(D)
    for lens in ([(3, 700), (150, 100)], [(2, 9000)], [(3, 200)]):
        for small in (False, True):
            x = batch(dtype, lens, D)
            for b, (n, c) in enumerate(lens):
                put(x, b, np.full(n + c, 256.0 if base > 0 else -256.0))
                put(x, b, rng.integers(-8, 9, n + c) / 4, element=1)
            x.q[..., 0] = abs(base) / 256
            if small:
                x.q[::2, 1, 0] = 0.0
            x.q[..., 1] = 2.0
            check(x, rt, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_jumps_between_tiles(rt, dtype):
    """From zero to far and back, in both directions, within a tile and from tile to tile."""
    for far in (2.0**12, 2.0**20, 2.0**31, -(2.0**31)):
        for lens in ([(2, 1000), (140, 500)], [(1, 1001)], [(5, 300), (2, 4000)]):
            x = batch(dtype, lens)
            x.q[..., 0] = abs(far)
            for b, (n, c) in enumerate(lens):
                values = np.zeros(n + c)
                values[(n + c) // 3 : (n + c) // 3 + 70] = np.sign(far)
                values[(n + c) // 2 + 1] = 2 * np.sign(far)
                put(x, b, values)
            check(x, rt, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("by", [0.0, 6.0, 12.0, 14.0, 40.0])
def test_a_maximum_in_each_place(rt, dtype, by):
    """One key above the others by some units, in each tile, first and last of it: the reference moves or does not."""
    for at in (0, 1, 127, 128, 255, 256, 380, 400):
        x = batch(dtype, [(1, 400), (9, 400)])
        x.q[..., 0] = by / 8 if by else 1.0
        for b in range(2):
            values = np.zeros(400 + (1, 9)[b])
            values[at] = 8.0
            put(x, b, values)
        check(x, rt, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", [[(17, 300), (1, 77)], [(1, 300), (2, 40)]])
def test_what_is_not_a_number_stays_with_those_that_see_it(rt, dtype, lens):
    """A NaN in a query: its row.  A NaN in a key that all tokens of a sequence see: that head's rows.  In a value: that
    element of them.  Nothing else changes."""
    want = attend(Batch8(lens, 4, 2, 64, 16, dtype, seed=3), rt, None)
    nan = torch.full((1,), 0x7F, dtype=torch.uint8, device="cuda")[0]
    x = Batch8(lens, 4, 2, 64, 16, dtype, seed=3)
    x.q[0, 1, 5] = float("nan")
    x.q[1, 2, 7] = float("inf")
    expect = want.copy()
    expect[0, 1] = expect[1, 2] = np.nan
    assert np.array_equal(attend(x, rt, None), expect, equal_nan=True)
    for p in (3, 130, 299):
        x = Batch8(lens, 4, 2, 64, 16, dtype, seed=3)
        x.k.view(torch.uint8)[int(x.table[0, p // 16]), p % 16, 1, 9] = nan
        expect = want.copy()
        expect[: lens[0][0], 2:] = np.nan
        assert np.array_equal(attend(x, rt, None), expect, equal_nan=True)
        x = Batch8(lens, 4, 2, 64, 16, dtype, seed=3)
        x.v.view(torch.uint8)[int(x.table[0, p // 16]), p % 16, 0, 9] = nan
        expect = want.copy()
        expect[: lens[0][0], :2, 9] = np.nan
        assert np.array_equal(attend(x, rt, None), expect, equal_nan=True)
