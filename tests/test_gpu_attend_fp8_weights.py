"""retrace_attend_fp8 where a few keys have nearly all of a row's weight.

Scores here are exact but for fp32's last places.  Tolerance, element by element: that of any bf16 call, 2^-8 of
sum p |v| and of the result, and for each visible key the 2^-24 of the row's largest weight (at most one) that its own
weight may be off by: 2^-24 of sum |v|, which counts where the keys with most of the weight have values of zero.
"""

import math

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


def check(x, rt, scale, **mask):
    ws = rt.AttendWorkspace(x.Hq, x.Hkv, x.D, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start, scale=scale, **mask)
    assert ws.check() == 0
    want, spread = ref.attend(f64(x.q), *x.values(), x.table.cpu().numpy(), x.starts, x.cached, scale, **mask)
    _, mean = ref.attend(0 * f64(x.q), *x.values(), x.table.cpu().numpy(), x.starts, x.cached, scale, **mask)
    most = max(c + n for n, c in zip(x.new, x.cached))
    keys = min(most, mask["window"] + mask["sinks"]) if mask["window"] else most
    tol = 2.0**-8 * (spread + np.abs(want)) + 2.0**-24 * keys * mean if x.dtype == BF16 else 2e-5 * spread
    err = np.abs(f64(x.out) - want)
    assert np.all(err <= tol + 1e-30), (float((err / (tol + 1e-30)).max()), np.argwhere(~(err <= tol))[:4])


def flat(dtype, lens, D, high, Hq=2, seed=1):
    """Keys of zero but the first one of each sequence, whose score is `high` (at scale 1); values of one sign, none in
    half of the first key's elements."""
    x = Batch8(lens, Hq, 1, D, 16, dtype, seed=seed, exps=(-6, -5))
    x.q.zero_()
    x.q[..., 0] = 1.0
    x.k.view(torch.uint8).zero_()
    x.v.copy_(x.v.float().abs().to(E4M3))
    for b in range(len(lens)):
        page = int(x.table[b, 0])
        x.k[page, 0, 0, 0] = high * 64
        x.v[page, 0, 0, ::2] = 0.0
    return x


LENS = {"tokens": [(1, 9000), (1, 3000), (1, 700)] * 60, "a token": [(1, 9000)], "blocks": [(9, 2000), (9, 900)], "a prompt": [(300, 1500)]}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("window, sinks", [(0, 0), (1024, 1), (1000, 4), (8192, 1)])
@pytest.mark.parametrize("powers", [12, 16, 18, 20, 22])
def test_a_sink_above_flat_scores(rt, dtype, lens, window, sinks, powers):
    """One key has 2^powers times the weight of each other one: sinks are kept because they have most of it."""
    lens = LENS[lens] if window else LENS[lens][:9]
    high = math.ceil(powers * math.log(2) * 4) / 4  # few bits
    check(flat(dtype, lens, 64, high if high < 7 else 7.0), rt, high / min(high, 7.0), window=window, sinks=sinks)


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("window, sinks", [(1024, 1), (1024, 4), (8000, 1)])
def test_a_sink_above_random_scores(rt, lens, window, sinks):
    """The sinks have most of the weight and small values."""
    x = Batch8(LENS[lens][:30], 4, 2, 128, 16, BF16, seed=3, exps=(-6, -5))
    x.q.copy_((x.q * 4).round() / 4)
    x.k.copy_((x.k.float() / 8).round().mul(8).clamp(-448, 448).to(E4M3))
    x.q[..., 0] = 8.0
    x.k[..., 0] = torch.zeros((), device="cuda").to(E4M3)
    for b in range(len(x.cached)):
        page = int(x.table[b, 0])
        x.k[page, :sinks, :, 0] = 448.0  # 8 * 7 * scale: 15 above the others, which spread by 3
        x.v[page, :sinks] = (x.v[page, :sinks].float() / 64).to(E4M3)
    check(x, rt, 128**-0.5 * 3, window=window, sinks=sinks)
