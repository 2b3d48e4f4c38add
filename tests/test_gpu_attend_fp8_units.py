"""retrace_attend_fp8 over pages whose values are in very different units.

Tolerance: 2^-8 of sum p |v| and of the result in bf16, 2e-5 of sum p |v| in fp32, element by element: so what pages of
small units add counts wherever pages of large units hold zeros or little.
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


def check(x, rt, ws=None, **mask):
    ws = ws or rt.AttendWorkspace(x.Hq, x.Hkv, x.D, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start, **mask)
    assert ws.check() == 0
    want, spread = ref.attend(f64(x.q), *x.values(), x.table.cpu().numpy(), x.starts, x.cached, x.D**-0.5, **mask)
    tol, err = 2.0**-8 * (spread + np.abs(want)) if x.dtype == BF16 else 2e-5 * spread, np.abs(f64(x.out) - want)
    assert np.all(err <= tol + 1e-30), (float((err / (tol + 1e-30)).max()), np.argwhere(~(err <= tol + 1e-30))[:4])


LENS = {"a token": [(1, 700)], "tokens": [(1, 300), (1, 1200), (1, 40)] * 20, "blocks": [(17, 700), (5, 90)], "a prompt": [(150, 200)],
        "a long context": [(2, 9000)], "a block over one": [(18, 5000)]}


def pages_of(x, which):
    """Pages of each sequence by their places in the table."""
    return torch.cat([row[row >= 0][which] for row in x.table]).long()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("D, page", [(64, 16), (128, 8), (128, 128), (80, 48)])
@pytest.mark.parametrize("unit", [-40, -11, 4, 40])
@pytest.mark.parametrize("which", [slice(0, 1), slice(-1, None), slice(1, None, 3)])
def test_pages_of_another_unit(rt, dtype, lens, D, page, unit, which):
    """Some pages in a unit far from the others', with zeros, the least numbers, and a few elements of any size."""
    if dtype == F32 and D != 64:
        return
    x = Batch8(LENS[lens], 8, 2, D, page, dtype, seed=unit + 50, exps=(-7, -5))
    pages = pages_of(x, which)
    x.v_exp[pages] = unit
    v = x.v.float()
    v[pages, :, :, : D // 2] = 0.0  # elements that the page has nothing of
    v[pages, :, :, D // 2 : D - 3] *= 2.0**-9
    x.v.copy_(v.to(E4M3))
    check(x, rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("span", [3, 8, 16, 40])
def test_units_all_over(rt, dtype, lens, D, span):
    """Every page and head has its own unit; each page has elements that are zero."""
    x = Batch8(LENS[lens], 4, 2, D, 16, dtype, seed=span, exps=(-7, -5))
    x.v_exp = torch.randint(-span, span + 1, x.v_exp.shape, generator=torch.Generator().manual_seed(D), dtype=torch.int8).cuda()
    v, some = x.v.float(), torch.rand((x.v.shape[0], 1, 2, D), generator=torch.Generator().manual_seed(span)).cuda() < 0.5
    x.v.copy_(torch.where(some, v, 0.0).to(E4M3))
    check(x, rt)
    check(x, rt, window=150, sinks=3)
    x.out.fill_(77.0)
    check(x, rt, causal=False)


@pytest.mark.parametrize("Hq, Hkv, n", [(4, 4, 1), (14, 1, 1), (32, 1, 1), (72, 1, 1), (3, 1, 12), (4, 1, 17), (1, 1, 72)])
def test_rows_of_a_unit(rt, Hq, Hkv, n):
    """One huge page, in the first tile or a later one, for each number of rows."""
    for place in (0, 9, 30):
        x = Batch8([(n, 700)] * 3, Hq, Hkv, 64, 16, BF16, seed=n, exps=(-7, -5))
        pages = pages_of(x, slice(place, place + 1))
        x.v_exp[pages] = 30
        x.v.view(torch.uint8)[pages] = 0
        x.v[pages, 3, :, 7] = 100.0
        check(x, rt)


@pytest.mark.parametrize("lens", ["tokens", "blocks", "a prompt", "a long context"])
@pytest.mark.parametrize("unit", [-30, -9, -3, 0, 25])
def test_a_sink_in_another_unit(rt, lens, unit):
    """The first page, with values of zero, has most of the weight: the others' weights are off by at most 2^-18 of it."""
    x = Batch8(LENS[lens], 2, 1, 64, 16, BF16, seed=1, exps=(-6, -5))
    x.q.zero_()
    x.q[..., 0] = 1.0
    x.k.view(torch.uint8).zero_()
    x.v.copy_(x.v.float().abs().to(E4M3))
    pages = pages_of(x, slice(0, 1))
    x.k[pages, 0, 0, 0] = 448.0
    x.v[pages] = torch.zeros((), device="cuda").to(E4M3)
    x.v_exp[pages] = unit
    for powers in (6.0, 12.0):
        ws, scale = rt.AttendWorkspace(2, 1, 64, E4M3), powers * float(np.log(2)) / 7
        rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start, scale=scale)
        table = x.table.cpu().numpy()
        want, spread = ref.attend(f64(x.q), *x.values(), table, x.starts, x.cached, scale)
        _, mean = ref.attend(0 * f64(x.q), *x.values(), table, x.starts, x.cached, scale)
        tol = 2.0**-8 * (spread + np.abs(want)) + 2.0**-18 * max(c + n for n, c in LENS[lens]) * mean
        assert np.all(np.abs(f64(x.out) - want) <= tol)


@pytest.mark.parametrize("rise", [1, 5, 30])
def test_units_rise_and_fall_with_the_position(rt, rise):
    for up in (1, -1):
        x = Batch8([(5, 1500), (1, 900)], 4, 2, 64, 16, BF16, seed=rise)
        for row in x.table:
            row = row[row >= 0].long()
            step = torch.arange(row.numel(), device="cuda") * rise // 8
            x.v_exp[row] = (up * (step - int(step.max()) // 2)).clamp(-40, 40).to(torch.int8)[:, None]
        some = torch.rand(x.v.shape, generator=torch.Generator().manual_seed(5)).cuda() < 0.3
        x.v.copy_(torch.where(some, x.v.float(), 0.0).to(E4M3))
        check(x, rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [1e4, 3e12, float("inf")])
def test_a_rejected_token_of_any_size(rt, dtype, size):
    """A block whose last token has huge values is appended, and rejected; the next block goes over it.  The page
    keeps its unit: its own small values are lost, nothing else is."""
    x = Batch8([(4, 300), (4, 37)], 4, 2, 64, 16, dtype, seed=21, exps=(-7, -5))
    x.nv[3] = x.nv[7] = size
    rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, x.cache(rt), x.cache_len, None, x.out, q_start=x.q_start)
    x.nv.normal_()
    rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, x.cache(rt), x.cache_len, None, x.out, q_start=x.q_start)
    assert int(x.v_exp[int(x.table[0, 18]), 0]) > 4
    check(x, rt)
