"""retrace_attend against its float64 statement.

Tolerance.  In bf16 (8 significant bits) the weights are rounded before the product
with v (at most 2^-8 each, so 2^-8 of sum p |v|) and the result once (at most 2^-8 of
it); the fp32 scores and exponentials add far less.  In fp32 a score of up to
256 products has an error of about sqrt(256) * 2^-24 of their absolute sum (20
to 40 here), which is the relative error of a weight: 2e-5 of sum p |v|.
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


def close(got, want, spread, dtype):
    tol = 2.0**-8 * (spread + np.abs(want)) if dtype == BF16 else 2e-5 * spread
    err = np.abs(got - want)
    assert np.all(err <= tol + 1e-30), (float(err.max()), float((err / (tol + 1e-30)).max()), np.argwhere(err > tol)[:4])


def check(x, rt, ws=None, q_start=True, scale=None, clean=True, **mask):
    ws = ws or rt.AttendWorkspace(x.Hq, x.Hkv, x.D, x.dtype)
    rt.retrace_attend(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start if q_start else None, scale=scale, **mask)
    torch.cuda.synchronize()
    assert ws.check() == 0
    if clean:
        want, spread = ref.attend(f64(x.q), f64(x.k), f64(x.v), x.table.cpu().numpy(), x.starts, x.cached,
                                  x.D**-0.5 if scale is None else scale, **mask)
        close(f64(x.out), want, spread, x.dtype)
    return f64(x.out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128, 80, 8, 256, 33])
def test_head_sizes(rt, dtype, D):
    check(Batch([(3, 5), (1, 0), (9, 300)], 4, 2, D, 16, dtype, seed=D), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (3, 1), (5, 5), (14, 2), (8, 1), (16, 2), (40, 1), (17, 1), (130, 1)])
def test_head_groups(rt, dtype, Hq, Hkv):
    check(Batch([(2, 140), (5, 3), (1, 77)], Hq, Hkv, 64, 16, dtype, seed=Hq), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n, c", [(1, 0), (1, 1), (1, 127), (1, 128), (2, 127), (17, 111), (33, 500), (130, 0), (200, 70), (1, 4000)])
def test_lengths(rt, dtype, n, c):
    """One sequence: row and key counts around the tiles' edges."""
    check(Batch([(n, c)], 4, 2, 64, 16, dtype, seed=n + c), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window, sinks", [(1, 0), (5, 0), (64, 4), (100, 1), (128, 130), (200, 300), (4096, 4)])
@pytest.mark.parametrize("causal", [True, False])
def test_window_and_sinks(rt, dtype, window, sinks, causal):
    check(Batch([(1, 700), (17, 333), (3, 0), (40, 129)], 4, 2, 64, 16, dtype, seed=window), rt, window=window, sinks=sinks,
          causal=causal)


@pytest.mark.parametrize("page", [1, 7, 8, 24, 48, 64, 256, 1000])
def test_page_sizes(rt, page):
    check(Batch([(5, 300), (1, 129)], 4, 2, 128, page, BF16, seed=page), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ragged_batch(rt, dtype):
    """No tokens, one, a block, a prompt; with and without a context."""
    lens = [(0, 9), (1, 0), (0, 0), (150, 0), (17, 260)] + [(1 + b % 3, 13 * b) for b in range(30)] + [(0, 5)]
    check(Batch(lens, 4, 2, 64, 16, dtype, seed=1), rt)


def test_many_sequences(rt):
    """More sequences than a CTA has threads."""
    check(Batch([((b * 7) % 3, b % 40) for b in range(900)], 2, 1, 64, 16, BF16, seed=2), rt)


def test_blocks_without_a_list(rt):
    check(Batch([(4, c) for c in (0, 90, 260)], 8, 2, 128, 16, BF16), rt, q_start=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_long_context_is_split(rt, dtype, D):
    """One head over a context that many CTAs share: their parts are joined."""
    check(Batch([(17, 9000)], 4, 1, D, 64, dtype, seed=D), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompt_over_several_tiles(rt, dtype):
    check(Batch([(700, 45), (333, 0)], 2, 1, 64, 16, dtype, seed=7), rt)
    check(Batch([(300, 600)], 2, 1, 128, 16, dtype, seed=8), rt, window=150, sinks=3)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_see_nothing(rt, dtype):
    """Negative lengths, contexts without pages: zeros."""
    x = Batch([(5, -3), (2, -2), (3, 20)], 4, 2, 64, 8, dtype, seed=4)
    x.table[2] = -1
    x.cached[2] = 20
    got = check(x, rt)
    assert not got[:3].any() and not got[5:].any() and got[3:5].any()
    y = Batch([(2, 30)], 4, 2, 64, 8, dtype)
    y.table[0, 1:] = 10**6  # the window's pages are gone, no sinks
    assert not check(y, rt, window=5).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_without_a_place_are_not_seen(rt, dtype):
    x = Batch([(4, 300), (20, 100)], 4, 2, 64, 8, dtype, seed=6)
    x.table[0, 5] = -1
    x.table[0, 17] = 2**30
    x.table[1, 0] = -2
    x.table[1, 15] = x.k.shape[0]
    check(x, rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("page", [8, 48])
def test_unseen_places_do_not_matter(rt, dtype, bad, page):
    """Slots never written and pages before the window hold anything."""
    lens = [(3, 250), (1, 77), (17, 400)]
    x, y = (Batch(lens, 4, 2, 64, page, dtype, seed=9) for _ in range(2))
    seen = torch.zeros(x.k.shape[:2], dtype=torch.bool)
    table = x.table.cpu()
    for b, (n, c) in enumerate(lens):
        for p in range(c + n):
            if p < 2 or p > c - 100:
                seen[int(table[b, p // page]), p % page] = True
    y.k[~seen.cuda()] = bad
    y.v[~seen.cuda()] = bad
    want = check(x, rt, window=100, sinks=2)
    got = check(y, rt, window=100, sinks=2, clean=False)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("spread", [1e-3, 30.0])
def test_flat_and_sharp_scores(rt, dtype, spread):
    x = Batch([(5, 600)], 4, 2, 64, 16, dtype, seed=11)
    x.q.mul_(spread)
    if dtype == F32 and spread > 1:  # scores of several hundred: their fp32 rounding is the weights' error
        x.q.copy_(x.q.bfloat16())
        x.k.copy_((x.k * 4).round() / 4)
    check(x, rt)


def test_rising_scores(rt):
    """The maximum grows with every tile: what is accumulated is rescaled each time."""
    x = Batch([(2, 1500)], 2, 1, 64, 16, BF16, seed=12)
    x.q.fill_(1.0)
    for p in range(1502):
        x.k[int(x.table[0, p // 16]), p % 16] = p / 64
    check(x, rt)


def test_scale(rt):
    x = Batch([(3, 200)], 4, 2, 64, 16, F32, seed=13)
    check(x, rt, scale=0.5)
    check(x, rt, scale=-0.25)
    check(x, rt, scale=0.0)
    check(Batch([(3, 200)], 4, 2, 64, 16, BF16, seed=13), rt, scale=-0.25)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_unaligned_and_strided(rt, dtype):
    check(Batch([(3, 200), (6, 2)], 4, 2, 64, 8, dtype, pad=1), rt)
    x = Batch([(3, 200), (6, 2)], 4, 2, 64, 8, dtype, pad=8)
    x.out = torch.zeros((9, 4, 80), dtype=dtype, device="cuda")[..., :64]
    check(x, rt)


def test_one_workspace_serves_every_batch(rt):
    ws = rt.AttendWorkspace(4, 2, 64, BF16)
    for seed, lens in enumerate([[(1, 3000)], [(130, 0), (40, 500)], [(2, 50)] * 70, [(1, 3000)]]):
        check(Batch(lens, 4, 2, 64, 16, BF16, seed=seed), rt, ws=ws)


def test_the_same_bits_again_on_another_stream_and_in_a_graph(rt):
    x = Batch([(17, 900), (3, 40)], 4, 2, 128, 16, BF16, seed=14)
    ws, cache = rt.AttendWorkspace(4, 2, 128, BF16), x.cache(rt)
    call = lambda: rt.retrace_attend(x.q, cache, x.cache_len, x.out, ws, q_start=x.q_start)  # noqa: E731
    call()
    want = x.out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x.out.zero_()
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(x.out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    x.out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x.out, want) and ws.check() == 0


def test_offsets_past_32_bits(rt):
    pages = 2**31 // (16 * 2 * 64) + 40
    k = torch.zeros((pages, 16, 2, 64), dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    x = Batch([(3, 200)], 4, 2, 64, 16, BF16, seed=15)
    want = check(x, rt)
    table = pages - 1 - x.table
    table[x.table < 0] = -1
    used = x.table[x.table >= 0].long()
    k[pages - 1 - used], v[pages - 1 - used] = x.k[used], x.v[used]
    x.k, x.v, x.table = k, v, table.to(torch.int32)
    assert np.array_equal(check(x, rt, clean=False), want)
