"""retrace_attend_fp8 against its float64 statement.

Tolerance.  The keys and values are what the cache stands for, exactly.  With bf16 queries the
result is rounded once (at most 2^-8 of it) and the weights lose at most 2^-8 of sum p |v|: half of
that by a rounding to 9 bits (2^-9 of each weight), the rest by weights below 2^-17 of the row's largest,
each off by at most 2^-26 of that one (2^-19 where the first keys are few).  The scores' errors add
far less.  In fp32 a score of up to 256 products has an error of about sqrt(256) * 2^-24 of
their absolute sum (20 to 40 here), which is the relative error of a weight: 2e-5 of sum p |v|.
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


def close(got, want, spread, dtype):
    tol = 2.0**-8 * (spread + np.abs(want)) if dtype == BF16 else 2e-5 * spread
    err = np.abs(got - want)
    assert np.all(err <= tol + 1e-30), (float(err.max()), float((err / (tol + 1e-30)).max()), np.argwhere(~(err <= tol))[:4])


def check(x, rt, ws=None, q_start=True, scale=None, clean=True, **mask):
    ws = ws or rt.AttendWorkspace(x.Hq, x.Hkv, x.D, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start if q_start else None, scale=scale, **mask)
    torch.cuda.synchronize()
    assert ws.check() == 0
    if clean:
        want, spread = ref.attend(f64(x.q), *x.values(), x.table.cpu().numpy(), x.starts, x.cached, x.D**-0.5 if scale is None else scale,
                                  **mask)
        close(f64(x.out), want, spread, x.dtype)
    return f64(x.out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128, 80, 96, 16, 8, 256, 33])
def test_head_sizes(rt, dtype, D):
    check(Batch8([(3, 5), (1, 0), (9, 300)], 4, 2, D, 16, dtype, seed=D), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (3, 1), (5, 5), (14, 2), (8, 1), (16, 2), (40, 1), (17, 1), (73, 1), (130, 1)])
def test_head_groups(rt, dtype, Hq, Hkv):
    check(Batch8([(2, 140), (5, 3), (1, 77)], Hq, Hkv, 64, 16, dtype, seed=Hq), rt)


@pytest.mark.parametrize("rows", [1, 4, 5, 8, 9, 16, 17, 31, 33, 47, 48, 49, 71, 72, 73, 80, 100, 144, 150])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_a_sequence(rt, rows, D):
    check(Batch8([(rows, 333)], 1, 1, D, 16, BF16, seed=rows), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n, c", [(1, 0), (1, 1), (1, 127), (1, 128), (2, 127), (17, 111), (33, 500), (130, 0), (200, 70), (1, 4000)])
def test_lengths(rt, dtype, n, c):
    """One sequence: row and key counts around the tiles' edges."""
    check(Batch8([(n, c)], 4, 2, 64, 16, dtype, seed=n + c), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window, sinks", [(1, 0), (5, 0), (64, 4), (100, 1), (128, 130), (200, 300), (4096, 4)])
@pytest.mark.parametrize("causal", [True, False])
def test_window_and_sinks(rt, dtype, window, sinks, causal):
    check(Batch8([(1, 700), (17, 333), (3, 0), (40, 129)], 4, 2, 64, 16, dtype, seed=window), rt, window=window, sinks=sinks,
          causal=causal)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [1, 7, 8, 24, 48, 64, 256, 1000])
def test_page_sizes(rt, page, D):
    check(Batch8([(5, 300), (1, 129)], 4, 2, D, page, BF16, seed=page), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ragged_batch(rt, dtype):
    """No tokens, one, a block, a prompt; with and without a context."""
    lens = [(0, 9), (1, 0), (0, 0), (150, 0), (17, 260)] + [(1 + b % 3, 13 * b) for b in range(30)] + [(0, 5)]
    check(Batch8(lens, 4, 2, 64, 16, dtype, seed=1), rt)


def test_many_sequences(rt):
    """More sequences than a CTA has threads."""
    check(Batch8([((b * 7) % 3, b % 40) for b in range(900)], 2, 1, 64, 16, BF16, seed=2), rt)


@pytest.mark.parametrize("Hq, Hkv", [(8, 2), (2, 2), (16, 1)])
def test_blocks_without_a_list(rt, Hq, Hkv):
    check(Batch8([(4, c) for c in (0, 90, 260)], Hq, Hkv, 128, 16, BF16), rt, q_start=False)
    check(Batch8([(1, 60 * b) for b in range(40)], Hq, Hkv, 64, 16, BF16), rt, q_start=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 17, 40])
def test_long_context_is_split(rt, dtype, D, n):
    """One head over a context that many CTAs share: their parts are joined."""
    check(Batch8([(n, 9000)], 4, 1, D, 64, dtype, seed=D), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompt_over_several_tiles(rt, dtype):
    check(Batch8([(700, 45), (333, 0)], 2, 1, 64, 16, dtype, seed=7), rt)
    check(Batch8([(300, 600)], 2, 1, 128, 16, dtype, seed=8), rt, window=150, sinks=3)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_see_nothing(rt, dtype):
    """Negative lengths, contexts without pages: zeros."""
    x = Batch8([(5, -3), (2, -2), (3, 20)], 4, 2, 64, 8, dtype, seed=4)
    x.table[2] = -1
    x.cached[2] = 20
    got = check(x, rt)
    assert not got[:3].any() and not got[5:].any() and got[3:5].any()
    y = Batch8([(2, 30)], 4, 2, 64, 8, dtype)
    y.table[0, 1:] = 10**6  # the window's pages are gone, no sinks
    assert not check(y, rt, window=5).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_without_a_place_are_not_seen(rt, dtype):
    x = Batch8([(4, 300), (20, 100)], 4, 2, 64, 8, dtype, seed=6)
    x.table[0, 5] = -1
    x.table[0, 17] = 2**30
    x.table[1, 0] = -2
    x.table[1, 15] = x.k.shape[0]
    check(x, rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bits", [0x7F, 0xFF, 0x7E])
@pytest.mark.parametrize("page", [8, 48])
def test_unseen_places_do_not_matter(rt, dtype, D, bits, page):
    """Slots never written and pages before the window hold anything (NaN, 448), and pages that nobody sees any exponent."""
    lens = [(3, 250), (1, 77), (17, 400)]
    x, y = (Batch8(lens, 4, 2, D, page, dtype, seed=9) for _ in range(2))
    seen = torch.zeros(x.k.shape[:2], dtype=torch.bool)
    table = x.table.cpu()
    for b, (n, c) in enumerate(lens):
        for p in range(c + n):
            if p < 2 or p > c - 100:
                seen[int(table[b, p // page]), p % page] = True
    for t in (y.k, y.v):
        t.view(torch.uint8)[~seen.cuda()] = bits
    for e in (y.k_exp, y.v_exp):
        e[~seen.any(1).cuda()] = 127
    want = check(x, rt, window=100, sinks=2)
    got = check(y, rt, window=100, sinks=2, clean=False)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("exps", [(-40, 41), (-128, 128), (-12, 5)])
def test_exponents_of_any_size(rt, dtype, exps):
    """Pages and heads in very different units: values, and (times a scale that keeps scores finite) keys."""
    x = Batch8([(3, 700), (17, 90), (1, 20)], 4, 2, 64, 16, dtype, seed=10)
    g = torch.Generator().manual_seed(11)
    x.v_exp = torch.randint(*exps, x.v_exp.shape, generator=g, dtype=torch.int16).to(torch.int8).cuda()
    check(x, rt)
    # keys whose scores are exact: one power of two in each, few bits in a query
    x.k_exp = torch.randint(-6, -1, x.k_exp.shape, generator=g, dtype=torch.int16).to(torch.int8).cuda()
    check(x, rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_keys_at_the_ends_of_the_exponents(rt, dtype):
    x = Batch8([(5, 300)], 2, 1, 64, 16, dtype, seed=12)
    x.q.copy_((x.q * 4).round() / 4)
    x.k.copy_((x.k.float() / 32).round().mul(32).clamp(-448, 448).to(E4M3))
    for e in (40, -40, 127, -128):
        x.k_exp.fill_(e)
        check(x, rt, scale=2.0 ** (-12 - min(max(e, -40), 40)))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_zero_pages(rt, dtype):
    """Values of zero in the least unit next to others: they weigh in the sum all the same."""
    x = Batch8([(3, 260), (2, 30)], 4, 2, 64, 16, dtype, seed=13)
    pages = x.table[0, ::2][x.table[0, ::2] >= 0].long()
    x.v.view(torch.uint8)[pages] = 0
    x.v_exp[pages] = -40
    check(x, rt)
    x.v.view(torch.uint8)[:] = 0
    x.v_exp[:] = -40
    assert not check(x, rt).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("spread", [1e-3, 30.0])
def test_flat_and_sharp_scores(rt, dtype, spread):
    x = Batch8([(5, 600)], 4, 2, 64, 16, dtype, seed=11)
    x.q.mul_(spread)
    if spread > 1:  # scores of several hundred: few bits, so that fp32 has them exactly
        x.q.copy_(x.q.bfloat16().float().div(8).round().mul(8).to(dtype))
        x.k.copy_(x.k.float().div(16).round().mul(16).to(E4M3))
    check(x, rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_queries_of_any_size(rt, dtype):
    """Rows of very different sizes, elements of one row far apart, rows of zeros."""
    x = Batch8([(12, 200)], 2, 1, 64, 16, dtype, seed=14)
    x.q.copy_(x.q.bfloat16())
    for i, f in enumerate([1e-30, 1e-20, 1e-3, 0.0, 1.0, 3.0]):
        x.q[i] *= f
    x.q[6, :, ::2] *= 2.0**-8
    x.q[7, :, 1:] *= 2.0**-12
    x.q[8, :, 5:] = 0
    check(x, rt)
    y = Batch8([(2, 200)], 2, 1, 64, 16, dtype, seed=15)
    y.q.copy_((y.q * 2).round() * 2.0**90)
    check(y, rt, scale=2.0**-96)


def test_one_key_above_a_flat_row(rt):
    """A sink that holds half of the weight, the other half spread over thousands of keys."""
    x = Batch8([(4, 20000)], 2, 1, 64, 64, BF16, seed=16)
    k = x.k.float()
    k[..., 0] = 0.0
    first = int(x.table[0, 0])
    k[first, 0] = 0.0
    k[first, 0, :, 0] = 256.0
    x.k.copy_(k.to(E4M3))
    x.k_exp.fill_(-8)
    x.q.fill_(0.0)
    x.q[:, :, 0] = 80.0  # a score of 80 / 8 = 10, among zeros
    check(x, rt)
    x.v.copy_(x.v.float().abs().to(E4M3))  # nothing cancels: a weight's bias would show
    check(x, rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 2, 30])
def test_rising_scores(rt, dtype, n):
    """The maximum grows with every tile: what is accumulated is rescaled each time."""
    x = Batch8([(n, 1500)], 2, 1, 64, 16, dtype, seed=12)
    x.q.fill_(1.0)
    for p in range(1500 + n):
        x.k[int(x.table[0, p // 16]), p % 16] = float(p // 32)
    x.k_exp.fill_(1)
    check(x, rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scale(rt, dtype):
    x = Batch8([(3, 200)], 4, 2, 64, 16, dtype, seed=13)
    check(x, rt, scale=0.5)
    check(x, rt, scale=-0.25)
    check(x, rt, scale=0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad", [1, 8, 16])
def test_unaligned_and_strided(rt, dtype, pad):
    x = Batch8([(3, 200), (6, 2)], 4, 2, 64, 8, dtype, pad=pad)
    packed = torch.stack([x.k_exp, x.v_exp], 1)
    x.k_exp, x.v_exp = packed[:, 0], packed[:, 1]
    check(x, rt)
    x.out = torch.zeros((9, 4, 80), dtype=dtype, device="cuda")[..., :64]
    check(x, rt)


def test_heads_before_slots(rt):
    """A cache laid out [pages, heads, slots, head_dim]."""
    x = Batch8([(3, 200), (18, 40)], 8, 2, 128, 16, BF16, seed=17)
    for name in ("k", "v"):
        t = getattr(x, name)
        apart = torch.empty((t.shape[0], 2, 16, 128), dtype=torch.uint8, device="cuda").view(E4M3).transpose(1, 2)
        apart.copy_(t)
        setattr(x, name, apart)
    check(x, rt)


def test_rows_behind_the_last_sequence(rt):
    x = Batch8([(3, 50), (17, 300)], 4, 2, 64, 8, BF16, seed=18)
    x.q_start = torch.tensor([0, 3, 12], dtype=torch.int32).cuda()
    ws = rt.AttendWorkspace(4, 2, 64, E4M3)
    rt.retrace_attend_fp8(x.q, x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start)
    want, spread = ref.attend(f64(x.q), *x.values(), x.table.cpu().numpy(), [0, 3, 12], x.cached, 64**-0.5)
    close(f64(x.out)[:12], want[:12], spread[:12], BF16)
    assert bool((x.out[12:] == 77.0).all())


def test_one_workspace_serves_every_batch(rt):
    ws = rt.AttendWorkspace(4, 2, 64, E4M3)
    for seed, lens in enumerate([[(1, 3000)], [(130, 0), (40, 500)], [(2, 50)] * 70, [(1, 3000)]]):
        for dtype in (BF16, F32):
            check(Batch8(lens, 4, 2, 64, 16, dtype, seed=seed), rt, ws=ws)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", [[(17, 900), (3, 40)], [(1, 5000)], [(1, 100)] * 90])
def test_the_same_bits_again_on_another_stream_and_in_a_graph(rt, dtype, lens):
    x = Batch8(lens, 4, 2, 128, 16, dtype, seed=14)
    ws, cache = rt.AttendWorkspace(4, 2, 128, E4M3), x.cache(rt)
    call = lambda: rt.retrace_attend_fp8(x.q, cache, x.cache_len, x.out, ws, q_start=x.q_start)  # noqa: E731
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
    pages = 2**32 // (16 * 2 * 64) + 40
    k = torch.zeros((pages, 16, 2, 64), dtype=torch.uint8, device="cuda").view(E4M3)
    v = torch.zeros((pages, 16, 2, 64), dtype=torch.uint8, device="cuda").view(E4M3)
    x = Batch8([(3, 200)], 4, 2, 64, 16, BF16, seed=15)
    want = check(x, rt)
    table = pages - 1 - x.table
    table[x.table < 0] = -1
    used = x.table[x.table >= 0].long()
    exps = [torch.zeros((pages, 2), dtype=torch.int8, device="cuda") for _ in range(2)]
    for big, small in ((k.view(torch.uint8), x.k.view(torch.uint8)), (v.view(torch.uint8), x.v.view(torch.uint8)), (exps[0], x.k_exp), (exps[1], x.v_exp)):
        big[pages - 1 - used] = small[used]
    x.k, x.v, x.table, (x.k_exp, x.v_exp) = k, v, table.to(torch.int32), exps
    assert np.array_equal(check(x, rt, clean=False), want)


def test_refusals(rt):
    x = Batch8([(3, 20)], 4, 2, 64, 8, BF16)
    ws, cache = rt.AttendWorkspace(4, 2, 64, E4M3), x.cache(rt)
    plain = rt.KvCache(torch.zeros(x.k.shape, dtype=BF16, device="cuda"), torch.zeros(x.k.shape, dtype=BF16, device="cuda"), x.table)
    with pytest.raises(TypeError):
        rt.retrace_attend_fp8(x.q, plain, x.cache_len, x.out, ws)
    with pytest.raises(TypeError):
        rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, plain, x.cache_len, None, x.out)
    with pytest.raises(ValueError):
        rt.retrace_attend(x.q, cache, x.cache_len, x.out, ws)
    with pytest.raises(ValueError):
        rt.retrace_attend_fp8(x.q, cache, x.cache_len, x.out.float(), ws)
    with pytest.raises(ValueError):
        rt.retrace_kv_append_fp8(x.q, x.nk, x.nv.float(), cache, x.cache_len, None, x.out)
    with pytest.raises(TypeError):
        rt.retrace_attend_fp8(x.q.half(), cache, x.cache_len, x.out.half(), ws)
    with pytest.raises(TypeError):
        rt.KvCacheFp8(plain.k, plain.v, x.table, x.k_exp, x.v_exp)
    for bad in (x.k_exp[:, :1], x.k_exp.float(), x.k_exp[:1].expand(x.k_exp.shape)):
        with pytest.raises(ValueError):
            rt.KvCacheFp8(x.k, x.v, x.table, bad, bad)
