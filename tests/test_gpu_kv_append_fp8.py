"""retrace_kv_append_fp8 against its float64 statement.

Tolerance.  A rotated element in fp32 is off by at most 3 * 2^-24 of |x c| + |y s| (two products, a
sum); a query then has one rounding to bf16 (2^-8 of it).  An element of the cache is the e4m3
number nearest to it, so it is as near to the exact element as the nearest number is, but
for twice that error.  Exponents, copied elements and every place that the call does
not own are exact.
"""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from serving import f64, rope_table
from serving_fp8 import E4M3, Batch8

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def check(x, rt, rot, interleaved, positions, q_start=True, query=True):
    rope = rope_table(positions, rot) if rot is not None else None
    before = f64(x.k), f64(x.v), x.k_exp.cpu().numpy(), x.v_exp.cpu().numpy(), x.table.cpu().numpy()
    rt.retrace_kv_append_fp8(x.q if query else None, x.nk, x.nv, x.cache(rt), x.cache_len, rope, x.out if query else None,
                             q_start=x.q_start if q_start else None, interleaved=interleaved)
    torch.cuda.synchronize()
    state = lambda rounded: ref.append_fp8(f64(x.q), f64(x.nk), f64(x.nv), *before, x.starts, x.cached,  # noqa: E731
                                           None if rope is None else f64(rope), interleaved, rounded)
    want, raw = state(True), state(False)
    finite = [t[torch.isfinite(t)].abs().max().item() if t.numel() else 0.0 for t in (x.q, x.nk, x.nv)]
    off = 3 * 2.0**-24 * 2 * max(finite)
    if query:
        unit = 2.0**-8 if x.dtype == BF16 else 0.0
        assert np.all(np.abs(f64(x.out) - want[0]) <= unit * np.abs(want[0]) + off * (1 + unit))
    assert np.array_equal(x.k_exp.cpu().numpy(), want[3]) and np.array_equal(x.v_exp.cpu().numpy(), want[4])
    for codes, w, r, e, turned in ((x.k, want[1], raw[1], want[3], rot), (x.v, want[2], raw[2], want[4], None)):
        got = f64(codes)
        assert np.array_equal(np.isnan(got), np.isnan(w))
        near = 0.0 if not turned else 2 * off * np.exp2(-np.clip(e.astype(float), -40, 40))[:, None, :, None]
        bad = ~np.isnan(w) & ~(np.abs(got - np.clip(r, -448, 448)) <= np.abs(w - np.clip(r, -448, 448)) + near)
        assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], w[bad][:4], r[bad][:4])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D, rot", [(128, 128), (64, 32), (96, 48), (80, 80), (256, 64), (40, 6), (33, 32), (16, 0)])
def test_heads_and_rotations(rt, dtype, interleaved, D, rot):
    check(Batch8([(3, 5), (1, 0), (7, 30)], 6, 2, D, 8, dtype, seed=D + rot), rt, rot, interleaved, 64)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_few_sequences_among_many(rt, dtype):
    """Long runs of sequences without tokens; rows behind the last sequence."""
    lens = [(0, 3)] * 300 + [(5, 14), (0, 0), (2, 7)] + [(0, 9)] * 400 + [(20, 1)] + [(1, 5)] * 40 + [(0, 2)] * 333
    check(Batch8(lens, 4, 2, 64, 16, dtype, seed=5), rt, 32, False, 64)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [8, 16, 24, 33, 64, 80, 128, 200, 256])
def test_without_a_rotation(rt, dtype, D):
    """Copied as they are, the bits of what is no number among them; zeros where a token has no position."""
    x = Batch8([(3, 5), (1, 0), (7, 30), (20, 0), (2, -1)], 6, 2, D, 8, dtype, seed=D)
    bits = torch.int16 if dtype == BF16 else torch.int32
    x.q.view(bits)[3, 1, D // 2] = 0x7FA5 if dtype == BF16 else 0x7FA12345
    x.q[4, 2, 0] = -0.0
    q = x.q.clone()
    q[31] = 0  # at position -1
    x.q[3, 1, D // 2], save = 0, x.q.view(bits)[3, 1, D // 2].clone()
    y_k, y_v, e_k, e_v = (t.clone() for t in (x.k, x.v, x.k_exp, x.v_exp))
    check(x, rt, None, False, 0)
    x.k.copy_(y_k), x.v.copy_(y_v), x.k_exp.copy_(e_k), x.v_exp.copy_(e_v)
    x.q.view(bits)[3, 1, D // 2] = save
    rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, x.cache(rt), x.cache_len, None, x.out, q_start=x.q_start)
    assert torch.equal(x.out.view(bits), q.view(bits))


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (7, 1), (32, 8), (71, 71)])
def test_head_counts(rt, Hq, Hkv):
    check(Batch8([(5, 9), (2, 0)], Hq, Hkv, 64, 16, BF16, seed=Hq), rt, 64, False, 32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [1, 3, 16, 128, 300])
def test_page_sizes(rt, dtype, page):
    """Pages of one slot, pages that a sequence begins and ends in, pages larger than what a warp keeps."""
    check(Batch8([(2, 1), (333, 0), (70, 65), (1, page - 1), (1, page)], 2, 2, 64, page, dtype, seed=page), rt, 64, False, 400)


def test_ragged_sequences(rt):
    lens = [(0, 4), (1, 0), (0, 0), (17, 40)] + [(b % 3, b) for b in range(40)] + [(0, 9)]
    check(Batch8(lens, 4, 2, 64, 16, BF16, seed=1), rt, 64, False, 64)


def test_many_sequences(rt):
    check(Batch8([((b * 7) % 4, b % 11) for b in range(1200)], 2, 1, 16, 4, F32, seed=3), rt, 16, False, 16)


def test_blocks_without_a_list(rt):
    check(Batch8([(4, c) for c in (0, 3, 12)], 4, 2, 64, 8, BF16), rt, 64, False, 32, q_start=False)


def test_keys_and_values_only(rt):
    x = Batch8([(4, 0), (4, 3)], 4, 2, 64, 8, BF16)
    check(x, rt, 64, False, 32, query=False)
    assert bool((x.out == 77.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_rotation(rt, dtype):
    """Bit-exact throughout."""
    x = Batch8([(4, 0), (4, 3), (30, 9)], 4, 2, 64, 8, dtype)
    check(x, rt, None, False, 0)
    assert torch.equal(x.out, x.q)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad", [1, 4, 8, 16])
def test_unaligned_and_strided(rt, dtype, pad):
    x = Batch8([(3, 5), (6, 2)], 4, 2, 64, 8, dtype, pad=pad)
    packed = torch.stack([x.k_exp, x.v_exp], 1)  # exponents side by side
    x.k_exp, x.v_exp = packed[:, 0], packed[:, 1]
    check(x, rt, 64, False, 32)


@pytest.mark.parametrize("D", [64, 33])
def test_larger_tokens_raise_a_pages_exponent(rt, D):
    """What the page holds is rounded to the new unit, again and again; smaller tokens leave it."""
    x = Batch8([(1, 0)], 2, 2, D, 8, F32, seed=4, exps=(20, 21))
    for p, size in enumerate([1e-3, 3.0, 0.5, 700.0, 1e5, 2.0, 3e9, 1.0]):
        x.cached = [p]
        x.cache_len.fill_(p)
        x.nk.normal_().mul_(size)
        x.nv.normal_().mul_(1 / size)
        check(x, rt, None, False, 0)


def test_rejected_tokens_are_overwritten(rt):
    """A block over the rejected part of the one before; the exponent stays until slot 0 is written again."""
    x = Batch8([(6, 3)], 2, 1, 64, 16, BF16, seed=6)
    x.nk.mul_(1000)
    check(x, rt, 64, False, 32)
    high = int(x.k_exp[int(x.table[0, 0]), 0])
    x.nk.div_(1000)
    x.cached = [5]
    x.cache_len.fill_(5)
    check(x, rt, 64, False, 32)
    assert int(x.k_exp[int(x.table[0, 0]), 0]) == high
    x.cached = [0]
    x.cache_len.fill_(0)
    check(x, rt, 64, False, 32)
    assert int(x.k_exp[int(x.table[0, 0]), 0]) < high - 5


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_zeros_infinities_and_nan(rt, dtype):
    x = Batch8([(20, 0), (5, 4)], 2, 2, 64, 8, dtype, seed=7, exps=(-128, 127))
    x.nk[:8] = 0.0  # a page of zeros
    x.nk[9, 0, 3] = float("nan")
    x.nk[10, 1, 5], x.nk[11, 1, 6] = float("inf"), -float("inf")
    x.nv[8:16] = float("nan")
    x.nv[20] = 1e30  # beyond 448 * 2^40
    x.nv[22] = 1e-30
    check(x, rt, None, False, 0)


def test_borders_of_the_exponent(rt):
    """Largest magnitudes just at, below and above 448 times a power of two; every number between neighbours."""
    x = Batch8([(8, 0)] * 40, 1, 1, 64, 8, F32, seed=8)
    borders = 448.0 * 2.0 ** torch.arange(-20, 20, dtype=torch.float32)
    for b in range(40):
        x.nk[8 * b : 8 * b + 8] = (torch.randn(8, 1, 64) * borders[b] / 8).clamp(-borders[b], borders[b]).cuda()
        x.nk[8 * b, 0, 0] = borders[b]
        x.nv[8 * b : 8 * b + 8] = x.nk[8 * b : 8 * b + 8]
        x.nv[8 * b, 0, 0] = torch.nextafter(borders[b], torch.tensor(float("inf")))
    check(x, rt, None, False, 0)
    pages = x.table[:, 0].long()
    assert torch.equal(x.v_exp[pages, 0].int(), x.k_exp[pages, 0].int() + 1)


def test_positions_without_a_place(rt):
    """Negative lengths, positions past the rotation table, past the page table, and pages outside the cache."""
    x = Batch8([(5, -3), (6, 10), (4, 2), (3, 4)], 4, 2, 64, 8, BF16, seed=5)
    x.table[2, 0] = 10**6
    x.table[3, 0] = -7
    check(x, rt, 64, False, 14)  # sequence 1: positions 14 and 15 have no angles
    y = Batch8([(4, 6)], 4, 2, 64, 8, BF16)
    y.cached = [14]  # past the table's two pages
    y.cache_len.fill_(14)
    check(y, rt, 64, False, 40)


def test_rows_behind_the_last_sequence(rt):
    """Fewer tokens than rows: the others' queries and every other slot stay as they are."""
    x = Batch8([(3, 5), (4, 2)], 4, 2, 64, 8, BF16, seed=9)
    x.q_start = torch.tensor([0, 3, 5], dtype=torch.int32).cuda()
    x.starts = np.array([0, 3, 5])
    rope = rope_table(32, 64)
    before = f64(x.k), f64(x.v), x.k_exp.cpu().numpy(), x.v_exp.cpu().numpy(), x.table.cpu().numpy()
    rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, x.cache(rt), x.cache_len, rope, x.out, q_start=x.q_start)
    want = ref.append_fp8(f64(x.q), f64(x.nk), f64(x.nv), *before, x.starts, x.cached, f64(rope), False)
    assert bool((x.out[5:] == 77.0).all()) and np.array_equal(f64(x.v), want[2]) and np.array_equal(x.v_exp.cpu().numpy(), want[4])


def test_offsets_past_32_bits(rt):
    """A cache of more than 2^32 elements: the last pages are written and nothing else."""
    pages = 2**32 // (16 * 2 * 64) + 40
    k = torch.zeros((pages, 16, 2, 64), dtype=torch.uint8, device="cuda").view(E4M3)
    v = torch.zeros((pages, 16, 2, 64), dtype=torch.uint8, device="cuda").view(E4M3)
    exps = [torch.full((pages, 2), 5, dtype=torch.int8, device="cuda") for _ in range(2)]
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    nk = torch.randn((3, 2, 64), device="cuda").to(BF16)
    rt.retrace_kv_append_fp8(None, nk, nk, rt.KvCacheFp8(k, v, table, *exps), torch.tensor([14], dtype=torch.int32, device="cuda"), None)
    for c, e in zip((k, v), exps):
        assert e[pages - 1].tolist() == [5, 5]  # the page held tokens
        top = nk[2].float().abs().amax(-1).tolist()
        assert e[pages - 2].tolist() == [ref.page_exponent([a]) for a in top]
        got = f64(c[pages - 2, 0]) * np.exp2(f64(e[pages - 2]))[:, None]
        assert np.all(np.abs(got - f64(nk[2])) <= 2.0**-4 * np.abs(f64(nk[2])) + 2.0**-10 * np.exp2(f64(e[pages - 2]))[:, None])
        touched = torch.nonzero((c.view(torch.uint8) & 127).view(pages, -1).amax(-1)).flatten()
        assert set(touched.tolist()) <= {pages - 2, pages - 1}
        assert int((e != 5).sum()) <= 2


def test_other_stream_and_graph(rt):
    x, y = (Batch8([(4, 0), (4, 3)], 4, 2, 64, 8, F32) for _ in range(2))
    rope, cache = rope_table(16, 64), x.cache(rt)
    start = x.k.view(torch.uint8).clone(), x.k_exp.clone()
    check(y, rt, 64, False, 16)
    call = lambda: rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, cache, x.cache_len, rope, x.out, q_start=x.q_start)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    same = lambda: torch.equal(x.k.view(torch.uint8), y.k.view(torch.uint8)) and torch.equal(x.k_exp, y.k_exp) and torch.equal(x.out, y.out)  # noqa: E731
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(2):
        x.k.view(torch.uint8).copy_(start[0])
        x.k_exp.copy_(start[1])
        x.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same()
