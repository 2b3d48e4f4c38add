"""retrace_kv_append against its float64 statement.

Tolerance.  A rotated element is x c - y s in fp32 (two products, a sum: at most
3 * 2^-24 of |x c| + |y s|), then one rounding to bf16 (8 significant bits: 2^-8 of the result).
Copied elements, and every place that the call does not own, are bit-exact.
"""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from serving import Batch, f64, rope_table

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def check(x, rt, rot, interleaved, positions, q_start=True, query=True):
    rope = rope_table(positions, rot) if rot is not None else None
    kc, vc, table = f64(x.k), f64(x.v), x.table.cpu().numpy()
    rt.retrace_kv_append(x.q if query else None, x.nk, x.nv, x.cache(rt), x.cache_len, rope, x.out if query else None,
                         q_start=x.q_start if q_start else None, interleaved=interleaved)
    torch.cuda.synchronize()
    want = ref.append(f64(x.q), f64(x.nk), f64(x.nv), kc, vc, table, x.starts, x.cached,
                      None if rope is None else f64(rope), interleaved)
    most = float(max(x.q.abs().max(), x.nk.abs().max())) if x.T else 0.0
    unit = 2.0**-8 if x.dtype == BF16 else 0.0
    for got, exp in ((f64(x.out), want[0]), (f64(x.k), want[1])):
        if got is not None and (query or exp is not want[0]):
            assert np.all(np.abs(got - exp) <= unit * np.abs(exp) + 3 * 2.0**-24 * 2 * most * (1 + unit))
    assert np.array_equal(f64(x.v), want[2])
    # what the call does not own keeps its bits
    same = want[1] == kc
    assert np.array_equal(f64(x.k)[same], kc[same])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D, rot", [(128, 128), (64, 32), (96, 48), (80, 80), (256, 64), (40, 6), (33, 32), (16, 0)])
def test_heads_and_rotations(rt, dtype, interleaved, D, rot):
    x = Batch([(3, 5), (1, 0), (7, 30)], 6, 2, D, 8, dtype, seed=D + rot)
    check(x, rt, rot, interleaved, 64)


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (7, 1), (32, 8), (71, 71)])
def test_head_counts(rt, Hq, Hkv):
    check(Batch([(5, 9), (2, 0)], Hq, Hkv, 64, 16, BF16, seed=Hq), rt, 64, False, 32)


@pytest.mark.parametrize("page", [1, 3, 16, 128])
def test_ragged_sequences(rt, page):
    """Sequences of no tokens, one, many; more sequences than one warp searches at a time."""
    lens = [(0, 4), (1, 0), (0, 0), (17, 40)] + [(b % 3, b) for b in range(40)] + [(0, 9)]
    check(Batch(lens, 4, 2, 64, page, BF16, seed=page), rt, 64, False, 64)


def test_many_sequences(rt):
    lens = [((b * 7) % 4, b % 11) for b in range(1200)]
    check(Batch(lens, 2, 1, 16, 4, F32, seed=3), rt, 16, False, 16)


def test_blocks_without_a_list(rt):
    check(Batch([(4, c) for c in (0, 3, 12)], 4, 2, 64, 8, BF16), rt, 64, False, 32, q_start=False)


def test_keys_and_values_only(rt):
    x = Batch([(4, 0), (4, 3)], 4, 2, 64, 8, BF16)
    check(x, rt, 64, False, 32, query=False)
    assert bool((x.out == 77.0).all())


def test_no_rotation(rt):
    check(Batch([(4, 0), (4, 3)], 4, 2, 64, 8, BF16), rt, None, False, 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_unaligned_and_strided(rt, dtype):
    """Heads an odd number of elements apart: no access of 16 bytes is aligned."""
    check(Batch([(3, 5), (6, 2)], 4, 2, 64, 8, dtype, pad=1), rt, 64, False, 32)


def test_queries_in_place(rt):
    x = Batch([(3, 5)], 4, 2, 64, 8, F32)
    rope, q0 = rope_table(16, 64), f64(x.q)
    rt.retrace_kv_append(x.q, x.nk, x.nv, x.cache(rt), x.cache_len, rope, x.q, q_start=x.q_start)
    want = np.stack([[ref.rotate(q0[t, h], f64(rope)[5 + t], False) for h in range(4)] for t in range(3)])
    assert np.abs(f64(x.q) - want).max() < 1e-6


def test_positions_without_a_place(rt):
    """Negative lengths, positions past the rotation table, past the page table, and pages outside the cache."""
    x = Batch([(5, -3), (6, 10), (4, 2), (3, 4)], 4, 2, 64, 8, BF16, seed=5)
    x.table[2, 0] = 10**6
    x.table[3, 0] = -7
    x.cached[1] = 10
    check(x, rt, 64, False, 14)  # sequence 1: positions 14 and 15 have no angles
    y = Batch([(4, 6)], 4, 2, 64, 8, BF16)
    y.cached = [14]  # past the table's two pages
    y.cache_len.fill_(14)
    check(y, rt, 64, False, 40)


def test_offsets_past_32_bits(rt):
    """A cache of more than 2^32 bytes and 2^31 elements: the last pages are written and nothing else."""
    pages = 2**31 // (16 * 2 * 64) + 40
    k = torch.zeros((pages, 16, 2, 64), dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    nk = torch.randn((3, 2, 64), device="cuda").to(BF16)
    rt.retrace_kv_append(None, nk, nk, rt.KvCache(k, v, table), torch.tensor([14], dtype=torch.int32, device="cuda"), None)
    assert torch.equal(v[pages - 1, 14:], nk[:2]) and torch.equal(k[pages - 2, 0], nk[2])
    assert int(torch.count_nonzero(k)) == int(torch.count_nonzero(nk))


def test_other_stream_and_graph(rt):
    x = Batch([(4, 0), (4, 3)], 4, 2, 64, 8, F32)
    rope, cache = rope_table(16, 64), x.cache(rt)
    call = lambda: rt.retrace_kv_append(x.q, x.nk, x.nv, cache, x.cache_len, rope, x.out, q_start=x.q_start)  # noqa: E731
    call()
    want = x.k.clone(), x.out.clone()
    x.k.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    got = x.k != 0
    assert torch.equal(x.k[got], want[0][got])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    x.out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x.out, want[1])
