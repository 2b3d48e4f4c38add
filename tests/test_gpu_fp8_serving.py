"""Pages, append and attention over a cache in 8 bits as a decoding loop uses them together.

Without a rotation the cache's contents are exact, so they are compared bit for bit; attention's
tolerance in bf16 is 2^-8 of sum p |v| and of the result (its weights and its own rounding).
"""

import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref
from serving import f64
from serving_fp8 import E4M3

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


class Loop:
    """A batch whose blocks of n tokens go into a cache and attend over it; some of them stay."""

    def __init__(self, rt, dtype, B=3, n=5, Hq=4, Hkv=2, D=64, page=16, width=12, pages=30, ws=None):
        self.rt, self.B, self.n, self.page, self.dtype = rt, B, n, page, dtype
        self.pool = rt.PagePool.of(pages, page, B, width)
        self.k, self.v = (torch.zeros((pages, page, Hkv, D), dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
        self.k_exp, self.v_exp = (torch.zeros((pages, Hkv), dtype=torch.int8, device="cuda") for _ in range(2))
        self.cache = rt.KvCacheFp8(self.k, self.v, self.pool.page_table, self.k_exp, self.v_exp)
        self.ws = ws or rt.AttendWorkspace(Hq, Hkv, D, E4M3)
        ints = lambda x, k: torch.full((k,), x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.length, self.new, self.none, self.q_start = ints(0, B), ints(n, B), ints(0, B), ints(0, B + 1)
        self.slots = torch.zeros(B * n, dtype=torch.int64, device="cuda")
        self.qkv = torch.zeros((B * n, Hq + 2 * Hkv, D), dtype=dtype, device="cuda")
        self.q, self.nk, self.nv = self.qkv.split([Hq, Hkv, Hkv], 1)
        self.turned, self.out = (torch.zeros((B * n, Hq, D), dtype=dtype, device="cuda") for _ in range(2))
        self.table, self.held, self.free = np.full((B, width), -1), [0] * B, list(range(pages))
        self.free = self.pool.free_pages.tolist()

    def block(self):
        self.rt.retrace_kv_reserve(self.length, self.new, self.pool, q_start=self.q_start, slots=self.slots)
        self.rt.retrace_kv_append_fp8(self.q, self.nk, self.nv, self.cache, self.length, None, self.turned, q_start=self.q_start)
        self.rt.retrace_attend_fp8(self.turned, self.cache, self.length, self.out, self.ws, q_start=self.q_start)

    def keep(self):
        self.rt.retrace_kv_reserve(self.length, self.none, self.pool)

    def state(self):
        return [f64(t) for t in (self.k, self.v)] + [t.cpu().numpy().astype(int) for t in (self.k_exp, self.v_exp)]

    def round(self, rng, gen, block, keep):
        length, new = self.length.tolist(), self.new.tolist()
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=gen) * torch.exp2(torch.randint(-3, 4, (self.qkv.shape[0], 1, 1), generator=gen)))
        before = self.state()
        block()
        torch.cuda.synchronize()
        T = self.B * self.n
        self.table, self.held, self.free, missing, starts, slots = ref.reserve(length, new, self.page, self.table, self.held, self.free, T)
        assert missing == 0 and np.array_equal(self.pool.page_table.cpu().numpy(), self.table)
        assert self.slots.tolist() == slots and self.q_start.tolist() == starts
        _, *want = ref.append_fp8(f64(self.q), f64(self.nk), f64(self.nv), *before, self.table, starts, length, None, False)
        for got, w in zip(self.state(), want):
            assert np.array_equal(got, w)
        total = starts[-1]
        assert torch.equal(self.turned[:total], self.q[:total])
        value = [c * np.exp2(e.astype(float))[:, None, :, None] for c, e in zip(want[:2], want[2:])]
        exact, spread = ref.attend(f64(self.q), *value, self.table, starts, length, self.q.shape[2] ** -0.5)
        tol = 2.0**-8 * (spread + np.abs(exact)) if self.dtype == BF16 else 2e-5 * spread
        assert np.all(np.abs(f64(self.out) - exact)[:total] <= tol[:total] + 1e-30)
        # some tokens stay; a sequence ends now and then
        kept = [c + int(rng.integers(0, n + 1)) for c, n in zip(length, new)]
        if rng.random() < 0.2:
            kept[rng.integers(self.B)] = 0
        kept = [0 if c > 100 else c for c in kept]
        self.length.copy_(torch.tensor(kept))
        self.new.copy_(torch.tensor(rng.integers(0, self.n + 1, self.B)))
        keep()
        torch.cuda.synchronize()
        self.table, self.held, self.free, *_ = ref.reserve(kept, [0] * self.B, self.page, self.table, self.held, self.free, 0)
        assert self.pool.held.tolist() == self.held and np.array_equal(self.pool.page_table.cpu().numpy(), self.table)
        assert self.ws.check() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rounds(rt, dtype):
    rng, gen = np.random.default_rng(1), torch.Generator().manual_seed(1)
    x = Loop(rt, dtype)
    for _ in range(25):
        x.round(rng, gen, x.block, x.keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rounds_in_graphs_that_share_a_workspace(rt, dtype):
    """Two loops, each captured, replayed in turn on one stream."""
    ws = rt.AttendWorkspace(4, 2, 64, E4M3)
    loops = [Loop(rt, dtype, ws=ws), Loop(rt, dtype, B=2, n=40, page=8, width=24, pages=48, ws=ws)]
    graphs = []
    for x in loops:
        x.block(), x.keep()  # before the capture: what a first call sets up
        x.pool.free_pages.copy_(torch.tensor(x.free, dtype=torch.int32))
        x.pool.counts.copy_(torch.tensor([len(x.free), 0]))
        x.pool.held.zero_(), x.pool.page_table.fill_(-1)
        torch.cuda.synchronize()
        pair = []
        for call in (x.block, x.keep):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
            pair.append(graph)
        graphs.append(pair)
    rngs = [(np.random.default_rng(s), torch.Generator().manual_seed(s)) for s in (2, 3)]
    for _ in range(10):
        for x, (block, keep), (rng, gen) in zip(loops, graphs, rngs):
            x.round(rng, gen, block.replay, keep.replay)


def test_a_prefix_that_sequences_share(rt):
    """Pages in several rows of the table: read by all of them, written behind them."""
    x = Loop(rt, BF16, B=4, n=5, pages=40)
    g = torch.Generator().manual_seed(5)
    prefix = torch.arange(3, dtype=torch.int32)
    x.k[prefix.long()] = (torch.randn(3, 16, 2, 64, generator=g) * 60).to(E4M3).cuda()
    x.v[prefix.long()] = (torch.randn(3, 16, 2, 64, generator=g) * 60).to(E4M3).cuda()
    x.k_exp[:3], x.v_exp[:3] = -6, -5
    table = torch.full((4, 12), -1, dtype=torch.int32)
    table[:, :3] = prefix
    table[:, 3] = torch.arange(10, 14)
    x.pool.page_table.copy_(table)
    x.length.copy_(torch.tensor([48, 48, 48, 48]))
    x.qkv.copy_(torch.randn(x.qkv.shape, generator=g))
    x.q_start.copy_(torch.arange(0, 25, 5))
    before, starts = x.state(), list(range(0, 25, 5))
    rt.retrace_kv_append_fp8(x.q, x.nk, x.nv, x.cache, x.length, None, x.turned, q_start=x.q_start)
    rt.retrace_attend_fp8(x.turned, x.cache, x.length, x.out, x.ws, q_start=x.q_start)
    _, *want = ref.append_fp8(f64(x.q), f64(x.nk), f64(x.nv), *before, table.numpy(), starts, [48] * 4, None, False)
    for got, w in zip(x.state(), want):
        assert np.array_equal(got, w)
    value = [c * np.exp2(e.astype(float))[:, None, :, None] for c, e in zip(want[:2], want[2:])]
    exact, spread = ref.attend(f64(x.q), *value, table.numpy(), starts, [48] * 4, 0.125)
    assert np.all(np.abs(f64(x.out) - exact) <= 2.0**-8 * (spread + np.abs(exact)))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_example(dtype):
    """The loop of examples/ with caches in 8 bits: it runs, and no page is lost."""
    spec = importlib.util.spec_from_file_location("decode_loop", os.path.join(ROOT, "examples", "decode_loop.py"))
    loop = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(loop)
    dec = loop.Decoder(B=4, dtype=dtype, top_k=20, top_p=0.95, positions=256, seed=4, cache="fp8")
    for _ in range(10):
        committed, count = dec.round()
        c = committed.cpu()
        for b in range(4):
            n = int(count[b])
            assert 1 <= n <= dec.K + 1 and bool(((c[b, :n] >= 0) & (c[b, :n] < dec.V)).all()) and bool((c[b, n:] == -1).all())
        for layer in (dec.target, dec.drafter):
            pool = layer.pool
            assert pool.held.tolist() == [-(-n // loop.PAGE) for n in dec.length.tolist()]
            used = [p for b, n in enumerate(pool.held.tolist()) for p in pool.page_table[b, :n].tolist()]
            assert sorted(used + pool.free_pages[: int(pool.counts[0])].tolist()) == list(range(pool.free_pages.numel()))
    assert dec.ws.check() == 0 and dec.target.ws.check() == 0 and dec.drafter.ws.check() == 0
