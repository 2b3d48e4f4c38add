"""retrace_kv_reserve against its plain statement: whole numbers, so everything is equal."""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Pages:
    """A pool and its plain counterpart, called together and compared."""

    def __init__(self, rt, num_pages, page, B, width, seed=None):
        self.rt, self.page, self.B = rt, page, B
        self.pool = rt.PagePool.of(num_pages, page, B, width)
        if seed is not None:
            self.pool.free_pages.copy_(torch.randperm(num_pages, generator=torch.Generator().manual_seed(seed)))
        self.free = self.pool.free_pages.cpu().tolist()
        self.table, self.held = np.full((B, width), -1), [0] * B

    def call(self, cached, new, T=None, slots=True, run=None):
        T = sum(max(0, n) for n in new) if T is None else T
        q_start = torch.full((self.B + 1,), -9, dtype=torch.int32, device="cuda") if slots is not None else None
        out = torch.full((T,), -9, dtype=torch.int64, device="cuda") if slots else None
        (run or self.rt.retrace_kv_reserve)(i32(cached), i32(new), self.pool, q_start=q_start, slots=out)
        torch.cuda.synchronize()
        self.table, self.held, self.free, missing, starts, want = ref.reserve(cached, new, self.page, self.table, self.held, self.free, T)
        p = self.pool
        assert p.counts.tolist() == [len(self.free), missing]
        assert p.held.tolist() == self.held and np.array_equal(p.page_table.cpu().numpy(), self.table)
        assert p.free_pages[: len(self.free)].tolist() == self.free
        if slots is not None:
            assert q_start.tolist() == starts
        if slots:
            assert out.tolist() == want
        return out


@pytest.mark.parametrize("B", [1, 3, 33, 200, 600, 1500, 5000])
@pytest.mark.parametrize("page", [1, 16, 100])
def test_rounds(rt, B, page):
    """Blocks reserved, some tokens committed, pages given back, sequences that end and begin."""
    rng = np.random.default_rng(B + page)
    x = Pages(rt, B * (300 // page + 3), page, B, 300 // page + 2, seed=B)
    cached = rng.integers(0, 200, B)
    x.call([0] * B, cached)
    for _ in range(4):
        new = rng.integers(0, 18, B)
        x.call(cached, new)
        cached = cached + (new * rng.random(B)).astype(int)
        ended = rng.random(B) < 0.1
        cached[ended] = 0
        x.call(cached, [0] * B, slots=None)
        assert x.pool.held.tolist() == [-(-int(c) // page) for c in cached]
        cached = np.minimum(cached, 220)


def test_a_long_list_of_tokens(rt):
    """More tokens than one kernel lists; room behind them, and a list that is cut off."""
    rng = np.random.default_rng(0)
    new = rng.integers(0, 900, 70)
    new[[3, 4, 5, 69]] = 0
    total = int(new.sum())
    assert total > 20000
    for T in (total, total + 1000, total - 700, 20000):
        x = Pages(rt, 70 * 60, 16, 70, 80, seed=T)
        x.call([5] * 70, new, T=T)


def test_a_long_list_of_few_sequences_among_many(rt):
    """Long runs of sequences without tokens, before, between and behind those that have some."""
    new = np.zeros(3000, int)
    new[[700, 701, 2100]] = [9000, 3, 9000]
    x = Pages(rt, 3000, 16, 3000, 600, seed=6)
    x.call(np.where(np.arange(3000) % 7 == 0, 5, 0), new)


@pytest.mark.parametrize("B", [5, 800, 4500])
def test_too_few_pages(rt, B):
    """The first sequences get theirs; the others try again when there are more."""
    x = Pages(rt, 4 * B, 4, B, 12, seed=1)
    x.call([0] * B, [25] * B)
    x.call([0] * B, [25] * B)
    x.call([3 if b % 2 else 0 for b in range(B)], [0 if b % 2 else 25 for b in range(B)])
    x.call([0] * B, [25 if b % 2 else 0 for b in range(B)])
    x.call([0] * B, [0] * B)
    assert len(x.free) == 4 * B and sorted(x.free) == list(range(4 * B))


def test_lengths_out_of_range(rt):
    """Negative lengths, lengths past the table, sums past 32 bits."""
    x = Pages(rt, 64, 8, 4, 9, seed=2)
    x.call([-5, 3, 60, 0], [9, -4, 30, 0])
    x.call([-20, 3, 100, 0], [9, 0, 1, 2], T=40)
    assert x.pool.held.tolist() == [0, 1, 9, 1]
    big = [2**30] * 4  # not by the plain statement, which lists every token
    q_start, slots = i32([0] * 5), torch.zeros(50, dtype=torch.int64, device="cuda")
    rt.retrace_kv_reserve(i32([0, 0, 0, 2**30]), i32(big), x.pool, q_start=q_start, slots=slots)
    assert q_start.tolist() == [0, 50, 50, 50, 50] and x.pool.held.tolist() == [9] * 4
    table = x.pool.page_table.cpu()
    assert slots.tolist() == [int(table[0, p // 8]) * 8 + p % 8 for p in range(50)]
    rt.retrace_kv_reserve(i32([0] * 4), i32(big), x.pool, q_start=q_start)
    assert q_start.tolist() == [0, 2**30, 2**30, 2**30, 2**30]


def test_no_sequences_and_no_tokens(rt):
    x = Pages(rt, 4, 8, 0, 3)
    x.call([], [], T=5)
    y = Pages(rt, 4, 8, 2, 0)
    y.call([0, 0], [3, 1])
    z = Pages(rt, 0, 8, 2, 2)
    z.call([0, 0], [3, 1])
    w = Pages(rt, 4, 8, 2, 2)
    w.call([3, 0], [0, 0], T=0)


def test_a_table_with_rows_apart(rt):
    x = Pages(rt, 40, 8, 3, 4, seed=3)
    wide = torch.full((3, 9), 55, dtype=torch.int32, device="cuda")
    wide[:, :4] = -1
    x.pool = rt.PagePool(wide[:, :4], 8, x.pool.free_pages, x.pool.counts, x.pool.held)
    x.call([0, 5, 20], [9, 9, 40])
    assert bool((wide[:, 4:] == 55).all())


def test_given_back_pages_come_again_in_the_same_order(rt):
    x = Pages(rt, 500, 16, 20, 20, seed=4)
    cached, new = list(range(0, 200, 10)), [17] * 20
    x.call(cached, [0] * 20)
    first = x.call(cached, new)
    x.call(cached, [0] * 20, slots=None)
    assert torch.equal(x.call(cached, new), first)


def test_other_stream_and_graph(rt):
    B = 40
    x, y = (Pages(rt, 900, 16, B, 20, seed=5) for _ in range(2))
    cached, new = [7 * b for b in range(B)], [b % 18 for b in range(B)]

    def on_side(*args, **kw):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            rt.retrace_kv_reserve(*args, **kw)
        torch.cuda.current_stream().wait_stream(side)

    def in_graph(*args, **kw):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            rt.retrace_kv_reserve(*args, **kw)
        graph.replay()

    for run, z in ((on_side, x), (in_graph, y)):
        z.call(cached, [0] * B, run=run)
        z.call(cached, new, run=run)
        z.call([0] * B, [0] * B, run=run)


def test_refusals(rt):
    x = rt.PagePool.of(10, 8, 2, 4)
    good = dict(cache_len=i32([0, 0]), new_len=i32([1, 1]))
    with pytest.raises(ValueError, match="slots"):
        rt.retrace_kv_reserve(**good, pool=x, slots=torch.zeros(4, dtype=torch.int64, device="cuda"))
    for kw in (dict(cache_len=i32([0])), dict(new_len=i32([0, 1, 2])), dict(q_start=i32([0, 0])), dict(cache_len=torch.zeros(2, dtype=torch.int32)),
               dict(slots=torch.zeros(4, dtype=torch.int32, device="cuda"), q_start=i32([0, 0, 0]))):
        with pytest.raises(ValueError):
            rt.retrace_kv_reserve(**{**good, **kw}, pool=x)
    with pytest.raises(TypeError):
        rt.retrace_kv_reserve(torch.zeros(2, device="cuda"), good["new_len"], x)
    assert x.counts.tolist() == [10, 0]
