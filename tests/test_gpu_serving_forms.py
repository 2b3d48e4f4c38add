"""The forms that the operators around a round choose by size, each against the float64
statement, and the binding's refusals.

Tolerances of attention: in bf16 the weights are rounded before the product with v and
the result once, at most 2^-8 of sum p |v| and of the result; in fp32 a score of up to 256
products has an error of about 16 * 2^-24 of their absolute sum (20 to 40 here), so a weight
one of 2e-5.  Sampling: uniforms in the middle of a token's share, probabilities to 1e-5.
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


def check(x, rt, q_start=True, cache=None, **mask):
    ws = rt.AttendWorkspace(x.Hq, x.Hkv, x.D, x.dtype)
    rt.retrace_attend(x.q, cache or x.cache(rt), x.cache_len, x.out, ws, q_start=x.q_start if q_start else None, **mask)
    torch.cuda.synchronize()
    assert ws.check() == 0
    want, spread = ref.attend(f64(x.q), f64(x.k), f64(x.v), x.table.cpu().numpy(), x.starts, x.cached, x.D**-0.5, **mask)
    tol = 2.0**-8 * (spread + np.abs(want)) if x.dtype == BF16 else 2e-5 * spread
    err = np.abs(f64(x.out) - want)
    assert np.all(err <= tol + 1e-30), (float(err.max()), np.argwhere(err > tol)[:4])


@pytest.mark.parametrize("D", [64, 72, 96, 128, 200])
@pytest.mark.parametrize("n", [1, 2, 9, 40, 140])
def test_fp32_rows_of_a_sequence(rt, D, n):
    """One row to hundreds: units of 8, 32 and 128 rows, in each width of a head."""
    check(Batch([(n, 70), (n, 0), (n, 333)], 3, 1, D, 16, F32, seed=n), rt, window=0)
    check(Batch([(n, 200), (n, 3)], 6, 2, D, 24, F32, seed=n + 1), rt, window=50, sinks=2, causal=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 20, 100])
def test_elements_that_are_not_whole_vectors(rt, dtype, n):
    """A head size of 50 and of 99: plain loads, columns past the head."""
    for D in (50, 99):
        check(Batch([(n, 90), (n, 0)], 4, 2, D, 10, dtype, seed=D), rt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n, G", [(1, 4), (1, 1), (4, 8), (5, 8)])
def test_blocks_of_one_size_share_units(rt, dtype, n, G):
    """Enough units that each is shared by two or three CTAs, of at most 32 rows and more."""
    lens = [(n, 700 + 37 * (b % 11)) for b in range(44)]
    check(Batch(lens, 2 * G, 2, 64, 16, dtype, seed=n), rt, q_start=False)
    check(Batch(lens, 2 * G, 2, 128, 16, dtype, seed=n), rt, q_start=False, window=300, sinks=5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_cache_of_another_order(rt, dtype, D):
    """Heads before slots within a page, and pages apart by more than their size."""
    x = Batch([(17, 300), (1, 90), (150, 0)], 8, 2, D, 16, dtype, seed=D)
    pages, page, heads, _ = x.k.shape
    room = torch.full((2, pages, heads, page + 3, D), float("nan"), dtype=dtype, device="cuda")
    k, v = (room[i, :, :, :page].permute(0, 2, 1, 3) for i in range(2))
    k.copy_(x.k)
    v.copy_(x.v)
    check(x, rt, cache=rt.KvCache(k, v, x.table))


def kept_middles(row, T, k, p, m, count, rng):
    tokens, probs = ref.kept_tokens(row, T, k, p, m)
    by = np.argsort(tokens)
    tokens, probs = tokens[by], probs[by]
    at = rng.choice(np.flatnonzero(probs >= 1e-5), size=count)
    return (np.cumsum(probs) - 0.5 * probs)[at], tokens[at], probs[at]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B, R, V", [(1, 1, 30011), (1, 16, 151936), (1, 19, 80000), (4, 16, 20000), (60, 10, 5003)])
def test_sampling_by_rows(rt, dtype, B, R, V):
    """A cluster to a row, clusters that share SMs, one CTA to a row, streamed rows; lists, flat
    rows and a large top_k.  Every row holds the same logits, so one statement serves all."""
    rng = np.random.default_rng(V + R)
    x = torch.tensor(rng.normal(0, 0.8, V), dtype=F32)
    x[rng.integers(0, V, 6)] += 2.0
    x = x.to(dtype)
    row = x.double().numpy()
    logits = x.cuda().expand(B, R, V)
    for T, k, p, m in [(1.0, 20, 1.0, 0.0), (1.0, 1800, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.5, 0, 0.5, 0.0), (1.0, 3000, 0.7, 0.0),
                       (0.0, 0, 0.9, 0.1), (1.0, 0, 1.0, 0.3)]:
        if p < 1 and T > 0:  # in the middle of a step of the running sum
            w = ref.kept_tokens(row, T, k, 1.0, 0.0)[1]
            steps = np.cumsum(w)
            i = int(np.searchsorted(steps, p))
            while w[i] < 1e-5:
                i -= 1
            p = float(steps[i] - 0.5 * w[i])
        p = float(np.float32(p))
        m = float(np.float32(m))
        u, want, probs = kept_middles(row, T, k, p, m, B * R, rng)
        each = lambda value, t: torch.full((B,), value, dtype=t, device="cuda")  # noqa: E731
        tokens = torch.full((B, R), -9, dtype=torch.int32, device="cuda")
        out = torch.full((B, R), -9.0, device="cuda")
        rt.retrace_sample(logits, torch.tensor(u, dtype=F32, device="cuda").view(B, R), tokens, out, temperature=each(T, F32),
                          top_k=each(k, torch.int32), top_p=each(p, F32), min_p=each(m, F32))
        torch.cuda.synchronize()
        assert np.array_equal(tokens.cpu().numpy().ravel(), want), (T, k, p, m)
        assert np.all(np.abs(out.cpu().numpy().ravel() - probs) <= 1e-5 * probs + 1e-9), (T, k, p, m)


def test_refusals_of_the_binding(rt):
    """Tensors of another type, shape or device, before anything is enqueued."""
    x = Batch([(2, 20), (2, 5)], 4, 2, 64, 16, BF16)
    cache, ws = x.cache(rt), rt.AttendWorkspace(4, 2, 64, BF16)
    rope = torch.zeros((64, 32, 2), device="cuda")
    attend = lambda **kw: rt.retrace_attend(**{**dict(q=x.q, cache=cache, cache_len=x.cache_len, out=x.out, ws=ws), **kw})  # noqa: E731
    append = lambda **kw: rt.retrace_kv_append(**{**dict(q=x.q, k=x.nk, v=x.nv, cache=cache, cache_len=x.cache_len, rope=rope,  # noqa: E731
                                                         q_out=x.out), **kw})
    for kw in (dict(q=x.q.float()), dict(q=x.q.cpu()), dict(q=x.q[:, :3]), dict(q=x.q[..., :32]), dict(out=x.out[:3]), dict(out=x.out.float()),
               dict(cache_len=x.cache_len.long()), dict(cache_len=x.cache_len.cpu()), dict(q_start=x.q_start.long()),
               dict(q_start=x.q_start[:2]), dict(q=x.q.transpose(1, 2))):
        with pytest.raises((ValueError, TypeError, rt.RetraceError)):
            attend(**kw)
    for kw in (dict(k=x.nk.float()), dict(v=x.nv[:, :1]), dict(k=x.nk.cpu()), dict(rope=rope.double()), dict(rope=rope.cpu()),
               dict(q_out=x.out[:, :2]), dict(cache_len=x.cache_len[:0])):
        with pytest.raises((ValueError, TypeError, rt.RetraceError)):
            append(**kw)
    logits, u = torch.zeros((2, 3, 50), device="cuda"), torch.zeros((2, 3), device="cuda")
    tokens = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    for args, kw in (((logits.half(), u, tokens), {}), ((logits.cpu(), u, tokens), {}), ((logits, u[:1], tokens), {}),
                     ((logits, u, tokens.long()), {}), ((logits, u, tokens), dict(top_k=torch.zeros(2, device="cuda"))),
                     ((logits, u, tokens), dict(top_p=torch.zeros(3, device="cuda")))):
        with pytest.raises((ValueError, TypeError, rt.RetraceError)):
            rt.retrace_sample(*args, **kw)
