"""retrace_sample against its float64 statement.

The kernel's weights are fp32 exponentials (a few 2^-24) taken to 31 binary
places, so its sums agree with float64 ones to about 1e-6 of the whole; the
tests put each uniform in the middle of a token's share (shares below 1e-4 of
the whole are left out), and each top_p in the middle of a step of the running
sum, so that the answer is one.  Probabilities agree to 1e-5.
"""

import numpy as np
import pytest
import torch

from oracle import serving_oracle as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def run(rt, logits, u, T=None, k=None, p=None, m=None, probs=True):
    B, R, _ = logits.shape
    dev = lambda x, t: None if x is None else torch.tensor(np.broadcast_to(x, (B,)).copy(), dtype=t, device="cuda")  # noqa: E731
    tokens = torch.full((B, R), -9, dtype=torch.int32, device="cuda")
    out = torch.full((B, R), -9.0, device="cuda") if probs else None
    rt.retrace_sample(logits, torch.tensor(u, dtype=F32, device="cuda").view(B, R), tokens, out, dev(T, F32), dev(k, torch.int32),
                      dev(p, F32), dev(m, F32))
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), out.cpu().numpy() if probs else None


def safe_p(x, T, k, p):
    """top_p near p, in the middle of a step of the running sum of the top-k tokens."""
    _, w = ref.kept_tokens(x, T, k, 1.0, 0.0)
    run_ = np.cumsum(w)
    i = min(int(np.searchsorted(run_, p)), len(w) - 1)
    while i > 0 and w[i] < 1e-4:
        i -= 1
    return float(run_[i] - 0.5 * w[i])


def middles(x, T, k, p, m, count, rng):
    """Uniforms in the middle of kept tokens' shares, with the tokens and their probabilities."""
    tokens, probs = ref.kept_tokens(x, T, k, p, m)
    by = np.argsort(tokens)
    tokens, probs = tokens[by], probs[by]
    big = np.flatnonzero(probs >= 1e-4)
    at = rng.choice(big, size=count)
    return (np.cumsum(probs) - 0.5 * probs)[at], tokens[at], probs[at]


CASES = [(1.0, 0, 1.0, 0.0), (0.7, 20, 0.95, 0.0), (1.3, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (0.9, 300, 0.8, 0.01), (1.0, 1, 0.5, 0.9),
         (1.0, 0, 0.01, 0.0), (2.0, 7, 1.0, 0.0), (0.01, 0, 0.99, 0.0)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 31, 1000, 4099, 32003, 151936])
def test_filters(rt, dtype, V):
    rng = np.random.default_rng(V)
    R = 6
    for T, k, p, m in CASES:
        x = torch.tensor(rng.normal(0, 2, (1, 1, V)), dtype=F32)
        x[0, 0, rng.integers(0, V, 12)] += torch.tensor(rng.uniform(2, 8, 12), dtype=F32)
        x = x.to(dtype)
        row = x[0, 0].double().numpy()
        T32, m32 = float(np.float32(T)), float(np.float32(m))
        p32 = float(np.float32(safe_p(row, T32, k, p))) if p < 1 else 1.0
        u, tokens, probs = middles(row, T32, k, p32, m32, R, rng)
        got, q = run(rt, x.cuda().expand(1, R, V), u, T32, k, p32, m32)
        assert np.array_equal(got[0], tokens), (T, k, p, m)
        assert np.all(np.abs(q[0] - probs) <= 1e-5 * probs + 1e-9), (T, k, p, m)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_kept_token_and_no_other(rt, dtype):
    """The uniforms walk over the whole kept set of rows with many equal logits: ties go to the lower index."""
    rng = np.random.default_rng(5)
    V = 200
    x = torch.tensor(rng.integers(0, 6, V) / 2.0, dtype=F32).to(dtype)
    row = x.double().numpy()
    for T, k, p, m in [(1.0, 37, 1.0, 0.0), (1.0, 0, 0.6003, 0.0), (1.0, 90, 0.7501, 0.0), (1.0, 0, 1.0, 0.3), (1.0, 50, 0.9007, 0.2)]:
        tokens, probs = ref.kept_tokens(row, T, k, float(np.float32(p)), float(np.float32(m)))
        by = np.argsort(tokens)
        u = (np.cumsum(probs[by]) - 0.5 * probs[by])
        got, q = run(rt, x.cuda().expand(1, len(u), V), u, T, k, p, m)
        assert np.array_equal(got[0], tokens[by]), (k, p, m)
        assert np.allclose(q[0], probs[by], rtol=1e-5, atol=0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_all_logits_equal(rt, dtype):
    V = 5000
    for value in (0.0, 3.5, -3e38, 3e38):
        x = torch.full((1, 4, V), value, dtype=F32).to(dtype).cuda()
        got, q = run(rt, x, [0.0, 0.5 + 0.5 / V, 0.25 + 0.5 / V, 0.9999], 1.0)
        assert got.tolist() == [[0, 2500, 1250, 4999]]
        assert np.allclose(q, 1 / V, rtol=1e-6)
        got, q = run(rt, x, [0.0, 0.5 + 0.05, 0.25, 0.9999], 1.0, 10)
        assert got.tolist() == [[0, 5, 2, 9]] and np.allclose(q, 0.1, rtol=1e-6)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masked_logits(rt, dtype):
    low = float(torch.finfo(dtype).min)
    inf, nan = float("inf"), float("nan")
    rows = [[-inf, 1.0, -inf, 1.0], [-inf] * 4, [nan, nan, 2.0, nan], [low, low, 0.0, low], [inf, 5.0, inf, 0.0], [nan] * 4,
            [low, low, low, low], [-0.0, 0.0, -1e30, low]]
    x = torch.tensor(rows, dtype=F32).to(dtype).view(len(rows), 1, 4).cuda()
    got, q = run(rt, x, [0.75] * len(rows), 1.0)
    assert got[:, 0].tolist() == [3, -1, 2, 2, 2, -1, 3, 1]
    assert np.allclose(q[:, 0], [0.5, 0, 1, 1, 0.5, 0, 0.25, 0.5])
    got, q = run(rt, x, [0.75] * len(rows), 0.0)
    assert got[:, 0].tolist() == [1, -1, 2, 2, 0, -1, 0, 0]
    assert np.allclose(q[:, 0], [1, 0, 1, 1, 1, 0, 1, 1])
    got, _ = run(rt, x, [0.75] * len(rows), 1.0, 3, 0.9, 0.1)
    assert got[:, 0].tolist() == [3, -1, 2, 2, 2, -1, 2, 1]


def test_settings_outside_their_range(rt):
    x = torch.tensor([3.0, 2.0, 1.0, 0.0], device="cuda").view(1, 1, 4)
    for kw, want in [(dict(T=-1.0), 0), (dict(T=float("nan")), 0), (dict(k=-5), 3), (dict(k=4), 3), (dict(k=10**9), 3),
                     (dict(p=0.0), 0), (dict(p=-1.0), 0), (dict(p=2.0), 3), (dict(p=float("nan")), 3), (dict(m=-1.0), 3),
                     (dict(m=float("nan")), 3), (dict(m=2.0), 0), (dict(T=1e30), 3), (dict(T=1e-30), 0)]:
        got, q = run(rt, x, [0.9999], **{"T": 1.0, **kw})
        assert got.tolist() == [[want]], kw
    for u, want in [(-1.0, 0), (float("nan"), 0), (1.0, 3), (7.0, 3), (float("inf"), 3)]:
        assert run(rt, x, [u])[0].tolist() == [[want]], u


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_settings_of_each_sequence(rt, dtype):
    rng = np.random.default_rng(8)
    B, R, V = 9, 5, 3001
    x = torch.tensor(rng.normal(0, 2, (B, R, V)), dtype=F32).to(dtype)
    T = np.array([1, 0, 0.5, 2, 1, 1, 0.8, 1.5, 0], np.float32)
    k = np.array([0, 5, 50, 1, 3000, 3001, 0, 10, 0])
    p = np.array([1, 0.5, 1, 1, 1, 1, 0.5, 1, 1], np.float32)
    m = np.array([0, 0, 0.1, 0, 0, 0.02, 0, 0, 0.5], np.float32)
    u, want = np.zeros((B, R)), np.zeros((B, R), int)
    for b in range(B):
        for r in range(R):
            row = x[b, r].double().numpy()
            if p[b] < 1 and T[b] > 0:  # one top_p serves the five rows: skip those whose cut is close
                w = ref.kept_tokens(row, T[b], k[b], 1.0, 0.0)[1]
                assert np.abs(np.cumsum(w) - p[b]).min() > 1e-6
            uu, tok, _ = middles(row, T[b], k[b], p[b], m[b], 1, rng)
            u[b, r], want[b, r] = uu[0], tok[0]
    assert np.array_equal(run(rt, x.cuda(), u, T, k, p, m)[0], want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad", [0, 1, 5, 8])
def test_strides_and_alignment(rt, dtype, pad):
    """Rows apart by any number of elements, starting anywhere."""
    rng = np.random.default_rng(pad)
    B, R, V = 3, 4, 10007
    whole = torch.tensor(rng.normal(0, 3, (B, R + 1, V + pad)), dtype=F32).to(dtype).cuda()
    x = whole[:, 1:, pad // 2:pad // 2 + V]
    for T, k, p, m in ((1.0, 50, 1.0, 0.0), (1.0, 0, 1.0, 0.0)):
        u, want = np.zeros((B, R)), np.zeros((B, R), int)
        for b in range(B):
            for r in range(R):
                uu, tok, _ = middles(x[b, r].double().cpu().numpy(), T, k, p, m, 1, rng)
                u[b, r], want[b, r] = uu[0], tok[0]
        assert np.array_equal(run(rt, x, u, T, k, p, m, probs=False)[0], want)


def test_the_same_token_whatever_the_batch(rt):
    """Rows alone and among many others (other kernels' shapes): every token and probability is the same."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for dtype, V in ((BF16, 50257), (F32, 32000)):
        x = torch.empty((400, 1, V), device="cuda").normal_(0, 1.5, generator=g).to(dtype)
        u = torch.rand((400,), generator=g, device="cuda").cpu().numpy()
        for T, k, p, m in ((1.0, 0, 0.9, 0.0), (0.8, 40, 0.95, 0.0), (1.0, 0, 1.0, 0.0)):
            many, q = run(rt, x, u, T, k, p, m)
            for n in (1, 5, 30):
                few, qf = run(rt, x[:n], u[:n], T, k, p, m)
                assert np.array_equal(few, many[:n]) and np.array_equal(qf, q[:n])


def test_vocabulary_past_shared_memory(rt):
    """A row of 2^21 logits: past what the shared memory of a cluster holds."""
    rng = np.random.default_rng(1)
    V = 1 << 21
    x = torch.tensor(rng.normal(0, 1, (1, 1, V)), dtype=F32)
    x[0, 0, [5, V // 2, V - 1]] += 12
    row = x[0, 0].double().numpy()
    for T, k, p, m in ((1.0, 40, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.7, 0, 1.0, 1e-3)):
        p32 = float(np.float32(safe_p(row, float(np.float32(T)), k, p))) if p < 1 else 1.0
        u, tokens, probs = middles(row, float(np.float32(T)), k, p32, float(np.float32(m)), 4, rng)
        got, q = run(rt, x.cuda().expand(1, 4, V), u, T, k, p32, m)
        assert np.array_equal(got[0], tokens) and np.all(np.abs(q[0] - probs) <= 1e-5 * probs + 1e-9)


def test_draws_follow_the_distribution(rt):
    """Frequencies over 200000 uniforms."""
    x = torch.tensor([2.0, 1.0, 0.0, -1.0, 1.5, -4.0], device="cuda")
    n = 200000
    u = np.random.default_rng(2).random(n)
    got, _ = run(rt, x.expand(1, n, 6), u, 0.9, 5, 0.97)
    tokens, probs = ref.kept_tokens(x.double().cpu().numpy(), float(np.float32(0.9)), 5, float(np.float32(0.97)), 0.0)
    for t in range(6):
        want = float(probs[tokens == t].sum())
        assert abs((got == t).mean() - want) < 5 * np.sqrt(max(want, 1e-9) / n) + 1e-9


def test_other_stream_and_graph(rt):
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty((2, 8, 32003), device="cuda").normal_(0, 2, generator=g).to(BF16)
    u = torch.rand((2, 8), generator=g, device="cuda")
    k = torch.tensor([20, 0], dtype=torch.int32, device="cuda")
    tokens = torch.zeros((2, 8), dtype=torch.int32, device="cuda")
    call = lambda: rt.retrace_sample(x, u, tokens, top_k=k)  # noqa: E731
    call()
    want = tokens.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tokens.zero_()
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(tokens, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    tokens.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(tokens, want)
