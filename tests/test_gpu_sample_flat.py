"""retrace_sample on rows where no short list holds what top-p keeps."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


def draw(rt, x, u, p):
    """Tokens and probabilities of rows [n, V] with a top_p each."""
    n = x.shape[0]
    tokens, probs = torch.full((n, 1), -9, dtype=torch.int32, device="cuda"), torch.full((n, 1), -9.0, device="cuda")
    rt.retrace_sample(x.view(n, 1, -1), u.view(n, 1), tokens, probs, top_p=p)
    return tokens, probs


@pytest.mark.parametrize("dtype, V", [(BF16, 151936), (F32, 32003), (F32, 2500)])
def test_the_same_cut_in_a_cluster_and_in_a_stream(rt, dtype, V):
    """Hundreds of cuts, by the CTAs of a cluster together and by one CTA among many: the same bits."""
    g = torch.Generator(device="cuda").manual_seed(V)
    for turn in range(20):
        x = torch.empty((400, V), device="cuda").normal_(0, 1 + turn % 3 / 2, generator=g).to(dtype)
        u = torch.rand((400,), generator=g, device="cuda")
        p = torch.rand((400,), generator=g, device="cuda") * 0.6 + 0.39
        many = draw(rt, x, u, p)
        for n in (1, 18, 30):
            few = draw(rt, x[:n], u[:n], p[:n])
            assert torch.equal(few[0], many[0][:n]) and torch.equal(few[1], many[1][:n]), (turn, n)
    assert bool((many[0] >= 0).all())


NEAR_ONE = (0.999, 0.9999, 0.99999, 1 - 2.0**-24)


@pytest.mark.parametrize("std", [1.0, 2.0, 3.0])
@pytest.mark.parametrize("dtype, V", [(BF16, 151936), (F32, 32003)])
@pytest.mark.parametrize("rows", [4, 400])
def test_nearly_the_whole_row_is_kept(rt, dtype, V, std, rows):
    """A token's probability is its share of the row over the kept share: top_p, to one token.
    Weights are fp32 exponentials to 31 binary places, so sums agree with float64 ones to about
    1e-6; a token of 1e-5 or less is what the kept share is past top_p."""
    rng = np.random.default_rng(int(std * 10) + V)
    x = torch.tensor(rng.normal(0, std, V), dtype=F32).to(dtype)
    w = np.exp(x.double().numpy() - float(x.max()))
    w /= w.sum()
    big = rng.choice(np.flatnonzero(w >= np.sort(w)[-30]), size=rows)
    by = np.argsort(-w, kind="stable")
    upto = np.cumsum(w[by])
    for p in NEAR_ONE:
        p32 = float(np.float32(p))
        kept = np.zeros(V, bool)
        kept[by[: int(np.searchsorted(upto, p32)) + 1]] = True
        q = w * kept / (w * kept).sum()
        u = (np.cumsum(q) - 0.5 * q)[big]
        tokens, probs = draw(rt, x.cuda().expand(rows, V), torch.tensor(u, dtype=F32, device="cuda"),
                             torch.full((rows,), p32, device="cuda"))
        assert np.array_equal(tokens.cpu().numpy().ravel(), big), p
        assert np.all(np.abs(probs.cpu().numpy().ravel() / q[big] - 1) <= 1.1e-5), p


@pytest.mark.parametrize("rows, V, dtype", [(16, 151936, BF16), (1024, 151936, BF16), (8, 50257, F32), (528, 32003, F32)])
def test_a_cut_near_the_end_costs_about_what_others_do(rt, rows, V, dtype):
    """top_p near one on a flat row is no case for the slowest way (10 to 25 times as long)."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.empty((rows, V), device="cuda").normal_(0, 2, generator=g).to(dtype)
    u = torch.rand((rows,), generator=g, device="cuda")

    def time(p):
        p = torch.full((rows,), p, device="cuda")
        draw(rt, x, u, p)
        took = []
        for _ in range(7):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(4):
                draw(rt, x, u, p)
            b.record()
            b.synchronize()
            took.append(a.elapsed_time(b))
        return sorted(took)[3]

    usual = time(0.9)
    for p in NEAR_ONE:
        assert time(p) < 4 * usual, p
