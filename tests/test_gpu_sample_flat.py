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
