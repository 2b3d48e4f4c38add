"""retrace_sample where thousands of tokens share the logit that decides.

No list holds these, so the row goes to the slowest way: selection by the digits of the logits.
Weights are fp32 exponentials to 31 binary places: a token's share agrees with float64 to 1e-5,
and a cut lies in the middle of a tied token's share, 1e-5 of the whole or more.
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


def rows_of(V, rng):
    """Few values, thousands of tokens each, in any order; single ones above, between and masked ones."""
    x = rng.choice([0.0, 1.0, -1.0, 1.5], V, p=[0.4, 0.3, 0.2, 0.1])
    x[rng.integers(0, V, 40)] = rng.choice([4.0, 3.0, 0.5, -np.inf, np.nan, -0.0], 40)
    return x


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V, rows", [(30011, 3), (60007, 1), (30011, 300)])
@pytest.mark.parametrize("T, k, m", [(1.0, 0, 0.0), (0.7, 0, 0.05), (1.0, 17000, 0.0), (1.3, 9000, 0.0), (2.0, 25000, 0.4), (0.0, 0, 0.0)])
@pytest.mark.parametrize("p", [1.0, 0.9, 0.5, 0.2])
def test_cuts_among_equal_logits(rt, dtype, V, rows, T, k, m, p):
    rng = np.random.default_rng(V + k)
    x = torch.tensor(rows_of(V, rng), dtype=F32).to(dtype)
    row = x.double().numpy()
    T, m = float(np.float32(T)), float(np.float32(m))
    if p < 1 and T > 0:  # in the middle of a token's share
        w = ref.kept_tokens(row, T, k, 1.0, 0.0)[1]
        upto = np.cumsum(w)
        i = int(np.searchsorted(upto, p))
        p = float(np.float32(upto[i] - 0.5 * w[i]))
    tokens, probs = ref.kept_tokens(row, T, k, p, m)
    by = np.argsort(tokens)
    tokens, probs = tokens[by][probs[by] > 0], probs[by][probs[by] > 0]
    # anywhere, the first kept token, and the last
    at = np.concatenate([rng.integers(0, len(tokens), rows), [0, len(tokens) - 1]])[-max(rows, 3):]
    u = (np.cumsum(probs) - 0.5 * probs)[at]
    n = len(at)
    full = lambda v, t: torch.full((n,), v, dtype=t, device="cuda")  # noqa: E731
    got, q = torch.full((n, 1), -9, dtype=torch.int32, device="cuda"), torch.full((n, 1), -9.0, device="cuda")
    rt.retrace_sample(x.cuda().expand(n, 1, V), torch.tensor(u, dtype=F32, device="cuda").view(n, 1), got, q,
                      temperature=full(T, F32), top_k=full(k, torch.int32), top_p=full(p, F32), min_p=full(m, F32))
    got, q = got.cpu().numpy().ravel(), q.cpu().numpy().ravel()
    found = np.searchsorted(tokens, got)
    assert np.all(found < len(tokens)) and np.array_equal(tokens[found], got)
    # where shares are below 1e-5 the uniform in fp32 may fall into the neighbour's
    assert np.abs(found - at).max() <= (0 if probs.min() >= 1e-5 else 1)
    assert np.all(np.abs(q - probs[found]) <= 1e-5 * probs[found])
