"""The decoding loop of examples/: appending, attention, sampling and the round together.

With top_k = 1 speculative decoding gives the tokens that the target alone gives, so
the loop's tokens are compared with a plain float64 decoding of the target, token by
token, without a cache.
"""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def loop():
    spec = importlib.util.spec_from_file_location("decode_loop", os.path.join(ROOT, "examples", "decode_loop.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def greedy(dec, anchors, steps):
    """The target's own tokens, in float64: every token's states from the whole prefix."""
    Hq, Hkv, D = dec.target.shape
    qkv, o, head, embed = (t.double() for t in (dec.target.qkv, dec.target.o, dec.target.head, dec.embed))
    cs = dec.target.rope.double()

    def turn(x):  # [n, H, D]
        c, s = cs[: x.shape[0], None, :, 0], cs[: x.shape[0], None, :, 1]
        a, b = x[..., : D // 2], x[..., D // 2 :]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    out, margin = [], []
    for b in range(dec.B):
        tokens = [int(anchors[b])]
        for _ in range(steps):
            x = embed[torch.tensor(tokens, device="cuda")]
            q, k, v = (x @ qkv.T).view(-1, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
            q, k = turn(q)[-1], turn(k)
            k, v = (t.repeat_interleave(Hq // Hkv, 1) for t in (k, v))
            w = torch.softmax(torch.einsum("hd,jhd->hj", q, k) * D**-0.5, -1)
            h = x[-1] + torch.einsum("hj,jhd->hd", w, v).reshape(-1) @ o.T
            top = (h @ head.T).topk(2)
            margin.append(float(top.values[0] - top.values[1]))
            tokens.append(int(top.indices[0]))
        out.append(tokens[1:])
    return out, min(margin)


def test_the_loop_gives_the_targets_own_tokens(loop):
    steps = 40
    dec = loop.Decoder(B=3, dtype=torch.float32, top_k=1, positions=256, seed=3)
    want, margin = greedy(dec, dec.anchor.clone(), steps)
    assert margin > 1e-4  # fp32 decides every token as float64 does
    got = [[] for _ in range(3)]
    most = 0
    while min(len(g) for g in got) < steps:
        committed, count = dec.round()
        most = max(most, int(count.max()))
        for b in range(3):
            got[b] += [int(t) for t in committed[b] if t >= 0]
    assert [g[:steps] for g in got] == want
    assert most > 1  # some drafts were accepted
    assert dec.ws.check() == 0 and dec.target.ws.check() == 0 and dec.drafter.ws.check() == 0


def test_the_loop_in_bf16_with_filters(loop):
    dec = loop.Decoder(B=4, dtype=torch.bfloat16, top_k=20, top_p=0.95, positions=256, seed=4)
    for _ in range(10):
        committed, count = dec.round()
        c = committed.cpu()
        for b in range(4):
            n = int(count[b])
            assert 1 <= n <= dec.K + 1 and bool(((c[b, :n] >= 0) & (c[b, :n] < dec.V)).all()) and bool((c[b, n:] == -1).all())
    assert dec.ws.check() == 0 and dec.target.ws.check() == 0 and dec.drafter.ws.check() == 0
