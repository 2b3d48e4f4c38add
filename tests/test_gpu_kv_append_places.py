"""What retrace_kv_append writes on another stream and in a graph: every place, and no other."""

import numpy as np
import pytest
import torch

from serving import Batch, rope_table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2608_29748_gb300 import binding

    return binding


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens", [[(4, 0), (4, 3)], [(17, 30), (0, 5), (1, 90)] + [(3, 7)] * 40])
def test_every_place_on_a_side_stream_and_in_a_graph(rt, dtype, lens):
    x = Batch(lens, 4, 2, 64, 8, dtype, seed=len(lens))
    x.k, x.v = torch.zeros_like(x.k), torch.zeros_like(x.v)
    x.nk[x.nk == 0] = 1.0
    x.nv[x.nv == 0] = 1.0
    rope, cache, table = rope_table(128, 64), x.cache(rt), x.table.cpu().numpy()
    mine = np.zeros(x.k.shape[:2], bool)  # the call's places
    for b, (n, c) in enumerate(lens):
        for p in range(c, c + n):
            mine[table[b, p // x.page], p % x.page] = True
    mine = torch.tensor(mine, device="cuda")
    tensors = (x.k, x.v, x.out)

    def clear():
        for t in tensors:
            t.zero_()

    def call():
        rt.retrace_kv_append(x.q, x.nk, x.nv, cache, x.cache_len, rope, x.out, q_start=x.q_start)

    clear()
    call()
    want = [t.clone() for t in tensors]
    for t in want[:2]:  # something in each place and nothing elsewhere
        assert torch.equal((t != 0).flatten(2).any(2), mine)
    assert bool((want[1][mine] != 0).all()) and bool((want[2] != 0).flatten(1).any(1).all())

    side = torch.cuda.Stream()
    clear()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(tensors, want))

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    clear()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(tensors, want))
