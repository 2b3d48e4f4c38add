"""Inputs of the tests of the operators around a round."""

import numpy as np
import torch


class Batch:
    """A paged cache with its lengths, on the GPU.  `lens`: (new, cached) tokens of each sequence; pages in a
    random order, -1 past a sequence's end."""

    def __init__(self, lens, Hq, Hkv, D, page, dtype, seed=0, spare=2, pad=0, packed=True):
        g = torch.Generator().manual_seed(seed)
        self.new, self.cached = [n for n, _ in lens], [c for _, c in lens]
        self.Hq, self.Hkv, self.D, self.page, self.dtype = Hq, Hkv, D, page, dtype
        self.T, B = sum(self.new), len(lens)
        need = [max(0, -(-(n + c) // page)) for n, c in lens]
        pages, width = sum(need) + spare, max(1, max(need, default=1))
        order = torch.randperm(pages, generator=g)
        table = torch.full((B, width), -1, dtype=torch.int32)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = order[at:at + k].to(torch.int32)
            at += k
        # `pad` elements more than head_dim between heads
        full = torch.randn((2, pages, page, Hkv, D + pad), generator=g).to(dtype)
        self.k, self.v = (full[i].cuda()[..., :D] for i in range(2))
        self.table = table.cuda()
        self.cache_len = torch.tensor(self.cached, dtype=torch.int32).cuda()
        self.starts = np.concatenate([[0], np.cumsum(self.new)]).astype(int)
        self.q_start = torch.tensor(self.starts, dtype=torch.int32).cuda()
        if packed:
            qkv = torch.randn((self.T, Hq + 2 * Hkv, D + pad), generator=g).to(dtype).cuda()[..., :D]
            self.q, self.nk, self.nv = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        self.out = torch.full((self.T, Hq, D), 77.0, dtype=dtype, device="cuda")

    def cache(self, rt):
        return rt.KvCache(self.k, self.v, self.table)


def f64(t):
    return t.detach().double().cpu().numpy()


def rope_table(positions, rot, seed=0):
    a = np.arange(0, rot, 2) / max(rot, 1)
    t = np.arange(positions)[:, None] * 10000.0 ** -a
    return torch.tensor(np.stack([np.cos(t), np.sin(t)], -1), dtype=torch.float32).cuda()
