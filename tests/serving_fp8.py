"""Inputs of the tests of the cache in 8 bits."""

import numpy as np
import torch

from serving import Batch, f64

E4M3 = torch.float8_e4m3fn


class Batch8(Batch):
    """A Batch whose cache is in 8 bits: random numbers, a power of two for each page and head."""

    def __init__(self, lens, Hq, Hkv, D, page, dtype, seed=0, spare=2, pad=0, exps=(-8, -4)):
        super().__init__(lens, Hq, Hkv, D, page, dtype, seed, spare, pad)
        self.k, self.v = (to_codes(x, D + pad) for x in (self.k, self.v))
        g = torch.Generator().manual_seed(seed + 1)
        self.k_exp, self.v_exp = (torch.randint(*exps, (self.k.shape[0], Hkv), generator=g, dtype=torch.int8).cuda() for _ in range(2))

    def cache(self, rt):
        return rt.KvCacheFp8(self.k, self.v, self.table, self.k_exp, self.v_exp)

    def values(self):
        """k and v as what they stand for, float64."""
        exp = lambda e: np.exp2(np.clip(f64(e), -40, 40))[:, None, :, None]  # noqa: E731
        return f64(self.k) * exp(self.k_exp), f64(self.v) * exp(self.v_exp)


def to_codes(x, width):
    """x [pages, page_size, heads, D] as e4m3 numbers with heads `width` elements apart."""
    full = torch.zeros((*x.shape[:3], width), dtype=E4M3, device=x.device)[..., : x.shape[3]]
    full.copy_((x.float() * 64).clamp(-448, 448).to(E4M3))
    return full
