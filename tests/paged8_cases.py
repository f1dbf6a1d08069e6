"""Inputs of the 8-bit paged-cache tests: random codes and scales, tables and lengths, made on the CPU."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged8 as O8
from paper_2606_07878_amd import configs

DT = {configs.MODE_BF16: torch.bfloat16, configs.MODE_FP32: torch.float32}
E4M3 = torch.float8_e4m3fn


def f64(x):
    return None if x is None else x.double().cpu().numpy()


def equal(a, b):
    """The same codes (a NaN is one code)."""
    return torch.equal(a.cpu().view(torch.uint8), b.cpu().view(torch.uint8))


class Paged8:
    """Pages of codes [n_pages, H, P, d] with a scale of its own for each block of 16 entries and
    head, a table of pages in random order and lengths."""

    def __init__(self, seed, lens, H, d, P, beta=True, spare=3, width=None):
        self.rng = np.random.default_rng(seed)
        self.lens_list, self.H, self.d, self.P = list(lens), H, d, P
        n = len(self.lens_list)
        self.width = width or max(1, -(-max(max(self.lens_list), 1) // P))
        self.n_pages = n * self.width + spare
        self.g = torch.Generator().manual_seed(seed)
        for x in "kv":
            e = torch.randint(-3, 3, (self.n_pages, H, P // 16), generator=self.g).float()
            codes = torch.randn(self.n_pages, H, P, d, generator=self.g) * 2 ** (3 - e).repeat_interleave(16, dim=-1)[..., None]
            setattr(self, x, codes.clamp(-448, 448).to(E4M3))
            setattr(self, x + "s", torch.exp2(e - 3))
        self.beta = torch.randn(self.n_pages, H, P, generator=self.g) if beta else None
        self.scores = torch.exp(2 * torch.randn(self.n_pages, H, P, generator=self.g))
        self.table = torch.from_numpy(self.rng.permutation(self.n_pages)[: n * self.width].astype(np.int32)).reshape(
            n, self.width)
        self.lens = torch.tensor(self.lens_list, dtype=torch.int32)

    def rows(self, n, mode=configs.MODE_BF16, heads=None):
        return torch.randn(n, heads or self.H, self.d, generator=self.g).to(DT[mode])

    def cuda(self):
        for x in ("k", "v", "ks", "vs", "beta", "scores", "table", "lens"):
            if getattr(self, x) is not None:
                setattr(self, x, getattr(self, x).cuda())
        return self

    def pools(self):
        return self.k, self.v, self.ks, self.vs

    def pages(self):
        return self.k, self.v, self.ks, self.vs, self.table, self.lens

    def values(self):
        """(k, v) that the entries stand for, float64 numpy."""
        return O8.values(f64(self.k), f64(self.ks)), O8.values(f64(self.v), f64(self.vs))
