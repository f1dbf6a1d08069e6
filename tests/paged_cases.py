"""Inputs of the paged-cache tests: random pages, tables and lengths, made on the CPU."""
from __future__ import annotations

import numpy as np
import torch

from paper_2606_07878_amd import configs

DT = {configs.MODE_BF16: torch.bfloat16, configs.MODE_FP32: torch.float32}


class Paged:
    """Pages [n_pages, H, P, d] holding ordinary values everywhere, a table of
    pages in random order and lengths; ``f64()`` gives the same as numpy."""

    def __init__(self, seed, lens, H, d, P, mode, beta=True, spare=3, width=None):
        self.rng = np.random.default_rng(seed)
        self.lens_list, self.H, self.d, self.P, self.mode = list(lens), H, d, P, mode
        n = len(self.lens_list)
        self.width = width or max(1, -(-max(max(self.lens_list), 1) // P))
        self.n_pages = n * self.width + spare
        g = torch.Generator().manual_seed(seed)
        self.k = torch.randn(self.n_pages, H, P, d, generator=g).to(DT[mode])
        self.v = torch.randn(self.n_pages, H, P, d, generator=g).to(DT[mode])
        self.beta = torch.randn(self.n_pages, H, P, generator=g) if beta else None
        self.table = torch.from_numpy(self.rng.permutation(self.n_pages)[: n * self.width].astype(np.int32)).reshape(
            n, self.width)
        self.lens = torch.tensor(self.lens_list, dtype=torch.int32)
        self.g = g

    def rows(self, n, heads=None):
        return torch.randn(n, heads or self.H, self.d, generator=self.g).to(DT[self.mode])

    def cuda(self):
        for x in ("k", "v", "beta", "table", "lens"):
            if getattr(self, x) is not None:
                setattr(self, x, getattr(self, x).cuda())
        return self

    def pages(self):
        return self.k, self.v, self.table, self.lens

    def f64(self):
        """(k, v, beta or None, table, lens) as numpy."""
        f = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
        return f(self.k), f(self.v), f(self.beta), self.table.cpu().numpy(), self.lens.cpu().numpy()
