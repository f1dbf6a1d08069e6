"""fp64 CPU oracle of the paged cache: append, gather and attention.

TEST INFRASTRUCTURE ONLY.  It shares no code with the GPU library.

Pages are float64 arrays [n_pages, H, P, d] (bias [n_pages, H, P]); entry j of
sequence s is slot j % P of page table[s, j // P].  A page number outside
[0, n_pages) is an absent page, a length below 0 counts as 0, one above the
table's capacity as the capacity.
"""
from __future__ import annotations

import math

import numpy as np

from . import compactor


def _length(lens, s: int, table, P: int) -> int:
    return int(min(max(int(lens[s]), 0), table.shape[1] * P))


def slot(table, s: int, j: int, P: int, n_pages: int):
    """(page, slot) of entry j, or None where the page is absent."""
    p = int(table[s, j // P])
    return (p, j % P) if 0 <= p < n_pages else None


def append(k, v, k_pages, v_pages, table, lens, offsets=None, positions=None, rope_theta: float = 0.0, beta=None,
           beta_pages=None):
    """New pages (k', v', beta' or None) after the append of k, v [n_tokens, H, d]."""
    n_pages, H, P, d = k_pages.shape
    kp, vp = k_pages.copy(), v_pages.copy()
    bp = None if beta_pages is None else beta_pages.copy()
    n, S = k.shape[0], table.shape[0]
    off = [s * (n // S) for s in range(S + 1)] if offsets is None else [int(x) for x in offsets]
    if rope_theta:
        k = np.stack([compactor.rope(k[:, h], np.asarray(positions, np.float64), rope_theta) for h in range(H)], axis=1)
    for s in range(S):
        for i in range(max(off[s], 0), min(off[s + 1], n)):
            j = int(lens[s]) - off[s + 1] + i
            if not 0 <= j < table.shape[1] * P:
                continue
            at = slot(table, s, j, P, n_pages)
            if at is None:
                continue
            kp[at[0], :, at[1]], vp[at[0], :, at[1]] = k[i], v[i]
            if bp is not None:
                bp[at[0], :, at[1]] = 0.0 if beta is None else beta[i]
    return kp, vp, bp


def gather(pages, table, lens, s: int, start: int, n: int) -> np.ndarray:
    """Entries [start, start + n) of sequence s, [H, n, ...]; zeros past its length and in absent pages."""
    n_pages, H, P = pages.shape[:3]
    out = np.zeros((H, n) + pages.shape[3:])
    for i in range(n):
        at = slot(table, s, start + i, P, n_pages) if start + i < _length(lens, s, table, P) else None
        if at is not None:
            out[:, i] = pages[at[0], :, at[1]]
    return out


def attend(q, k_pages, v_pages, table, lens, causal: bool = False, scale: float = 0.0, beta_pages=None,
           q_positions=None, rope_theta: float = 0.0) -> np.ndarray:
    """q [n_seqs * n_queries, H * group, d] -> out like q (float64)."""
    n_pages, H, P, d = k_pages.shape
    S = table.shape[0]
    nq, group = q.shape[0] // S, q.shape[1] // H
    q = np.asarray(q, np.float64)
    if rope_theta:
        q = np.stack([compactor.rope(q[:, h], np.asarray(q_positions, np.float64), rope_theta)
                      for h in range(q.shape[1])], axis=1)
    sc = scale or 1.0 / math.sqrt(d)
    out = np.zeros_like(q)
    for s in range(S):
        L = _length(lens, s, table, P)
        there = [j for j in range(L) if slot(table, s, j, P, n_pages) is not None]
        if not there:
            continue
        at = [slot(table, s, j, P, n_pages) for j in there]
        pg, sl = np.array([a[0] for a in at]), np.array([a[1] for a in at])
        idx = np.array(there)
        for i in range(nq):
            seen = idx <= (L - nq + i if causal else L - 1)
            if not seen.any():
                continue
            for hq in range(q.shape[1]):
                h = hq // group
                x = sc * (k_pages[pg[seen], h, sl[seen]] @ q[s * nq + i, hq])
                if beta_pages is not None:
                    x = x + beta_pages[pg[seen], h, sl[seen]]
                if np.all(np.isneginf(x)):
                    continue
                e = np.exp(x - x.max())
                out[s * nq + i, hq] = (e @ v_pages[pg[seen], h, sl[seen]]) / e.sum()
    return out
