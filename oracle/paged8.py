"""fp64 CPU oracle of the paged cache in 8 bits, of the attention weights that entries
gather, and of the eviction by them.

TEST INFRASTRUCTURE ONLY.  It shares no code with the GPU library.

Pages hold e4m3 numbers as float64 [n_pages, H, P, d], scales are
[n_pages, H, P // 16]; lengths, tables and absent pages as in oracle.paged.
"""
from __future__ import annotations

import math

import numpy as np

from . import compactor
from .paged import _length, slot

BLOCK, LARGEST, LEAST = 16, 448.0, 2.0 ** -100


def e4m3(x) -> np.ndarray:
    """The nearest of the e4m3 numbers, found in the list of all of them, ties to the even code;
    NaN for what is not finite.  |x| <= 448."""
    x = np.asarray(x, np.float64)
    codes = np.arange(0x7F)                       # 0x7F is NaN
    e, f = codes >> 3, codes & 7
    values = np.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * 2.0 ** (e.astype(float) - 7))
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(values, a), 1, len(values) - 1)
    lo = hi - 1
    below, above = a - values[lo], values[hi] - a
    code = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isfinite(x), np.copysign(values[code], x), np.nan)


def scale_for(top: float) -> float:
    """The smallest power of two, LEAST at least, whose 448-fold reaches top."""
    if top == 0.0:
        return LEAST
    k = math.frexp(top)[1] - 10
    while LARGEST * 2.0 ** k < top:
        k += 1
    return max(2.0 ** k, LEAST)


def values(pages, scales) -> np.ndarray:
    """What the entries of all pages stand for."""
    return np.asarray(pages, np.float64) * np.repeat(np.asarray(scales, np.float64), BLOCK, axis=2)[..., None]


def append(k, v, k_pages, v_pages, k_scales, v_scales, table, lens, offsets=None, positions=None,
           rope_theta: float = 0.0, beta=None, beta_pages=None):
    """New (k', v', k_scales', v_scales', beta' or None)."""
    n_pages, H, P, d = k_pages.shape
    pools, scales = [k_pages.copy(), v_pages.copy()], [np.array(k_scales, np.float64), np.array(v_scales, np.float64)]
    bp = None if beta_pages is None else beta_pages.copy()
    n, S = k.shape[0], table.shape[0]
    off = [s * (n // S) for s in range(S + 1)] if offsets is None else [int(x) for x in offsets]
    if rope_theta:
        k = np.stack([compactor.rope(k[:, h], np.asarray(positions, np.float64), rope_theta) for h in range(H)], axis=1)
        k = k.astype(np.float32).astype(np.float64)
    for s in range(S):
        blocks = {}                                # block of the sequence: [(token, slot of the page)]
        for i in range(max(off[s], 0), min(off[s + 1], n)):
            j = int(lens[s]) - off[s + 1] + i
            if 0 <= j < table.shape[1] * P and slot(table, s, j, P, n_pages) is not None:
                blocks.setdefault(j // BLOCK, []).append((i, j % P))
        for b, new in blocks.items():
            page = slot(table, s, b * BLOCK, P, n_pages)[0]
            first, at = new[0][1] % BLOCK, new[0][1] // BLOCK
            for rows, pool, scale in ((k, pools[0], scales[0]), (v, pools[1], scales[1])):
                for h in range(H):
                    x = np.array([rows[i, h] for i, _ in new])
                    need = scale_for(np.abs(x[np.isfinite(x)]).max(initial=0.0))
                    old = scale[page, h, at]
                    now = max(old, need) if first else need
                    if first and now > old:
                        held = slice(at * BLOCK, at * BLOCK + first)
                        pool[page, h, held] = e4m3(pool[page, h, held] * (old / now))
                    for (_, sl), row in zip(new, x):
                        pool[page, h, sl] = e4m3(row / now)
                    scale[page, h, at] = now
            if bp is not None:
                for i, sl in new:
                    bp[page, :, sl] = 0.0 if beta is None else beta[i]
    return pools[0], pools[1], scales[0], scales[1], bp


def logits(q, k_pages, table, lens, causal: bool = False, scale: float = 0.0, beta_pages=None, q_positions=None,
           rope_theta: float = 0.0):
    """For each sequence (its present entries [n], logits [n_queries, H * group, n], minus infinity
    where a query does not see)."""
    n_pages, H, P, d = k_pages.shape
    S = table.shape[0]
    nq, group = q.shape[0] // S, q.shape[1] // H
    q = np.asarray(q, np.float64)
    if rope_theta:
        q = np.stack([compactor.rope(q[:, h], np.asarray(q_positions, np.float64), rope_theta)
                      for h in range(q.shape[1])], axis=1)
    out = []
    for s in range(S):
        L = _length(lens, s, table, P)
        there = np.array([j for j in range(L) if slot(table, s, j, P, n_pages) is not None], dtype=int)
        at = [slot(table, s, j, P, n_pages) for j in there]
        pg, sl = np.array([a[0] for a in at], dtype=int), np.array([a[1] for a in at], dtype=int)
        x = np.full((nq, q.shape[1], len(there)), -np.inf)
        for i in range(nq):
            seen = there <= (L - nq + i if causal else L - 1)
            for hq in range(q.shape[1]):
                y = (scale or 1.0 / math.sqrt(d)) * (k_pages[pg, hq // group, sl] @ q[s * nq + i, hq])
                if beta_pages is not None:
                    y = y + beta_pages[pg, hq // group, sl]
                x[i, hq, seen] = y[seen]
        out.append((there, x))
    return out


def lse(*args, **kw) -> np.ndarray:
    """log sum exp of every row's logits, [n_seqs * n_queries, H * group] (arguments of ``logits``)."""
    rows = []
    for _, x in logits(*args, **kw):
        m = x.max(axis=-1, initial=-np.inf)
        ref = np.where(np.isneginf(m), 0.0, m)
        with np.errstate(divide="ignore"):
            rows.append(np.log(np.exp(x - ref[..., None]).sum(axis=-1)) + ref)
    return np.concatenate(rows)


def score(q, row_lse, k_pages, scores, table, lens, known=None, **kw) -> np.ndarray:
    """New scores [n_pages, H, P]: the rows' weights e^(logit - row_lse) of every entry, summed over the
    rows of its KV head, added to its score, or in its place from entry known[s] on."""
    n_pages, H, P, _ = k_pages.shape
    nq, group = q.shape[0] // table.shape[0], q.shape[1] // H
    out = np.array(scores, np.float64)
    for s, (there, x) in enumerate(logits(q, k_pages, table, lens, **kw)):
        row = np.asarray(row_lse, np.float64)[s * nq:(s + 1) * nq]
        w = np.where(np.isneginf(x), 0.0, np.exp(np.where(np.isneginf(x), 0.0, x - np.where(np.isneginf(row), 0.0, row)[..., None])))
        w = w.reshape(nq, H, group, -1).sum(axis=(0, 2))
        for n, j in enumerate(there):
            page, sl = slot(table, s, j, P, n_pages)
            out[page, :, sl] = w[:, n] + (out[page, :, sl] if known is None or j < known[s] else 0.0)
    return out


def keep_entries(scores, n: int, keep: int, first: int, recent: int) -> np.ndarray:
    """The kept of n entries, in order: the first and the recent ones, then those of largest score
    (NaN lowest, ties to the lower entry) to `keep` in all."""
    if n <= keep:
        return np.arange(n)
    rank = sorted(range(n), key=lambda j: (not (j < first or j >= n - recent),
                                           math.inf if math.isnan(scores[j]) else -scores[j], j))
    return np.array(sorted(rank[:keep]), dtype=int)


def evict(table, lens, scores, keep: int, first: int = 0, recent: int = 0, shared: bool = False):
    """(kept [n_seqs, H or 1, keep] with -1 behind them, new lengths)."""
    n_pages, H, P = scores.shape
    S = table.shape[0]
    kept = np.full((S, 1 if shared else H, keep), -1, dtype=int)
    new = np.zeros(S, dtype=int)
    for s in range(S):
        n = _length(lens, s, table, P)
        x = np.full((H, n), -np.inf)               # (absent pages: lowest)
        for j in range(n):
            at = slot(table, s, j, P, n_pages)
            if at is not None:
                x[:, j] = scores[at[0], :, at[1]]
        if shared:
            with np.errstate(invalid="ignore"):
                x = x.astype(np.float64).sum(axis=0, keepdims=True).astype(np.float32)
        for h in range(len(x)):
            ids = keep_entries([float(y) for y in x[h]], n, keep, first, recent)
            kept[s, h, : len(ids)] = ids
        new[s] = min(n, keep)
    return kept, new


def move(pages, table, kept) -> np.ndarray:
    """Pages [n_pages, H, P, ...] with every sequence's kept entries at its front, in order."""
    n_pages, H, P = pages.shape[:3]
    out = pages.copy()
    for s in range(table.shape[0]):
        for h in range(H):
            ids = kept[s, h % kept.shape[1]]
            for to, j in enumerate(ids[ids >= 0]):
                src, dst = slot(table, s, int(j), P, n_pages), slot(table, s, to, P, n_pages)
                if dst is not None:
                    out[dst[0], h, dst[1]] = pages[src[0], h, src[1]] if src is not None else 0.0
    return out


def move8(pages, scales, table, kept):
    """(pages, scales) of 8 bits after the same: a block's scale is the largest of those that its entries had,
    LEAST where none was there."""
    n_pages, H, P, _ = pages.shape
    out, new = pages.copy(), np.array(scales, np.float64)
    for s in range(table.shape[0]):
        for h in range(H):
            ids = kept[s, h % kept.shape[1]]
            ids = ids[ids >= 0]
            for b in range(0, len(ids), BLOCK):
                dst = slot(table, s, b, P, n_pages)
                if dst is None:
                    continue
                src = [slot(table, s, int(j), P, n_pages) for j in ids[b:b + BLOCK]]
                had = [scales[x[0], h, x[1] // BLOCK] if x is not None else LEAST for x in src]
                top = max(had)
                for i, x in enumerate(src):
                    out[dst[0], h, dst[1] + i] = e4m3(pages[x[0], h, x[1]] * (had[i] / top)) if x is not None else 0.0
                new[dst[0], h, dst[1] // BLOCK] = top
    return out, new
