"""The weights that one call of still_paged_score / still_paged8_score adds, held against the fp64
oracle by themselves: scores of entries that hardly any row looks at are small, and an old score
beside them must not hide that.

Bars, from the arithmetic: a row's weight is off by `off` of itself: its logit's error (scale
sum|q k| times 2 d 2^-24, 4e-7 more where rotated), the rounding of its argument, which holds the
logit and the lse (2^-24 each of them, and 2^-24 of their difference), and the exponential's
2^-22.  Weights below 2^-126 are held as zero.  The sum of R rows and the old score is off by
(R + 1) 2^-24 of itself.  What no row sees and no call writes: equal.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged8 as O8
from paper_2606_07878_amd import binding, configs
from tests.helpers import log
from tests.paged8_cases import DT, Paged8, f64

pytestmark = pytest.mark.gpu

BF16, FP32, E8 = configs.MODE_BF16, configs.MODE_FP32, "e4m3"
TYPES = [(BF16, BF16), (FP32, FP32), (E8, BF16), (E8, FP32)]


def keys_of(c, kind):
    """(keys of c in this type, their scales or None, what they stand for in float64)."""
    if kind == E8:
        return c.k, c.ks, c.values()[0]
    k = torch.from_numpy(c.values()[0]).to(DT[kind])
    return k, None, f64(k)


def off_of(c, q, K, row_lse, scale, theta):
    """What a weight may be off by, of itself."""
    S, qk = len(c.lens_list), 0.0
    nq, group = q.shape[0] // S, q.shape[1] // c.H
    for s in range(S):
        pages = [int(p) for p in c.table[s] if 0 <= int(p) < c.n_pages]
        qs = np.abs(f64(q)[s * nq:(s + 1) * nq])
        qs = qs + np.roll(qs, c.d // 2, axis=-1) if theta else qs
        for h in range(c.H):
            rows = np.abs(np.nan_to_num(K[pages, h])).reshape(-1, c.d)
            qk = max(qk, (qs[:, h * group:(h + 1) * group].reshape(-1, c.d) @ rows.T).max())
    scale = scale or c.d ** -0.5
    fine = np.abs(row_lse[np.isfinite(row_lse)]).max(initial=0.0)
    return scale * qk * (2 * c.d * 2.0 ** -24 + (4e-7 if theta else 0.0)) + 4 * max(fine, scale * qk) * 2.0 ** -24 + 2.0 ** -22


def check_weights(c, q, kind, causal=False, scale=0.0, qpos=None, theta=0.0, known=None, scores=None):
    """One call on these scores (c's), against the oracle's weights of the same rows."""
    k, ks, K = keys_of(c, kind)
    scores = c.scores if scores is None else scores
    tn, ln = c.table.numpy(), c.lens.numpy()
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    how = dict(causal=causal, scale=scale, beta_pages=f64(c.beta), q_positions=f64(qpos), rope_theta=theta)
    lse = torch.from_numpy(O8.lse(f64(q), K, tn, ln, **how)).float()
    got = scores.cuda().clone()
    binding.paged_score(q.cuda(), lse.cuda(), k.cuda(), got, c.table.cuda(), c.lens.cuda(), causal=causal, scale=scale,
                        k_scales=dev(ks), beta_pages=dev(c.beta), known=dev(known), q_positions=dev(qpos), rope_theta=theta)
    torch.cuda.synchronize()
    kn = None if known is None else known.numpy()
    w = O8.score(f64(q), f64(lse), K, np.zeros(c.scores.shape), tn, ln, None, **how)
    ref = O8.score(f64(q), f64(lse), K, f64(scores), tn, ln, kn, **how)
    R = q.shape[0] // len(c.lens_list) * q.shape[1] // c.H
    off = off_of(c, q, K, f64(lse), scale, theta)
    g = f64(got)
    excess = np.abs(g - ref) - off * np.minimum(w, R) - R * 2.0 ** -126 - (R + 1) * 2.0 ** -24 * np.abs(ref)
    seen = w > 0.0
    log(f"  weights: worst excess {excess.max():.3e}, of a weight {off:.2e}, smallest of them {w[seen].min(initial=1.0):.1e}")
    assert excess.max() <= 0.0
    assert np.array_equal(g[~seen], ref[~seen])
    return got


@pytest.mark.parametrize("kind,mode", TYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq", [(1, 1), (2, 1), (4, 1), (1, 3), (5, 1), (2, 4), (7, 1), (3, 3), (3, 5), (8, 4), (17, 1), (1, 32)])
def test_weights_of_rows_and_widths(kind, mode, d, group, nq):
    """In place of what the slots held: the weights alone."""
    log(f"weights kind={kind} mode={mode} d={d} group={group} nq={nq}")
    c = Paged8(90, [600, 77, 0, 3], 2, d, 32)
    check_weights(c, c.rows(4 * nq, mode, heads=2 * group), kind, causal=nq > 1, known=torch.zeros(4, dtype=torch.int32))


@pytest.mark.parametrize("kind,mode", TYPES)
@pytest.mark.parametrize("group,nq", [(1, 1), (4, 1), (2, 4), (3, 5), (8, 4)])
def test_weights_beside_old_scores(kind, mode, group, nq):
    """Added to scores of their own size, to zeros, and in place of some."""
    log(f"weights kind={kind} mode={mode} group={group} nq={nq}, added")
    c = Paged8(91, [600, 77, 0, 3], 2, 128, 32)
    q = c.rows(4 * nq, mode, heads=2 * group)
    check_weights(c, q, kind, causal=nq > 1, scores=c.scores * 2.0 ** -10)
    check_weights(c, q, kind, causal=nq > 1, scores=torch.zeros_like(c.scores))
    check_weights(c, q, kind, causal=nq > 1, scores=c.scores * 2.0 ** -10, known=torch.tensor([599, 40, 0, 0], dtype=torch.int32))


@pytest.mark.parametrize("kind,mode", TYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq", [(1, 1), (1, 3), (4, 2), (3, 5), (8, 4), (1, 32), (32, 1)])
def test_weights_of_rotated_queries(kind, mode, d, group, nq):
    """Every tile of rows, rows that leave a tile partly empty, and the widest rows of the most queries."""
    log(f"weights rotated kind={kind} mode={mode} d={d} group={group} nq={nq}")
    c = Paged8(92, [600, 77, 0, 3], 2, d, 32)
    pos = 131000.0 + torch.arange(4 * nq, dtype=torch.float64) * 1.5
    check_weights(c, c.rows(4 * nq, mode, heads=2 * group), kind, causal=nq > 1, qpos=pos, theta=1e6,
                  known=torch.zeros(4, dtype=torch.int32))


@pytest.mark.parametrize("kind,mode", TYPES)
def test_weights_of_sharp_rows(kind, mode):
    """Logits far apart, so that most weights are tiny or below what 32 bits hold."""
    log(f"weights sharp kind={kind} mode={mode}")
    c = Paged8(93, [500, 40], 2, 128, 16)
    check_weights(c, c.rows(2, mode, heads=8), kind, scale=2.0, known=torch.zeros(2, dtype=torch.int32))


@pytest.mark.parametrize("kind", [E8, BF16])
def test_weights_of_a_window_in_several_calls(kind):
    """The last 40 tokens of a prompt, 4 query rows a KV head each: eight tokens a call, whose lengths end
    at its last token; entries behind the lengths of the call before are new."""
    c = Paged8(94, [300, 41], 2, 128, 16)
    window, step, group = 40, 8, 4
    k, ks, K = keys_of(c, kind)
    q = c.rows(2 * window, heads=2 * group).view(2, window, 2 * group, 128)
    got, known = c.scores.cuda().clone(), torch.zeros(2, dtype=torch.int32, device="cuda")
    k, ks, beta, table = k.cuda(), None if ks is None else ks.cuda(), c.beta.cuda(), c.table.cuda()
    v, vs = (k, ks)
    for i in range(0, window, step):
        rows = q[:, i:i + step].reshape(2 * step, 2 * group, 128).cuda()
        lens = (c.lens - window + i + step).cuda()
        lse = torch.empty(rows.shape[:2], device="cuda")
        if kind == E8:
            binding.paged8_attend(rows, k, v, ks, vs, table, lens, causal=True, beta_pages=beta, lse=lse)
        else:
            binding.paged_attend(rows, k, v, table, lens, causal=True, beta_pages=beta, lse=lse)
        binding.paged_score(rows, lse, k, got, table, lens, causal=True, k_scales=ks, beta_pages=beta, known=known)
        known.copy_(lens)
    torch.cuda.synchronize()
    every = q.reshape(2 * window, 2 * group, 128)
    how = dict(causal=True, beta_pages=f64(c.beta))
    tn, ln = c.table.numpy(), c.lens.numpy()
    row_lse = O8.lse(f64(every), K, tn, ln, **how)
    ref = O8.score(f64(every), row_lse, K, f64(c.scores), tn, ln, [0, 0], **how)
    # the attention's lse is off like a logit, by its sum's n / 4 + 64 roundings and 2^-23 of itself more
    off = 2 * off_of(c, every, K, row_lse, 0.0, 0.0) + (300 / 4 + 64) * 2.0 ** -24 + 2.0 ** -23 * np.abs(row_lse[np.isfinite(row_lse)]).max()
    R = window * group
    excess = np.abs(f64(got) - ref) - off * np.where(ref == f64(c.scores), 0.0, ref) - R * 2.0 ** -126 - (R + 1) * 2.0 ** -24 * np.abs(ref)
    assert excess.max() <= 0.0
    written = math.prod(ref.shape) - int((ref == f64(c.scores)).sum())
    assert written == 2 * (300 + 41)
