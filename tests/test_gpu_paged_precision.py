"""What the paged attention keeps of its weights, rotated queries and
exponentials: 24 bits, as the dense attention does.

The stored bf16 output would hide anything finer, so the values are made to
cancel: the output is some 2^-18 of its terms, and what the weights lost shows
in it whole.  Each bar counts the roundings by 2^-24 (half a step) or 2^-23
(an instruction that may be off by a step).
"""
import numpy as np
import pytest
import torch

from oracle import paged as O
from paper_2606_07878_amd import configs
from tests.helpers import log

pytestmark = pytest.mark.gpu

BF16, FP32 = configs.MODE_BF16, configs.MODE_FP32
U = 2.0 ** -24


def bf(x):
    """Nearest bf16 of float64 values, as float64."""
    return torch.from_numpy(np.asarray(x)).to(torch.bfloat16).double().numpy()


def f32(x):
    return np.asarray(x, np.float32).astype(np.float64)


def pages_of(rows, P=16):
    """[S, H, n, ...] (n <= P) as one page per sequence, the slots behind the entries NaN."""
    full = np.full(rows.shape[:2] + (P,) + rows.shape[3:], np.nan)
    full[:, :, : rows.shape[2]] = rows
    return torch.from_numpy(full)


def run(k, v, beta, q, dtype, width, pos=None, theta=0.0, scale=0.0):
    """(output, oracle's) of sequences of n entries: k, v [S, H, n, d], beta [S, H, n], q [S, H, d], values of `dtype`."""
    from paper_2606_07878_amd import binding
    S, H, n, d = v.shape
    table = torch.full((S, width), -1, dtype=torch.int32)
    table[:, 0] = torch.arange(S, dtype=torch.int32)
    lens = torch.full((S,), n, dtype=torch.int32)
    kp, vp, bp = pages_of(k), pages_of(v), pages_of(beta)
    got = binding.paged_attend(torch.from_numpy(q).to(dtype).cuda(), kp.to(dtype).cuda(), vp.to(dtype).cuda(), table.cuda(),
                               lens.cuda(), beta_pages=bp.float().cuda(), scale=scale,
                               q_positions=None if pos is None else torch.from_numpy(pos).cuda(), rope_theta=theta)
    ref = O.attend(q, kp.numpy(), vp.numpy(), table.numpy(), lens.numpy(), False, scale, bp.numpy(), pos, theta)
    return got.double().cpu().numpy(), ref


# a workgroup per sequence and head, a wave, parts of the line
KERNELS = [(30, 1), (40, 1), (30, 80)]


@pytest.mark.parametrize("seqs,width", KERNELS)
def test_weights(seqs, width):
    """Logits are the bias (q = 0): weights 1, p2 in (0.5, 1) and p3 near 2^-9.4;
    v2 takes v1's weighted value away, v3 what bf16 left of it.  9 products
    (three entries, at most three parts) are summed in at most 2^-23 of |v1|
    each; p2's exponential is off by 3 U and p3's counts 2^-8 of that.  A
    weight of 16 bits is off by up to 2^-17."""
    rng = np.random.default_rng(seqs + width)
    H, d = 8, 64
    beta = f32(np.stack([np.zeros((seqs, H)), rng.uniform(-0.69, 0.0, (seqs, H)), rng.uniform(-7.0, -6.0, (seqs, H))], -1))
    p = np.exp(beta)
    v1 = bf(rng.uniform(1.0, 2.0, (seqs, H, d)) * rng.choice([-1.0, 1.0], (seqs, H, d)))
    v2 = bf(-v1 / p[..., 1:2])
    v3 = bf(-(v1 + p[..., 1:2] * v2) / p[..., 2:3])
    v = np.stack([v1, v2, v3], 2)
    k = bf(rng.standard_normal(v.shape))
    got, ref = run(k, v, beta, np.zeros((seqs, H, d)), torch.bfloat16, width)
    bound = 24 * U * np.abs(v1) / p.sum(-1)[..., None] + 2.0 ** -8 * np.abs(ref)
    worst = (np.abs(got - ref) / bound).max()
    log(f"  weights: worst error {worst:.2f} of the bound")
    assert worst <= 1.0


@pytest.mark.parametrize("seqs,width", KERNELS)
def test_rotated_queries(seqs, width):
    """A query of one feature a, keys of one feature x and of none: after the
    rotation one product scale a x cos(phi) remains, some hundreds, against the
    second entry's bias of the same size.  The logit is off by 2e-7 scale a x
    (the cosine), 6 U of it (rotation, scale, bias and its sum, each half a
    step) and three parts summed in a step each (6 U); equal weights turn half
    of that into output.  A query of 16 bits is off by up to 2^-17."""
    rng = np.random.default_rng(seqs + width)
    H, d, theta, scale = 8, 64, 1e6, 0.125
    pos = rng.integers(0, 131072, seqs).astype(np.float64)
    q, k, v = np.zeros((seqs, H, d)), np.zeros((seqs, H, 2, d)), np.zeros((seqs, H, 2, d))
    beta, size = np.zeros((seqs, H, 2)), np.zeros((seqs, H, 1))
    phi = pos[:, None] * theta ** (-2.0 * np.arange(d // 2) / d)
    for s in range(seqs):
        for h in range(H):
            e = rng.choice(np.flatnonzero(np.abs(np.cos(phi[s])) > 0.8))
            a, x = bf(rng.uniform(16.0, 32.0)), bf(rng.uniform(64.0, 128.0))
            q[s, h, e], k[s, h, 0, e] = a, x
            beta[s, h, 1] = f32(scale * a * x * np.cos(phi[s, e]))
            size[s, h] = scale * a * x
    v[:, :, 0] = bf(rng.uniform(1.0, 2.0, (seqs, H, d)))
    v[:, :, 1] = -v[:, :, 0]
    got, ref = run(k, v, beta, q, torch.bfloat16, width, pos, theta, scale)
    bound = np.abs(v[:, :, 0]) * (0.5 * (2e-7 + 12 * U) * size + 12 * U) + 2.0 ** -8 * np.abs(ref)
    worst = (np.abs(got - ref) / bound).max()
    log(f"  rotated queries: worst error {worst:.2f} of the bound")
    assert worst <= 1.0


@pytest.mark.parametrize("seqs,width", KERNELS)
def test_small_weights(seqs, width):
    """fp32: a weight of e^-3 .. e^-60 beside one of 1 whose value is 0, so that
    the output is the small weight.  The exponential is off by 3 U (the
    instruction's step and its correction), the sum, its reciprocal, the two
    products and the store by a step or half of one each: 9 U."""
    rng = np.random.default_rng(seqs + width)
    H, d = 8, 64
    beta = f32(np.stack([np.zeros((seqs, H)), rng.uniform(-60.0, -3.0, (seqs, H))], -1))
    v = np.zeros((seqs, H, 2, d))
    v[:, :, 1] = f32(rng.uniform(1.0, 2.0, (seqs, H, d)))
    got, ref = run(f32(rng.standard_normal(v.shape)), v, beta, np.zeros((seqs, H, d)), torch.float32, width)
    worst = (np.abs(got - ref) / np.abs(ref)).max() / (12 * U)
    log(f"  small weights: worst error {worst:.2f} of the bound")
    assert worst <= 1.0
