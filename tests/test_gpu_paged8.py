"""GPU parity of the 8-bit paged cache (still_paged8_append, still_paged8_gather,
still_paged8_attend) against the fp64 oracle.

Bars, from the arithmetic:
* append: equal codes and scales.  The key is rotated in 64 bits on both sides and rounded to
  32; the two differ by about 1e-11 (angles of 1e5 rad), so one number in 10^4 rounds to the
  other 32-bit neighbour, and a code or scale differs only where that lies on a border
  between two codes (one in 2^20) or scales: not once in these tests' 10^6 numbers.
* gather: equal; a code times a power of two is a bf16 number.
* attention: products of bf16 numbers (codes, and queries or weights in parts that hold all of
  their bits) summed in 32 bits.  A logit is off by scale sum|q k| times 2 d 2^-24 (d sums, the
  scales, the bias and the maximum), 4e-7 more for a rotated query, its exponential by 2^-22 and
  by what rounding its argument takes (1.25 2^-24 of it, less than the first term), a sum over n
  entries, at least four of them in parallel, by (n / 4 + 64) 2^-24.  The output: twice that
  times max|v|, and its own half step.  The log of the sum: that, and 2^-23 of itself.
* attention, 2-norm over the whole output: half a step is at most 2^-8 / sqrt(3) = 2.26e-3 rms
  in bf16, so 2.5e-3; in fp32 1e-5.
"""
import numpy as np
import pytest
import torch

from oracle import paged as O, paged8 as O8
from paper_2606_07878_amd import binding, configs
from tests.helpers import log
from tests.paged8_cases import DT, E4M3, Paged8, equal, f64

pytestmark = pytest.mark.gpu

BF16, FP32 = configs.MODE_BF16, configs.MODE_FP32
HALF_STEP = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}


# ---- append ----------------------------------------------------------------

def check_append(c, k, v, offsets=None, positions=None, theta=0.0, beta=None, table=None, lens=None):
    table, lens = c.table if table is None else table, c.lens if lens is None else lens
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    pools, bias = [x.cuda() for x in c.pools()], dev(c.beta)
    binding.paged8_append(k, v, *pools, table.cuda(), lens.cuda(), offsets=dev(offsets), positions=dev(positions),
                          rope_theta=theta, beta=beta, beta_pages=bias)
    torch.cuda.synchronize()
    want = O8.append(f64(k), f64(v), *(f64(x) for x in c.pools()), table.cpu().numpy(), lens.cpu().numpy(),
                     None if offsets is None else offsets.numpy(), None if positions is None else positions.numpy(),
                     theta, f64(beta), f64(c.beta))
    for name, got, ref in zip(("k", "v", "k_scales", "v_scales", "beta"), pools + [bias], want):
        if ref is not None:
            np.testing.assert_array_equal(f64(got), ref, err_msg=name)
    return pools


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d,H,P", [(64, 1, 16), (128, 8, 16), (128, 3, 64), (256, 2, 32), (64, 5, 4096)])
def test_append_one_token_each(mode, d, H, P):
    """A decode step: one token per sequence, at a block's and a page's first and last slot."""
    log(f"append8 step mode={mode} d={d} H={H} P={P}")
    c = Paged8(10, [1, P, P + 1, 2 * P, 2 * P - 1, 9], H, d, P, beta=False)
    pos = torch.tensor([0.0, 5.0, 131072.25, 1e6, -3.0, 77.0], dtype=torch.float64)
    k = c.rows(6, mode)
    k[1] *= 300.0          # the blocks grow
    check_append(c, k.cuda(), c.rows(6, mode).cuda(), positions=pos, theta=1e6)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_append_ragged_prompts_with_bias(mode, d):
    log(f"append8 prompts mode={mode} d={d}")
    lens, new = [90, 33, 40, 16, 250, 7], [90, 1, 23, 0, 200, 7]
    c = Paged8(11, lens, 2, d, 32)
    n = sum(new)
    off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
    pos = torch.arange(n, dtype=torch.float64) * 3 + 130000
    size = torch.exp2(torch.randint(-12, 9, (n, 1, 1), generator=c.g).float())
    check_append(c, (c.rows(n, mode) * size).to(DT[mode]).cuda(), (c.rows(n, mode) * size).to(DT[mode]).cuda(), offsets=off,
                 positions=pos, theta=1e4, beta=torch.randn(n, 2, generator=c.g).cuda())


@pytest.mark.parametrize("per", [7, 8, 9, 31])
def test_append_equal_runs_without_offsets(per):
    """Runs around the length from which 16 tokens share a workgroup."""
    log(f"append8 runs of {per}")
    c = Paged8(12, [per + 5 * s for s in range(40)], 2, 64, 64, beta=False)
    check_append(c, c.rows(40 * per).cuda(), c.rows(40 * per).cuda())


@pytest.mark.parametrize("seqs", [63, 64, 65, 200])
def test_append_finds_the_sequence_among_many(seqs):
    """Runs of 0 to 40 tokens, so that one workgroup's tokens belong to many sequences, some empty."""
    log(f"append8 among {seqs}")
    rng = np.random.default_rng(seqs)
    new = rng.choice([0, 0, 0, 1, 1, 2, 40], seqs)
    new[:3] = [40, 40, 40]
    new[-30:-20] = 0
    lens = new + rng.integers(0, 30, seqs)
    new = np.concatenate([new, [8 * seqs]])        # (long enough a mean for workgroups of 16)
    lens = np.concatenate([lens, [8 * seqs]])
    c = Paged8(13, lens, 1, 64, 16, beta=False)
    off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
    check_append(c, c.rows(int(off[-1])).cuda(), c.rows(int(off[-1])).cuda(), offsets=off)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("seqs", [80, 128, 200])
@pytest.mark.parametrize("busy", [(0,), (5,), (-1,), (40, 41), (0, -1), (3, 70)])
def test_append_to_a_batch_of_idle_sequences(mode, seqs, busy):
    """Prompts in a table of which all other sequences get nothing: 64 and more start within one
    workgroup's 16 tokens, in front of, between and behind the ones that have some."""
    log(f"append8 mode={mode} {len(busy)} of {seqs} have tokens")
    rng = np.random.default_rng(seqs)
    new, held = np.zeros(seqs, int), rng.integers(0, 30, seqs)
    for i, s in enumerate(busy):
        new[s] = (8 * seqs + 5) // len(busy) + 3 * i + 1
    assert new.sum() % 16 and new.sum() > 256 and new.sum() >= 8 * seqs
    c = Paged8(19, held + new, 1, 64, 16)
    n = int(new.sum())
    off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
    check_append(c, c.rows(n, mode).cuda(), c.rows(n, mode).cuda(), offsets=off, positions=torch.arange(n, dtype=torch.float64),
                 theta=1e4, beta=torch.randn(n, 1, generator=c.g).cuda())


def test_append_of_as_many_tokens_as_an_int_counts():
    """2^31 - 1 tokens, one row over and over; the last entries have a place, those in front of the tables do not."""
    n = (1 << 31) - 1
    for lens, last in (([40], []), ([5, 23, 17], [n - 40, n - 17]), ([7] + [0] * 70 + [20], [n - 9] * 70 + [n - 9])):
        c = Paged8(49, lens, 1, 64, 16, beta=False)
        off = torch.tensor([0, *last, n], dtype=torch.int32)
        row = c.rows(1).cuda()
        want = [x.clone() for x in c.cuda().pools()]
        new = np.minimum(lens, np.diff(off.numpy()))      # of them with a place
        few = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
        binding.paged8_append(row.expand(int(few[-1]), 1, 64), row.expand(int(few[-1]), 1, 64), *want, c.table, c.lens, offsets=few)
        torch.cuda.synchronize()
        log(f"append8 of 2^31 - 1 tokens to {len(lens)} sequences")
        binding.paged8_append(row.expand(n, 1, 64), row.expand(n, 1, 64), *c.pages(), offsets=off.cuda())
        torch.cuda.synchronize()
        assert all(equal(a, b) if a.dtype == E4M3 else torch.equal(a, b) for a, b in zip(c.pools(), want))


def test_append_strided_rows_and_no_bias_given():
    c = Paged8(14, [40, 33], 3, 128, 16)
    qkv = torch.randn(9, 12 * 128, generator=c.g).bfloat16().cuda()
    k, v = (qkv[:, a * 128:(a + 3) * 128].unflatten(1, (3, 128)) for a in (5, 9))
    off = torch.tensor([0, 4, 9], dtype=torch.int32)
    check_append(c, k, v, offsets=off)
    heads = torch.randn(3, 9, 128, generator=c.g).cuda()
    check_append(c, heads.transpose(0, 1), heads.flip(0).transpose(0, 1), offsets=off)


def test_append_skips_what_has_no_place():
    """Entries in front of the table, behind it and on absent pages; tokens outside every sequence."""
    c = Paged8(15, [5, 70, 40, 20], 2, 64, 16, width=4)
    c.table[2, 1] = -1
    c.table[3, 1] = c.n_pages
    off = torch.tensor([2, 12, 20, 40, 44], dtype=torch.int32)
    check_append(c, c.rows(50).cuda(), c.rows(50).cuda(), offsets=off)
    check_append(c, c.rows(50).cuda(), c.rows(50).cuda(), offsets=off, lens=torch.tensor([-4, 2 ** 31 - 1, 9, -2 ** 31], dtype=torch.int32))


def test_append_offsets_that_make_no_sense_stay_inside():
    """They may write anything into the sequences' pages, and nothing anywhere else."""
    for off in ([5, 0, 90, -7, 3], [0, 0, 0, 0, 0], [-50, 900, 900, 900, 2000], [2 ** 31 - 1] * 5, [-2 ** 31, 0, 64, 64, 2 ** 31 - 1]):
        c = Paged8(16, [64] * 4, 2, 64, 16, spare=5)
        k0 = c.k.clone()
        c.cuda()
        binding.paged8_append(c.rows(64).cuda(), c.rows(64).cuda(), *c.pages(), offsets=torch.tensor(off, dtype=torch.int32).cuda(),
                              beta_pages=c.beta)
        torch.cuda.synchronize()
        others = sorted(set(range(c.n_pages)) - set(c.table.cpu().flatten().tolist()))
        assert equal(c.k[others], k0[others])


def test_append_numbers_at_the_ends_of_their_range():
    """Zeros, infinities and NaN, the largest and smallest numbers, numbers on the borders of scales."""
    c = Paged8(17, [48], 1, 64, 16, beta=False)
    x = torch.zeros(48, 1, 64)
    x[16:32] = torch.randn(16, 1, 64, generator=c.g)
    x[17, 0, :6] = torch.tensor([float("inf"), float("-inf"), float("nan"), 448.0, -448.0, 3.0])
    x[32, 0, :3] = torch.tensor([3.3895e38, -3.3895e38, 1.0])
    x[33:48, 0] = 2.0 ** -80
    check_append(c, x.bfloat16().cuda(), x.bfloat16().cuda())
    x[0, 0, 0], x[16:32] = 2.0 ** -126, 0.0
    x[16, 0, :2] = torch.tensor([448.5, 2.0 ** -140])
    pools = check_append(c, x.cuda(), x.cuda())
    assert float(pools[2][int(c.table[0, 0])].max()) == 2.0 ** -100
    # tokens one by one: a NaN among them, growing and shrinking numbers
    for n in range(1, 34):
        row = torch.full((1, 1, 64), 2.0 ** ((n * 7) % 19 - 9))
        row[0, 0, n] = float("nan") if n % 5 == 0 else 0.3
        got = check_append(c, row.cuda(), row.cuda(), lens=torch.tensor([n], dtype=torch.int32))
        c.k, c.v, c.ks, c.vs = (y.cpu() for y in got)


def test_append_nothing():
    c = Paged8(18, [40], 2, 64, 16).cuda()
    before = c.k.clone()
    binding.paged8_append(c.rows(0).cuda(), c.rows(0).cuda(), *c.pages(), beta_pages=c.beta)
    assert equal(c.k, before)


# ---- gather ------------------------------------------------------------------

@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d,H,P,start,n", [(64, 1, 16, 0, 300), (128, 8, 16, 37, 64), (256, 3, 64, 5, 290), (128, 2, 128, 299, 21)])
def test_gather(mode, d, H, P, start, n):
    c = Paged8(20, [40, 300], H, d, P, width=-(-320 // P))
    c.table[1, min(2, c.table.shape[1] - 1)] = -7
    want = [*c.values(), f64(c.beta)]
    c.cuda()
    got = binding.paged8_gather(*c.pages(), 1, n, start=start, dtype=DT[mode], beta_pages=c.beta)
    for g, x in zip(got, want):
        np.testing.assert_array_equal(f64(g), O.gather(x, c.table.cpu().numpy(), c.lens.cpu().numpy(), 1, start, n))
    out = tuple(torch.full_like(x, float("nan")) for x in got[:2])
    assert binding.paged8_gather(*c.pages(), 1, n, start=start, out=out) is out
    assert torch.equal(out[0], got[0]) and torch.equal(out[1], got[1])


def test_append_after_gather_gives_the_same_codes():
    """What a block stands for is what it holds: dense rows of it, appended elsewhere, are its codes."""
    c = Paged8(21, [64, 64], 2, 128, 16, beta=False)
    want = c.k.clone()
    c.cuda()
    K, V = binding.paged8_gather(*c.pages(), 0, 64)
    binding.paged8_append(K.transpose(0, 1), V.transpose(0, 1), *c.pools(), c.table[1:].contiguous(), c.lens[1:].contiguous())
    again = binding.paged8_gather(*c.pages(), 1, 64)
    assert torch.equal(again[0], K) and torch.equal(again[1], V)
    assert equal(c.k[c.table[0].long()], want[c.table[0].cpu().long()])


# ---- attention ---------------------------------------------------------------

def bound_of(c, q, K, tn, ln, scale, theta):
    """What a weight, and a log of a sum, may be off by."""
    n, qk = 1, 0.0
    for s in range(tn.shape[0]):
        L = min(max(int(ln[s]), 0), tn.shape[1] * c.P)
        if not L:
            continue
        n = max(n, L)
        rows = O.gather(K, tn, ln, s, 0, L)
        nq = q.shape[0] // tn.shape[0]
        qs = np.abs(f64(q)[s * nq:(s + 1) * nq])
        if theta:
            qs = qs + np.roll(qs, c.d // 2, axis=-1)
        for h in range(q.shape[1]):
            y = qs[:, h] @ np.abs(np.nan_to_num(rows[h // (q.shape[1] // c.H)])).T
            qk = max(qk, y.max())
    return (scale or c.d ** -0.5) * qk * (2 * c.d * 2.0 ** -24 + (4e-7 if theta else 0.0)) + 2.0 ** -22 + (n / 4 + 64) * 2.0 ** -24


def check_attend(c, q, causal=False, scale=0.0, qpos=None, theta=0.0, beta=True, **kw):
    mode = FP32 if q.dtype == torch.float32 else BF16
    K, V = c.values()
    tn, ln = c.table.cpu().numpy(), c.lens.cpu().numpy()
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    bp = c.beta if beta else None
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    got = binding.paged8_attend(q.cuda(), *(x.cuda() for x in c.pages()), causal=causal, scale=scale, beta_pages=dev(bp),
                                q_positions=dev(qpos), rope_theta=theta, lse=lse, **kw)
    torch.cuda.synchronize()
    ref = O.attend(f64(q), K, V, tn, ln, causal, scale, f64(bp), f64(qpos), theta)
    ref_lse = O8.lse(f64(q), K, tn, ln, causal, scale, f64(bp), f64(qpos), theta)
    g, gl = f64(got), f64(lse)
    assert got.shape == q.shape and got.dtype == q.dtype and got.is_contiguous()
    assert np.array_equal(np.isnan(g), np.isnan(ref)), "NaN in other places than the oracle's"
    assert np.array_equal(np.isneginf(gl), np.isneginf(ref_lse))
    off = bound_of(c, q, K, tn, ln, scale, theta)
    vmax = np.nanmax(np.abs(V)) if V.size else 0.0
    excess = np.nanmax(np.abs(g - ref) - HALF_STEP[mode] * np.abs(ref) - 2 * vmax * off)
    fine = np.isfinite(ref_lse)
    over = (np.abs(gl[fine] - ref_lse[fine]) - off - 2.0 ** -23 * np.abs(ref_lse[fine])).max(initial=-1.0)
    norm = np.linalg.norm(np.nan_to_num(ref))
    rel = np.linalg.norm(np.nan_to_num(g) - np.nan_to_num(ref)) / (norm or 1.0)
    log(f"  attend8 rel {rel:.3e}  worst excess {excess:.3e} of {2 * vmax * off:.2e}, lse {over:.3e} of {off:.2e}")
    assert excess <= 0.0 and over <= 0.0
    assert rel <= (2.5e-3 if mode == BF16 else 1e-5)
    return got


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq", [(1, 1), (4, 1), (3, 5), (16, 1), (8, 4), (1, 32), (17, 1)])
def test_attend_rows_and_widths(mode, d, group, nq):
    log(f"attend8 mode={mode} d={d} group={group} nq={nq}")
    c = Paged8(30, [1200, 77, 0], 2, d, 32)
    check_attend(c, c.rows(3 * nq, mode, heads=2 * group), causal=nq > 1)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("P,n", [(16, 1), (16, 16), (32, 17), (64, 129), (16, 511), (256, 1025), (4096, 4097)])
def test_attend_lengths(mode, P, n):
    log(f"attend8 lengths mode={mode} P={P} n={n}")
    c = Paged8(31, [n, max(n - 1, 0), 1], 2, 128, P)
    check_attend(c, c.rows(6, mode, heads=8), causal=True)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("group,nq,d", [(4, 1, 128), (2, 8, 256), (8, 4, 64), (5, 5, 128)])
def test_attend_rotates_queries(mode, group, nq, d):
    log(f"attend8 rotated mode={mode} d={d}")
    c = Paged8(32, [900, 2000, 30], 2, d, 64)
    check_attend(c, c.rows(3 * nq, mode, heads=2 * group), causal=True, qpos=131000.0 + torch.arange(3 * nq, dtype=torch.float64),
                 theta=1e6)


@pytest.mark.parametrize("seqs,longest", [(1, 40000), (5, 9000), (300, 500), (70, 3000)])
def test_attend_parts_of_many_and_long_sequences(seqs, longest):
    """Sequences cut into parts, and several in one part."""
    log(f"attend8 seqs={seqs} longest={longest}")
    rng = np.random.default_rng(seqs)
    lens = rng.integers(0, min(longest, 200), seqs)
    lens[seqs // 2] = longest
    c = Paged8(33, lens, 1, 64, 64)
    check_attend(c, c.rows(seqs, heads=2))


@pytest.mark.parametrize("nq", [1, 8])
def test_attend_streaming_loads(nq):
    """A table that could hold more than the memory-side cache."""
    c = Paged8(34, [3000, 5], 2, 128, 64)
    c.table = torch.cat([c.table, torch.zeros(2, 9000, dtype=torch.int32)], dim=1)
    check_attend(c, c.rows(2 * nq, heads=8), causal=True)


ROWS = [(1, 1), (4, 1), (3, 5), (8, 4), (1, 32)]


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq", ROWS)
@pytest.mark.parametrize("theta", [0.0, 1e6])
def test_attend_short_tables(mode, d, group, nq, theta):
    """Up to 1024 entries: a workgroup takes all of a sequence."""
    log(f"attend8 short mode={mode} d={d} group={group} nq={nq} theta={theta}")
    c = Paged8(45, [1000, 77, 0, 512, 3], 2, d, 32)
    check_attend(c, c.rows(5 * nq, mode, heads=2 * group), causal=nq > 1, theta=theta,
                 qpos=131000.0 + torch.arange(5 * nq, dtype=torch.float64) if theta else None)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq,theta", [(1, 1, 0.0), (4, 1, 1e6), (8, 4, 1e6), (1, 32, 0.0)])
def test_attend_many_short_tables(mode, d, group, nq, theta):
    """Up to 512 entries and more than 256 sequences and heads: a wave takes all of one."""
    log(f"attend8 many short mode={mode} d={d} group={group} nq={nq} theta={theta}")
    lens = np.random.default_rng(d).integers(0, 60, 65)
    lens[7] = 500
    c = Paged8(46, lens, 4, d, 16)
    check_attend(c, c.rows(65 * nq, mode, heads=4 * group), causal=nq > 1, theta=theta,
                 qpos=131000.0 + torch.arange(65 * nq, dtype=torch.float64) if theta else None)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("group,nq,theta", [(4, 1, 0.0), (8, 4, 1e6), (1, 32, 0.0)])
def test_attend_streaming_loads_of_other_widths(mode, d, group, nq, theta):
    log(f"attend8 streaming mode={mode} d={d} group={group} nq={nq} theta={theta}")
    c = Paged8(47, [3000, 5], 2, d, 64)
    c.table = torch.cat([c.table, torch.zeros(2, 9000 * 128 // d, dtype=torch.int32)], dim=1)
    check_attend(c, c.rows(2 * nq, mode, heads=2 * group), causal=nq > 1, theta=theta,
                 qpos=131000.0 + torch.arange(2 * nq, dtype=torch.float64) if theta else None)


def test_attend_the_smallest_scales():
    """2^-100, which blocks of zeros and of numbers near them have."""
    c = Paged8(48, [700, 90], 2, 128, 16)
    c.ks, c.vs = c.ks * 2.0 ** -94, c.vs * 2.0 ** -94
    assert float(c.vs.min()) == 2.0 ** -100
    check_attend(c, c.rows(2, FP32, heads=4) * 2.0 ** 90)
    check_attend(c, c.rows(2, heads=4))


def test_attend_any_scales():
    """Scales need not be powers of two to be read."""
    c = Paged8(35, [700, 90], 2, 128, 16)
    c.ks, c.vs = c.ks * 1.37, c.vs * 0.613
    check_attend(c, c.rows(2, FP32, heads=4))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("width", [4, 100])
def test_attend_ignores_what_no_query_sees(bad, width):
    """Codes, scales and bias behind the lengths and on absent pages."""
    c = Paged8(36, [37, 0, 40], 2, 64, 16, width=width, spare=4)
    c.table[2, 1] = -1
    used = np.zeros((c.n_pages, 16), bool)
    for s, n in enumerate(c.lens_list):
        for j in range(n):
            if 0 <= int(c.table[s, j // 16]) < c.n_pages:
                used[int(c.table[s, j // 16]), j % 16] = True
    free = torch.from_numpy(~used)
    c.k.view(torch.uint8).masked_fill_(free[:, None, :, None], 0x7F)
    c.v.view(torch.uint8).masked_fill_(free[:, None, :, None], 0x7F)
    c.beta.masked_fill_(free[:, None], bad)
    none = torch.from_numpy(~used.any(axis=1))
    c.ks[none], c.vs[none] = bad, bad
    assert torch.isfinite(check_attend(c, c.rows(3, heads=4))).all()


def test_attend_bias_of_minus_infinity_and_the_lowest_value():
    c = Paged8(37, [64, 40, 30], 2, 64, 16)
    c.beta[:, :, ::2] = float("-inf")
    c.beta[int(c.table[1, 0])] = torch.finfo(torch.float32).min
    c.beta[c.table[2].long()] = float("-inf")      # leaves nothing
    got = check_attend(c, c.rows(3, heads=4))
    assert not got[2].any()


def test_attend_strided_queries_and_rows_behind():
    c = Paged8(38, [300, 50], 2, 128, 16).cuda()
    qkv = torch.randn(2, 20 * 128, generator=c.g).bfloat16().cuda()
    q = qkv[:, 256:256 + 8 * 128].unflatten(1, (8, 128))
    out = torch.full((5, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((5, 8), 7.0, device="cuda")
    binding.paged8_attend(q, *c.pages(), out=out[:2], lse=lse[:2])
    assert torch.equal(out[:2], binding.paged8_attend(q.contiguous(), *c.pages()))
    assert (out[2:] == 7.0).all() and (lse[2:] == 7.0).all()


def test_pages_past_four_gib():
    """Rows, scales and bias behind 2^32 bytes of codes."""
    H, d, P = 8, 256, 4096
    n_pages = 520                                   # 4.06 GiB each
    k, v = (torch.zeros(n_pages, H, P, d, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ks, vs = (torch.ones(n_pages, H, P // 16, device="cuda") for _ in range(2))
    table, lens = torch.tensor([[519, 3]], dtype=torch.int32, device="cuda"), torch.tensor([4100], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(3)
    rows = torch.randn(4100, H, d, generator=g).bfloat16().cuda()
    binding.paged8_append(rows, -rows, k, v, ks, vs, table, lens)
    K, V = binding.paged8_gather(k, v, ks, vs, table, lens, 0, 4100)
    small = [torch.zeros(2, *x.shape[1:], dtype=torch.uint8, device="cuda").view(E4M3) if x.dtype == E4M3 else torch.ones(2, *x.shape[1:], device="cuda")
             for x in (k, v, ks, vs)]
    near = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    binding.paged8_append(rows, -rows, *small, near, lens)
    assert equal(k[519], small[0][1]) and equal(v[519], small[1][1]) and torch.equal(ks[519], small[2][1])
    assert torch.equal(V, -K)
    q = torch.randn(1, H, d, generator=g).bfloat16().cuda()
    assert torch.equal(binding.paged8_attend(q, k, v, ks, vs, table, lens), binding.paged8_attend(q, *small, near, lens))


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("width", [16, 400])
def test_attend_of_other_caches_gives_the_log_of_the_sum_too(mode, width):
    """lse of paged_attend over pages of q's type: one workgroup a sequence, and parts."""
    c = Paged8(39, [200, 0, 33], 2, 64, 16, width=width)
    K, V = (torch.from_numpy(x).to(DT[mode]) for x in c.values())
    q = c.rows(6, mode, heads=4)
    lse = torch.full((6, 4), float("nan"), device="cuda")
    args = (q.cuda(), K.cuda(), V.cuda(), c.table.cuda(), c.lens.cuda())
    got = binding.paged_attend(*args, causal=True, beta_pages=c.beta.cuda(), lse=lse)
    assert torch.equal(got, binding.paged_attend(*args, causal=True, beta_pages=c.beta.cuda()))
    ref = O8.lse(f64(q), f64(K), c.table.numpy(), c.lens.numpy(), True, 0.0, f64(c.beta))
    off = bound_of(c, q, f64(K), c.table.numpy(), c.lens.numpy(), 0.0, 0.0)
    g = f64(lse)
    assert np.array_equal(np.isneginf(g), np.isneginf(ref))
    fine = np.isfinite(ref)
    assert (np.abs(g[fine] - ref[fine]) <= off + 2.0 ** -23 * np.abs(ref[fine])).all()


def test_attend_is_the_same_every_time_and_on_other_streams():
    c = [Paged8(40 + i, [3000 + 500 * i, 17], 2, 128, 32).cuda() for i in range(2)]
    q = [x.rows(2, heads=8).cuda() for x in c]
    want = [binding.paged8_attend(y, *x.pages(), beta_pages=x.beta) for x, y in zip(c, q)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(binding.STILL_PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [[torch.empty_like(q[i]) for _ in range(10)] for i in range(2)]
    for r in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                binding.paged8_attend(q[i], *c[i].pages(), beta_pages=c[i].beta, workspace=ws[i], out=outs[i][r])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])


def test_steps_captured_in_a_graph_follow_the_lengths():
    """append + attend of a step, captured once and replayed while lengths, positions and inputs
    change in place and eager calls run between."""
    S, H, group, d, P, theta = 4, 2, 4, 128, 16, 1e6
    c = Paged8(62, [100, 1, 600, 0], H, d, P, width=90).cuda()
    other = [x.clone() for x in c.pools()]
    nk, nv, q = c.rows(S).cuda(), c.rows(S).cuda(), c.rows(S, heads=H * group).cuda()
    pos = (c.lens + 7).double()
    ws = torch.empty(binding.STILL_PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(S, H * group, device="cuda")

    def step(pools, o, n):
        binding.paged8_append(nk, nv, *pools, c.table, c.lens, positions=pos, rope_theta=theta)
        return binding.paged8_attend(q, *pools, c.table, c.lens, q_positions=pos, rope_theta=theta, workspace=ws, out=o, lse=n)

    c.lens.add_(1)
    eager_lse = torch.empty_like(lse)
    eager = step(other, None, eager_lse).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step(c.pools(), out, lse)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(5):
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse), f"replay {rep}"
        assert all(equal(a, b) for a, b in zip(c.pools()[:2], other)) and torch.equal(c.ks, other[2])
        c.lens.add_(1 if rep else 30)
        pos.add_(1.0)
        for x in (nk, nv):
            x.copy_(c.rows(S) * 2.0 ** rep)
        q.copy_(c.rows(S, heads=H * group))
        eager = step(other, None, eager_lse).clone()
        torch.cuda.synchronize()


@pytest.mark.parametrize("mode,bits", [(BF16, [0x7F81, -127, 0x7FC0, 0x7FFF]), (FP32, [0x7F800001, -8388607, 0x7FC00000, 0x7FFFFFFF])])
def test_append_every_nan(mode, bits):
    """Signalling and quiet ones of both signs leave the scale alone, whatever holds the largest number."""
    c = Paged8(19, [32], 1, 64, 16, beta=False)
    x = torch.randn(32, 1, 64, generator=c.g).to(DT[mode])
    raw = x.view(torch.int16 if mode == BF16 else torch.int32)
    raw[torch.arange(0, 32, 2), 0, torch.arange(16) * 3] = torch.tensor(bits * 4, dtype=raw.dtype)
    assert x.isnan().sum() == 16
    check_append(c, x.cuda(), x.flip(0).contiguous().cuda())
    check_append(c, x.cuda(), x.flip(0).contiguous().cuda(), positions=torch.arange(32, dtype=torch.float64), theta=1e4)
