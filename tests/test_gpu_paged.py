"""GPU parity of the paged cache (still_paged_append, still_paged_gather,
still_paged_attend, binding.compact_paged) against the fp64 oracle.

Bars, from the arithmetic:
* appended keys: the rotation is fp32 with angles reduced in fp64.  Its sine
  and cosine are off by at most 2e-7, its two products and their sum round by
  2^-24 each: 4e-7 (|a| + |b|) for the pair (a, b); the store to bf16 adds half
  a step, 2^-8 relative.  Values, unrotated keys and bias are copies: equal.
* gathered rows are copies: equal.
* attention, per element: the stored output's half step (2^-8 relative in bf16,
  2^-24 in fp32) plus the weights' errors times 2 max|v| (numerator and
  denominator).  A weight is off by what its logit is off: scale sum|q k| times
  d 2^-24 (fp32 sums; doubled for the scale, the bias and the maximum) and, for
  rotated bf16 queries, 2^-16 (two bf16 parts) + 4e-7; by the exponential's
  2^-22; in bf16 mode by 2^-16 (a weight in two bf16 parts); and by its sum over
  n entries, at least four of them in parallel: (n / 4 + 64) 2^-24.
* attention, 2-norm over the whole output: half a step is at most 2^-8 / sqrt(3)
  = 2.26e-3 rms in bf16, so 2.5e-3; in fp32 1e-5, the bar of still_attend.
"""
import numpy as np
import pytest
import torch

from oracle import paged as O
from paper_2606_07878_amd import configs, synth
from tests.helpers import dev_tensor, log, weights_to_device
from tests.paged_cases import Paged

pytestmark = pytest.mark.gpu

BF16, FP32 = configs.MODE_BF16, configs.MODE_FP32
HALF_STEP = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}


def f64(x):
    return None if x is None else x.double().cpu().numpy()


# ---- append ----------------------------------------------------------------

def check_append(c, k, v, offsets=None, positions=None, theta=0.0, beta=None, table=None, lens=None):
    from paper_2606_07878_amd import binding
    table, lens = c.table if table is None else table, c.lens if lens is None else lens
    kp, vp, bp, _, _ = c.f64()
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    K, V, B = c.k.cuda(), c.v.cuda(), dev(c.beta)
    binding.paged_append(k, v, K, V, table.cuda(), lens.cuda(), offsets=dev(offsets), positions=dev(positions),
                         rope_theta=theta, beta=beta, beta_pages=B)
    torch.cuda.synchronize()
    off = None if offsets is None else offsets.numpy()
    pos = None if positions is None else positions.numpy()
    rk, rv, rb = O.append(f64(k), f64(v), kp, vp, table.numpy(), lens.numpy(), off, pos, theta, f64(beta), bp)
    gk = f64(K)
    if theta:
        sums = np.abs(f64(k))
        h = c.d // 2
        sums = sums[..., :h] + sums[..., h:]
        bound = np.zeros(rk.shape)     # |a| + |b| of the new entries, through the same append without rotation
        spread, _, _ = O.append(np.concatenate([sums, sums], -1), f64(v), np.zeros_like(rk), vp, table.numpy(),
                                lens.numpy(), off)
        bound += 4e-7 * spread + np.where(spread > 0, HALF_STEP[c.mode] * np.abs(rk), 0.0)
        worst = (np.abs(gk - rk) - bound).max()
        log(f"  append worst excess {worst:.3e}")
        assert worst <= 0.0
    else:
        np.testing.assert_array_equal(gk, rk)
    np.testing.assert_array_equal(f64(V), rv)
    if bp is not None:
        np.testing.assert_array_equal(f64(B), rb)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d,H,P", [(64, 1, 16), (128, 8, 16), (128, 3, 64), (256, 2, 32), (64, 5, 4096)])
def test_append_one_token_each(mode, d, H, P):
    """A decode step: one token per sequence, sequences of length 1, at a page's first and last slot."""
    log(f"append step mode={mode} d={d} H={H} P={P}")
    c = Paged(10, [1, P, P + 1, 2 * P, 2 * P - 1], H, d, P, mode, beta=False)
    pos = torch.tensor([0.0, 5.0, 131072.25, 1e6, -3.0], dtype=torch.float64)
    check_append(c, c.rows(5).cuda(), c.rows(5).cuda(), positions=pos, theta=1e6)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_append_ragged_prompts_with_bias(mode, d):
    """Odd counts (0, 1 and more than a page among them), tokens before the first and behind the last sequence."""
    log(f"append ragged mode={mode} d={d}")
    new, first = [3, 0, 1, 50, 17], 2
    c = Paged(11, [20, 7, 1, 61, 17], 3, d, 16, mode)
    off = torch.tensor(np.cumsum([first] + new), dtype=torch.int32)
    n = first + sum(new) + 5
    pos = torch.from_numpy(c.rng.uniform(0, 2e5, n))
    beta = torch.randn(n, 3, generator=c.g).cuda()
    check_append(c, c.rows(n).cuda(), c.rows(n).cuda(), off, pos, 1e4 if d == 256 else 1e6, beta)


def test_append_without_bias_clears_it():
    c = Paged(12, [5, 9], 2, 64, 16, BF16)
    check_append(c, c.rows(4).cuda(), c.rows(4).cuda())


@pytest.mark.parametrize("mode", [BF16, FP32])
def test_append_strided_rows(mode):
    """Slices of a fused projection, and the compactor's [H, t, d] with its [H, t] bias."""
    c = Paged(13, [40], 4, 128, 16, mode)
    fused = torch.randn(33, 16 * 128, generator=c.g).to(c.k.dtype).cuda()
    k, v = fused[:, 8 * 128:12 * 128].view(33, 4, 128), fused[:, 12 * 128:].view(33, 4, 128)
    check_append(c, k, v, positions=torch.arange(33, dtype=torch.float64), theta=1e6)
    ck, cv = (torch.randn(4, 40, 128, generator=c.g).to(c.k.dtype).cuda().transpose(0, 1) for _ in range(2))
    check_append(c, ck, cv, beta=torch.randn(4, 40, generator=c.g).cuda().t())


def test_append_skips_what_has_no_place():
    """Absent pages (numbers below 0 and past the pool), entries before the
    start of the sequence and past its table: skipped, the rest written."""
    c = Paged(14, [40, 10, 48, 300], 2, 128, 16, BF16)
    table = c.table[:, :3].contiguous()
    table[0, 1] = -1
    table[2, 2] = c.n_pages
    lens = torch.tensor([40, 3, 48, 60], dtype=torch.int32)
    check_append(c, c.rows(80).cuda(), c.rows(80).cuda(), positions=torch.arange(80, dtype=torch.float64), theta=1e4,
                 table=table, lens=lens)
    check_append(c, c.rows(4).cuda(), c.rows(4).cuda(), table=table,
                 lens=torch.tensor([-2**31, 0, 2**31 - 1, 49], dtype=torch.int32))


@pytest.mark.parametrize("seqs", [63, 64, 65, 130, 5000])
def test_append_finds_the_sequence_among_many(seqs):
    new = np.random.default_rng(seqs).integers(0, 3, seqs)
    new[seqs - 1] = 2
    lens = new + np.random.default_rng(seqs + 1).integers(0, 30, seqs)
    c = Paged(17, [32] * seqs, 1, 64, 16, BF16, beta=False)
    n = int(new.sum())
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    check_append(c, c.rows(n).cuda(), c.rows(n).cuda(), off, lens=torch.from_numpy(lens.astype(np.int32)))


def test_append_offsets_that_make_no_sense_stay_inside():
    """Offsets that fall, are negative or pass the tokens: every token is skipped or lands in its sequence's pages."""
    from paper_2606_07878_amd import binding
    c = Paged(18, [30, 30, 30], 2, 64, 16, BF16, beta=False).cuda()
    guard = [x.clone() for x in (c.k, c.v)]
    k = c.rows(12).cuda()
    for off in ([5, 2, 9, 1], [-7, -3, 2, 2**31 - 1], [0, 100, 50, 12], [2**31 - 1, 0, 0, 0]):
        binding.paged_append(k, k, c.k, c.v, c.table, c.lens, offsets=torch.tensor(off, dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    others = torch.ones(c.n_pages, dtype=torch.bool, device="cuda")
    others[c.table.reshape(-1).long()] = False
    assert torch.equal(c.k[others], guard[0][others]) and torch.equal(c.v[others], guard[1][others])


def test_append_nothing():
    c = Paged(15, [4, 4], 2, 64, 16, BF16)
    check_append(c, c.rows(0).cuda(), c.rows(0).cuda())


def test_append_table_rows_of_a_wider_table():
    c = Paged(16, [33, 40, 20], 2, 64, 16, BF16, width=9)
    check_append(c, c.rows(2).cuda(), c.rows(2).cuda(), table=c.table[::2, :4], lens=torch.tensor([33, 20], dtype=torch.int32))


# ---- gather ----------------------------------------------------------------

@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d,H,P,start,n", [(64, 1, 16, 0, 1), (128, 8, 16, 5, 200), (256, 3, 64, 63, 130),
                                           (128, 2, 32, 250, 70), (64, 7, 128, 0, 0)])
def test_gather(mode, d, H, P, start, n):
    """Starts inside a page, ends past the length (250 + 70 > 300) and in absent pages."""
    from paper_2606_07878_amd import binding
    log(f"gather mode={mode} d={d} H={H} P={P} start={start} n={n}")
    c = Paged(20, [40, 300], H, d, P, mode, width=-(-320 // P))
    c.table[1, min(2, c.table.shape[1] - 1)] = -7
    k, v, b, table, lens = c.f64()
    c.cuda()
    got = binding.paged_gather(*c.pages(), 1, n, start=start, beta_pages=c.beta)
    assert len(got) == 3
    for g, x in zip(got, (k, v, b)):
        np.testing.assert_array_equal(f64(g), O.gather(x, table, lens, 1, start, n))
    out = tuple(torch.full_like(x, float("nan")) for x in got[:2])
    assert binding.paged_gather(*c.pages(), 1, n, start=start, out=out) is out
    assert torch.equal(out[0], got[0]) and torch.equal(out[1], got[1])


# ---- attention --------------------------------------------------------------

def check_attend(c, q, causal=False, scale=0.0, qpos=None, theta=0.0, beta=True, table=None, lens=None, **kw):
    from paper_2606_07878_amd import binding
    table, lens = c.table if table is None else table, c.lens if lens is None else lens
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    bp = c.beta if beta else None
    got = binding.paged_attend(q.cuda(), dev(c.k), dev(c.v), table.cuda(), lens.cuda(), causal=causal, scale=scale,
                               beta_pages=dev(bp), q_positions=dev(qpos), rope_theta=theta, **kw)
    torch.cuda.synchronize()
    tn, ln = table.cpu().numpy(), lens.cpu().numpy()
    # unseen slots may hold anything: the oracle never reads them
    ref = O.attend(f64(q), f64(c.k), f64(c.v), tn, ln, causal, scale, f64(bp), f64(qpos), theta)
    g = f64(got)
    assert got.shape == q.shape and got.dtype == q.dtype and got.is_contiguous()
    assert np.array_equal(np.isnan(g), np.isnan(ref)), "NaN in other places than the oracle's"
    S, n = tn.shape[0], int(max(1, min(max(ln.max(), 0), tn.shape[1] * c.P)))
    cap = tn.shape[1] * c.P
    vmax = qk = 0.0
    group = q.shape[1] // c.H
    for s in range(S):
        L = min(max(int(ln[s]), 0), cap)
        if L:
            K, V = O.gather(f64(c.k), tn, ln, s, 0, L), O.gather(f64(c.v), tn, ln, s, 0, L)
            vmax = max(vmax, np.abs(V).max())
            qs = np.abs(f64(q)[s * (q.shape[0] // S):(s + 1) * (q.shape[0] // S)])
            if theta:
                qs = qs + np.roll(qs, c.d // 2, axis=-1)
            for h in range(q.shape[1]):
                qk = max(qk, (qs[:, h] @ np.abs(K[h // group]).T).max())
    sc = scale or c.d ** -0.5
    weight = sc * qk * (2 * c.d * 2.0 ** -24 + (4e-7 + (2.0 ** -16 if c.mode == BF16 else 0.0) if theta else 0.0))
    weight += 2.0 ** -22 + (n / 4 + 64) * 2.0 ** -24 + (2.0 ** -16 if c.mode == BF16 else 0.0)
    excess = (np.abs(g - ref) - HALF_STEP[c.mode] * np.abs(ref) - 2 * vmax * weight)
    norm = np.linalg.norm(ref)
    rel = np.linalg.norm(g - ref) / norm if norm else np.linalg.norm(g - ref)
    log(f"  attend rel {rel:.3e}  worst excess {np.nanmax(excess):.3e} (bound of the weights {2 * vmax * weight:.2e})")
    assert np.nanmax(excess) <= 0.0
    assert rel <= (2.5e-3 if c.mode == BF16 else 1e-5)
    return got


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq", [(1, 1), (4, 1), (3, 5), (16, 1), (8, 3), (1, 32)])
def test_attend_rows_and_widths(mode, d, group, nq):
    """Ragged lengths with one, none and fewer entries than queries among them; pages that end inside a tile."""
    log(f"attend mode={mode} d={d} group={group} nq={nq}")
    lens = [1, 0, 129, 31, 33, 700, 3]
    c = Paged(30, lens, 2, d, 16, mode)
    check_attend(c, c.rows(len(lens) * nq, 2 * group), causal=nq > 1)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("P", [16, 32, 128, 1024])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 1000])
def test_attend_lengths(mode, P, n):
    c = Paged(31, [n], 3, 64, P, mode)
    check_attend(c, c.rows(1, 6))


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("group,nq,d", [(4, 1, 128), (4, 8, 128), (2, 3, 256)])
def test_attend_rotates_queries(mode, group, nq, d):
    """At logical positions behind a long compacted prefix, another one per token."""
    c = Paged(32, [719, 40, 200], 2, d, 64, mode)
    n = 3 * nq
    pos = torch.from_numpy(131072.0 + c.rng.integers(0, 5000, n))
    check_attend(c, c.rows(n, 2 * group), causal=nq > 1, qpos=pos.double(), theta=1e6)


def test_attend_long_and_short_together():
    """One sequence far longer than the others: its work is split, theirs is not."""
    c = Paged(33, [20011, 1, 5, 300, 64], 2, 128, 64, BF16)
    check_attend(c, c.rows(5, 8))


@pytest.mark.parametrize("seqs", [255, 257, 600])
def test_attend_many_sequences(seqs):
    c = Paged(34, [int(x) for x in np.random.default_rng(seqs).integers(0, 90, seqs)], 1, 64, 16, BF16)
    check_attend(c, c.rows(seqs, 2))


@pytest.mark.parametrize("heads,seqs,long", [(8, 300, 9000), (2, 520, 5000)])
def test_attend_more_sequences_than_workgroups_per_head(heads, seqs, long):
    """Several rounds of lengths, parts that hold many sequences, a long one among them split over many."""
    lens = [int(x) for x in np.random.default_rng(seqs).integers(0, 120, seqs)]
    lens[seqs // 2], lens[seqs // 2 + 1] = long, 0
    c = Paged(51, [120] * seqs, heads, 64, 16, BF16)
    # one long sequence over all the other pages: shared pages are fine to read
    width = -(-long // 16)
    table = torch.zeros(seqs, width, dtype=torch.int32)
    table[:, :8] = c.table
    table[seqs // 2] = torch.from_numpy(c.rng.integers(0, c.n_pages, width).astype(np.int32))
    check_attend(c, c.rows(seqs, heads), table=table, lens=torch.tensor(lens, dtype=torch.int32))


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("group,nq,d", [(4, 8, 256), (1, 32, 128), (1, 32, 64), (2, 4, 128), (1, 3, 256)])
def test_attend_several_short_sequences_per_workgroup_with_rotation(mode, group, nq, d):
    """The query rows and angles of one sequence after another in the same LDS."""
    lens = [5, 30, 16, 1, 0, 33, 9, 2, 31, 64, 7, 12, 40]
    c = Paged(52, lens, 1, d, 16, mode)
    n = len(lens) * nq
    pos = torch.from_numpy(c.rng.uniform(0, 1e5, n))
    check_attend(c, c.rows(n, group), causal=True, qpos=pos, theta=1e6)
    wide = torch.zeros(len(lens), 80, dtype=torch.int32)     # capacity above 1024: parts instead of whole sequences
    wide[:, : c.table.shape[1]] = c.table
    check_attend(c, c.rows(n, group), causal=True, qpos=pos, theta=1e6, table=wide)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 100, 511, 768])
def test_attend_narrow_and_wide_tables(mode, d, n):
    """The same sequence through a table of its own pages and through a wide one (other kernels)."""
    c = Paged(53, [n, 3], 2, d, 16, mode)
    wide = torch.full((2, 300), -1, dtype=torch.int32)
    wide[:, : c.table.shape[1]] = c.table
    q = c.rows(2, 8)
    a, b = check_attend(c, q), check_attend(c, q, table=wide)
    assert (a.double() - b.double()).abs().max() <= 2 * HALF_STEP[mode] * a.double().abs().max() + 1e-5


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq", [(4, 1), (3, 5), (4, 8), (1, 32)])
def test_attend_many_short_sequences(mode, d, group, nq):
    """Enough sequences and heads that a wave takes each (90 x 3), the table's columns short."""
    lens = [int(x) for x in np.random.default_rng(d + nq).integers(0, 80, 90)]
    lens[:4] = [0, 1, 16, 79]
    c = Paged(56, lens, 3, d, 16, mode)
    n = 90 * nq
    pos = torch.from_numpy(c.rng.uniform(0, 1e5, n))
    rot = nq != 5
    check_attend(c, c.rows(n, 3 * group), causal=nq > 1, qpos=pos if rot else None, theta=1e4 if rot else 0.0)


def test_attend_many_heads():
    """More KV heads than workgroups: one part per head, nothing to join."""
    c = Paged(54, [70, 300], 600, 64, 16, BF16, width=70)
    check_attend(c, c.rows(2, 600))


@pytest.mark.parametrize("width", [1, 70])
def test_attend_as_many_sequences_as_a_call_takes(width):
    """65535 sequences of one entry (a few of none): each row is its value.
    Short tables take a wave per sequence, wide ones parts."""
    from paper_2606_07878_amd import binding
    n, pages = 65535, 1000
    g = torch.Generator(device="cuda").manual_seed(5)
    k = torch.randn(pages, 1, 16, 64, generator=g, device="cuda").bfloat16()
    v = torch.randn(pages, 1, 16, 64, generator=g, device="cuda").bfloat16()
    table = torch.randint(0, pages, (n, width), generator=g, device="cuda", dtype=torch.int32)
    lens = torch.ones(n, dtype=torch.int32, device="cuda")
    lens[::1000] = 0
    q = torch.randn(n, 1, 64, generator=g, device="cuda").bfloat16()
    out = binding.paged_attend(q, k, v, table, lens)
    want = v[table[:, 0].long(), 0, 0] * lens[:, None]
    assert torch.equal(out[:, 0], want)


def test_attend_is_the_same_every_time():
    c = Paged(55, [9000, 1, 300, 40], 2, 128, 32, BF16)
    q = c.rows(4, 8)
    a = check_attend(c, q)
    from paper_2606_07878_amd import binding
    c.cuda()
    outs = [binding.paged_attend(q.cuda(), *c.pages(), beta_pages=c.beta) for _ in range(20)]
    assert all(torch.equal(o, a) for o in outs)


def test_attend_without_bias_and_with_a_scale():
    c = Paged(35, [100, 400], 3, 128, 32, BF16)
    check_attend(c, c.rows(2, 3), beta=False, scale=0.3)


def test_attend_everything_empty():
    c = Paged(36, [64, 64], 2, 64, 16, BF16)
    for lens in ([0, 0], [-5, 0]):
        out = check_attend(c, c.rows(2, 4), lens=torch.tensor(lens, dtype=torch.int32))
        assert not out.any()


def test_attend_length_past_the_table_counts_as_the_table():
    c = Paged(37, [96, 96], 2, 64, 16, FP32)
    check_attend(c, c.rows(2, 4), lens=torch.tensor([2**31 - 1, 97], dtype=torch.int32))


@pytest.mark.parametrize("mode", [BF16, FP32])
def test_attend_absent_pages_are_not_seen(mode):
    """Holes at the start, inside and at the end, a sequence of nothing but holes; causal rows that see holes only."""
    c = Paged(38, [100, 150, 60, 40], 2, 128, 16, mode)
    c.table[0, :3] = -1
    c.table[1, 4] = 2**31 - 1
    c.table[1, 9] = c.n_pages
    c.table[2, :] = -2**31
    c.table[3, 0] = -1     # entries 0 .. 15 absent
    check_attend(c, c.rows(4, 4))
    check_attend(c, c.rows(4 * 8, 8), causal=True)


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_attend_ignores_what_no_query_sees(mode, bad):
    """Slots past a sequence's length, absent and foreign pages hold NaN or infinity."""
    lens = [5, 17, 130, 0, 40]
    c = Paged(39, lens, 2, 128, 16, mode)
    seen = torch.zeros(c.n_pages, c.P, dtype=torch.bool)
    c.table[4, 1] = -1
    for s, n in enumerate(lens):
        for j in range(n):
            p = int(c.table[s, j // 16])
            if p >= 0:
                seen[p, j % 16] = True
    hide = ~seen[:, None, :].expand(-1, 2, -1)
    c.k[hide], c.v[hide], c.beta[hide] = bad, bad, bad
    out = check_attend(c, c.rows(5, 8))
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("mode", [BF16, FP32])
def test_attend_bias_of_minus_infinity_and_the_lowest_value(mode):
    """-inf removes an entry; a sequence of nothing but -inf gives zeros; a
    sequence whose entries all carry the lowest finite value weighs them as if
    they carried none (the logits vanish beside it: equal weights)."""
    c = Paged(40, [50, 33, 64], 2, 64, 16, mode)
    low = torch.finfo(torch.float32).min
    for s, val in ((1, float("-inf")), (2, low)):
        for p in c.table[s]:
            c.beta[int(p)] = val
    c.beta[int(c.table[0, 1]), :, ::2] = float("-inf")
    out = check_attend(c, c.rows(3, 4))
    assert not out[1].any()
    mean = np.stack([f64(c.v)[c.table[2].numpy(), h].reshape(-1, 64).mean(axis=0) for h in (0, 0, 1, 1)])
    assert np.abs(f64(out)[2] - mean).max() <= 2e-2 * np.abs(mean).max()


def test_attend_large_logits():
    """Logits of hundreds: one entry wins; the running maximum moves far."""
    c = Paged(41, [500, 900], 2, 128, 32, FP32)
    check_attend(c, c.rows(2, 4) * 4.0, scale=4.0)


@pytest.mark.parametrize("mode", [BF16, FP32])
def test_attend_strided_queries(mode):
    c = Paged(42, [77, 200, 31], 2, 128, 16, mode)
    fused = torch.randn(3 * 4, 12 * 128, generator=c.g).to(c.k.dtype).cuda()
    q = fused[:, : 8 * 128].view(12, 8, 128)
    a = check_attend(c, q, causal=True)
    b = check_attend(c, q.contiguous(), causal=True)
    assert torch.equal(a, b)


def test_attend_does_not_touch_rows_behind_the_last_sequence():
    from paper_2606_07878_amd import binding
    c = Paged(43, [77, 0, 31], 2, 128, 16, BF16).cuda()
    q = c.rows(8, 8).cuda()
    out = torch.full((8, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    binding.paged_attend(q[:3], *c.pages(), out=out[:3])
    torch.cuda.synchronize()
    assert (out[3:] == 7.0).all() and not (out[:3] == 7.0).all(dim=-1).any()
    assert not out[1].any()


@pytest.mark.parametrize("mode", [BF16, FP32])
def test_pool_past_four_gib(mode):
    """Entries whose byte and element offsets pass 32 bits: append, gather and attention there."""
    from paper_2606_07878_amd import binding
    H, P, d = 8, 16, 128
    es = 2 if mode == BF16 else 4
    pages = (1 << 32) // (H * P * d * 2) + 40          # more than 2^31 elements, 2^32 bytes
    log(f"pool of {pages * H * P * d * es / 2**30:.1f} GiB")
    c = Paged(44, [60, 90], H, d, P, mode)
    small = c.n_pages
    k = torch.zeros(pages, H, P, d, dtype=c.k.dtype, device="cuda")
    v = torch.zeros_like(k)
    beta = torch.zeros(pages, H, P, device="cuda")
    k[pages - small:], v[pages - small:], beta[pages - small:] = c.k.cuda(), c.v.cuda(), c.beta.cuda()
    table, lens = (c.table + pages - small).cuda(), c.lens.cuda()
    q = c.rows(2, 32)
    got = binding.paged_attend(q.cuda(), k, v, table, lens, beta_pages=beta)
    want = check_attend(c, q)
    assert torch.equal(got, want)
    rows = binding.paged_gather(k, v, table, lens, 1, 90)
    np.testing.assert_array_equal(f64(rows[0]), O.gather(f64(c.k), c.table.numpy(), c.lens.numpy(), 1, 0, 90))
    nk = c.rows(2).cuda()
    binding.paged_append(nk, nk, k, v, table, lens, beta_pages=beta)
    back = binding.paged_gather(k, v, table, lens, 1, 1, start=89)
    assert torch.equal(back[0][:, 0], nk[1]) and torch.equal(back[1][:, 0], nk[1])
    assert not k[:pages - small].any()


# ---- refusals that need GPU tensors -------------------------------------------

def test_binding_refuses_rows_that_do_not_fit():
    from paper_2606_07878_amd import binding
    c = Paged(50, [20, 30], 2, 64, 16, BF16).cuda()
    q, k, P = c.rows(2, 4).cuda(), c.rows(2).cuda(), c.pages()

    def refused(status, f, *args, **kw):
        with pytest.raises(binding.StillError) as e:
            f(*args, **kw)
        assert e.value.status == status, str(e.value)

    refused(-2, binding.paged_attend, q[:, :3], *P)                     # 3 query heads, 2 KV heads
    refused(-2, binding.paged_attend, c.rows(3, 4).cuda(), *P)          # 3 tokens, 2 sequences
    refused(-2, binding.paged_attend, q[:, :, :32], *P)
    refused(-3, binding.paged_attend, q.float(), *P)
    refused(-1, binding.paged_attend, q.cpu(), *P)
    refused(-1, binding.paged_attend, q.transpose(0, 1).contiguous().transpose(0, 1), *P)
    refused(-2, binding.paged_attend, q, *P, q_positions=torch.zeros(3, dtype=torch.float64, device="cuda"))
    refused(-3, binding.paged_attend, q, *P, q_positions=torch.zeros(2, device="cuda"))
    refused(-1, binding.paged_attend, q, *P, rope_theta=1e6)            # rotation needs positions
    refused(-2, binding.paged_attend, q, *P, out=torch.empty_like(q[:1]))
    refused(-1, binding.paged_attend, q, *P, workspace=torch.empty(1 << 20, dtype=torch.uint8))
    refused(-5, binding.paged_attend, c.rows(2 * 17, 4).cuda(), *P)     # 34 query rows per KV head
    refused(-1, binding.paged_append, k, k, *P, rope_theta=1e6)
    refused(-2, binding.paged_append, k[:1], k[:1], *P)                 # one token, two sequences
    refused(-2, binding.paged_append, k, k[:1], *P)
    refused(-3, binding.paged_append, k, k.float(), *P)
    refused(-2, binding.paged_append, k, k, *P, offsets=torch.zeros(2, dtype=torch.int32, device="cuda"))
    refused(-1, binding.paged_append, k, k, *P, beta=torch.zeros(2, 2, device="cuda"))   # a cache without bias
    refused(-2, binding.paged_append, k, k, *P, beta=torch.zeros(2, 3, device="cuda"), beta_pages=c.beta)
    refused(-1, binding.paged_attend, q[:1].expand(2, 4, 64), *P)       # the same token twice
    refused(-1, binding.paged_attend, q, *P, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[::2])
    refused(-2, binding.paged_attend, q, P[0], P[1], P[2][:1].expand(2, -1), P[3])       # one table row for both
    refused(-2, binding.paged_gather, *P, 0, 5, start=1 << 32)
    refused(-2, binding.paged_gather, *P, 1 << 32, 5)
    refused(-2, binding.paged_gather, *P, 2, 5)
    refused(-2, binding.paged_gather, *P, 0, 33)
    refused(-2, binding.paged_gather, *P, 0, -1)
    refused(-2, binding.paged_gather, *P, 0, 5, out=(k, k, k))
    refused(-2, binding.paged_gather, *P, 0, 5, out=(k, k))


def test_binding_refuses_no_sequences_and_counts_past_32_bits():
    from paper_2606_07878_amd import binding
    c = Paged(66, [20, 30], 2, 64, 16, BF16).cuda()
    none = (c.k, c.v, c.table[:0], c.lens[:0])
    row = c.rows(1).cuda()
    many = row.expand((1 << 32) + 2, 2, 64)                             # the low 32 bits say 2
    before = c.k.clone()
    for f, args in ((binding.paged_attend, (c.rows(2, 4)[:0].cuda(), *none)), (binding.paged_append, (row[:0], row[:0], *none)),
                    (binding.paged_gather, (*none, 0, 0)), (binding.paged_append, (many, many, *c.pages()))):
        with pytest.raises(binding.StillError) as e:
            f(*args)
        assert e.value.status == -2, str(e.value)
    assert torch.equal(c.k, before)


def test_compact_paged_changes_nothing_where_a_layers_bias_pages_do_not_fit():
    from paper_2606_07878_amd import binding
    w = configs.shrink(configs.get_workload(1), n_tokens=100, t=32)
    c = Paged(67, [100], w.cfg.n_kv_heads, w.cfg.head_dim, 16, BF16).cuda()
    W = weights_to_device(synth.make_weights(w, 0, t=32), BF16)
    k2, v2 = c.k.clone(), c.v.clone()
    pos = torch.arange(100, dtype=torch.float64, device="cuda")
    before = c.k.clone(), c.v.clone(), c.beta.clone()
    with pytest.raises(binding.StillError) as e:
        binding.compact_paged(w.cfg, [W, W], [c.k, k2], [c.v, v2], c.table, c.lens, 0, 100, pos, w.rope_theta, 32,
                              beta_pages=[c.beta, c.beta[:1]])
    assert e.value.status == -2
    torch.cuda.synchronize()
    assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1]) and torch.equal(c.beta, before[2])
    assert c.lens.tolist() == [100]


# ---- together ----------------------------------------------------------------

def test_decode_loop_matches_the_oracle():
    """Prompts, then steps of one token each (append, then attend), over sequences that cross pages."""
    from paper_2606_07878_amd import binding
    S, H, group, d, P, theta = 3, 2, 4, 128, 16, 1e6
    c = Paged(60, [30, 14, 1], H, d, P, BF16, width=4)
    k, v, b, table, lens = c.f64()
    c.cuda()
    lens_h = np.array([30, 14, 1])
    for step in range(6):
        nk, nv, q = c.rows(S), c.rows(S), c.rows(S, H * group)
        lens_h = lens_h + 1
        c.lens.add_(1)
        pos = torch.from_numpy(lens_h + 5000.0)
        binding.paged_append(nk.cuda(), nv.cuda(), *c.pages(), positions=pos.cuda(), rope_theta=theta, beta_pages=c.beta)
        got = binding.paged_attend(q.cuda(), *c.pages(), beta_pages=c.beta, q_positions=pos.cuda(), rope_theta=theta)
        k, v, b = O.append(f64(nk), f64(nv), k, v, table, lens_h, None, pos.numpy(), theta, None, b)
        # the stored keys are bf16
        k = torch.from_numpy(k).to(torch.bfloat16).double().numpy()
        ref = O.attend(f64(q), k, v, table, lens_h, False, 0.0, b, pos.numpy(), theta)
        rel = np.linalg.norm(f64(got) - ref) / np.linalg.norm(ref)
        assert rel <= 4e-3, f"step {step}: {rel:.2e}"   # output rounding 2.3e-3, keys that round the other way


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("start,end,bias", [(0, None, False), (0, 300, True), (37, 300, False)])
def test_compact_paged_is_compact_subrange_in_the_pages(mode, start, end, bias):
    """Two layers: the same entries as the dense calls give, the rest of the pool untouched."""
    from paper_2606_07878_amd import binding
    w = configs.shrink(configs.get_workload(1), n_tokens=350, t=32)
    n, t, L, H, d, P = 350, 32, 2, w.cfg.n_kv_heads, w.cfg.head_dim, 16
    e = n if end is None else end
    caches = [synth.make_cache(w, l, n_tokens=n) for l in range(L)]
    wts = [weights_to_device(synth.make_weights(w, l, t=t), mode) for l in range(L)]
    wb = [dev_tensor(synth.make_beta_weight(w, l), mode) for l in range(L)]
    pos = torch.from_numpy(caches[0]["positions"]).cuda()
    c = Paged(61, [40, n, 90], H, d, P, mode).cuda()
    pages = [[x.clone() for x in (c.k, c.v, c.beta)] for _ in range(L)]
    dense = []
    one = torch.tensor([n], dtype=torch.int32, device="cuda")
    for l in range(L):
        K, V = dev_tensor(caches[l]["K"], mode), dev_tensor(caches[l]["V"], mode)
        bias0 = torch.randn(H, n, device="cuda")
        binding.paged_append(K.transpose(0, 1), V.transpose(0, 1), *pages[l][:2], c.table[1:2], one, beta=bias0.t(),
                             beta_pages=pages[l][2])
        dense.append((K, V, bias0))
    before = [[x.clone() for x in p] for p in pages]
    kw = dict(w_beta=wb, beta_max=2.0, mass_alpha=0.5) if bias else {}
    got_pos = binding.compact_paged(w.cfg, wts, [p[0] for p in pages], [p[1] for p in pages], c.table, c.lens, 1, n,
                                    pos, w.rope_theta, t, start=start, end=end, beta_pages=[p[2] for p in pages], **kw)
    m = n - (e - start) + t
    assert c.lens.tolist() == [40, m, 90] and got_pos.shape == (m,)
    for l in range(L):
        K, V, b0 = dense[l]
        rk, rv, rp = binding.compact_subrange(w.cfg, wts[l], K, V, pos, w.rope_theta, t, start, e, mode=mode)
        if bias:
            _, _, _, (nb,) = binding.compact_model_beta(w.cfg, [wts[l]], [K[:, start:e].contiguous()],
                                                        [V[:, start:e].contiguous()], pos[start:e].contiguous(),
                                                        w.rope_theta, t, [wb[l]], 2.0, 0.5, mode=mode)
        else:
            nb = torch.zeros(H, t, device="cuda")
        k, v, b = binding.paged_gather(*pages[l][:2], c.table, c.lens, 1, m, beta_pages=pages[l][2])
        assert torch.equal(k, rk) and torch.equal(v, rv) and torch.equal(got_pos, rp)
        assert torch.equal(b[:, start:start + t], nb)
        assert torch.equal(b[:, :start], b0[:, :start]) and torch.equal(b[:, start + t:], b0[:, e:])
        others = torch.ones(c.n_pages, dtype=torch.bool, device="cuda")
        others[c.table[1].long()] = False
        for x, y in zip(pages[l], before[l]):
            assert torch.equal(x[others], y[others])


def test_compact_paged_changes_nothing_where_a_layer_is_refused():
    from paper_2606_07878_amd import binding
    w = configs.shrink(configs.get_workload(1), n_tokens=100, t=32)
    H, d = w.cfg.n_kv_heads, w.cfg.head_dim
    c = Paged(64, [100], H, d, 16, BF16).cuda()
    good, bad = (weights_to_device(synth.make_weights(w, 0, t=t), BF16) for t in (32, 16))
    k2, v2 = c.k.clone(), c.v.clone()
    pos = torch.arange(100, dtype=torch.float64, device="cuda")
    before = c.k.clone(), c.v.clone()
    with pytest.raises(binding.StillError) as e:
        binding.compact_paged(w.cfg, [good, bad], [c.k, k2], [c.v, v2], c.table, c.lens, 0, 100, pos, w.rope_theta, 32)
    assert e.value.status == -2
    other = Paged(65, [100], H + 1, d, 16, BF16).cuda()
    with pytest.raises(binding.StillError) as e:
        binding.compact_paged(w.cfg, [good], [other.k], [other.v], other.table, other.lens, 0, 100, pos, w.rope_theta, 32)
    assert e.value.status == -2
    torch.cuda.synchronize()
    assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1]) and c.lens.tolist() == [100]


def test_steps_captured_in_a_graph_follow_the_lengths():
    """append + attend of a step, captured once and replayed while lengths,
    positions and inputs change in place and eager calls run between."""
    from paper_2606_07878_amd import binding
    S, H, group, d, P, theta = 4, 2, 4, 128, 16, 1e6
    c = Paged(62, [100, 1, 600, 0], H, d, P, BF16, width=40).cuda()
    k2, v2 = c.k.clone(), c.v.clone()
    nk, nv, q = c.rows(S).cuda(), c.rows(S).cuda(), c.rows(S, H * group).cuda()
    pos = (c.lens + 7).double()
    ws = torch.empty(binding.STILL_PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)

    def step(k, v, o):
        binding.paged_append(nk, nv, k, v, c.table, c.lens, positions=pos, rope_theta=theta)
        return binding.paged_attend(q, k, v, c.table, c.lens, q_positions=pos, rope_theta=theta, workspace=ws, out=o)

    c.lens.add_(1)
    eager = step(k2, v2, None).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step(c.k, c.v, out)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(5):
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), f"replay {rep}"
        assert torch.equal(c.k, k2) and torch.equal(c.v, v2)
        c.lens.add_(1 if rep else 30)
        pos.add_(1.0)
        nk.copy_(c.rows(S))
        nv.copy_(c.rows(S))
        q.copy_(c.rows(S, H * group))
        eager = step(k2, v2, None).clone()
        torch.cuda.synchronize()


def test_two_streams_with_their_own_workspaces():
    from paper_2606_07878_amd import binding
    c = [Paged(63 + i, [3000 + 500 * i, 17], 2, 128, 32, BF16).cuda() for i in range(2)]
    q = [x.rows(2, 8).cuda() for x in c]
    want = [binding.paged_attend(y, *x.pages(), beta_pages=x.beta) for x, y in zip(c, q)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(binding.STILL_PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [[torch.empty_like(q[i]) for _ in range(10)] for i in range(2)]
    for r in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                binding.paged_attend(q[i], *c[i].pages(), beta_pages=c[i].beta, workspace=ws[i], out=outs[i][r])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])
