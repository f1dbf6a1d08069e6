"""GPU parity of the entries' scores (still_paged_score, still_paged8_score) and of the eviction by
them (still_paged_evict, still_paged8_evict) against the fp64 oracle.

Bars, from the arithmetic:
* a score: every row's weight is off by its logit's error (scale sum|q k| times 2 d 2^-24, 4e-7 more
  where rotated), the rounding of its argument, which holds the logit and the lse (2^-24 each of
  them, and 2^-24 of their difference), and the exponential's 2^-22; the sum of R rows and the old
  score by (R + 1) 2^-24 of itself.
* kept entries, lengths, moved rows, codes, scales, bias: equal.  A sum of H scores in 64 bits,
  rounded to 32, is the oracle's unless it lies within 2^-50 of a border: not once in 10^5.
"""
import numpy as np
import pytest
import torch

from oracle import paged as O, paged8 as O8
from paper_2606_07878_amd import binding, configs, synth
from tests.helpers import dev_tensor, log, weights_to_device
from tests.paged8_cases import DT, E4M3, Paged8, equal, f64

pytestmark = pytest.mark.gpu

BF16, FP32, E8 = configs.MODE_BF16, configs.MODE_FP32, "e4m3"


def as_type(c, kind):
    """The pages of c in this type: (k, v, k_scales or None, v_scales or None), CPU."""
    if kind == E8:
        return c.pools()
    return (*(torch.from_numpy(x).to(DT[kind]) for x in c.values()), None, None)


# ---- scores --------------------------------------------------------------------

def check_score(c, q, kind, causal=False, scale=0.0, qpos=None, theta=0.0, beta=True, known=None, lse=None):
    k, _, ks, _ = as_type(c, kind)
    K = O8.values(f64(k), f64(ks)) if kind == E8 else f64(k)
    tn, ln = c.table.cpu().numpy(), c.lens.cpu().numpy()
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    bp = c.beta if beta else None
    if lse is None:
        lse = torch.from_numpy(O8.lse(f64(q), K, tn, ln, causal, scale, f64(bp), f64(qpos), theta)).float()
    got = c.scores.cuda().clone()
    binding.paged_score(q.cuda(), lse.cuda(), k.cuda(), got, c.table.cuda(), c.lens.cuda(), causal=causal, scale=scale,
                        k_scales=dev(ks), beta_pages=dev(bp), known=dev(known), q_positions=dev(qpos), rope_theta=theta)
    torch.cuda.synchronize()
    nk = None if known is None else known.numpy()
    ref = O8.score(f64(q), f64(lse), K, f64(c.scores), tn, ln, nk, causal=causal, scale=scale, beta_pages=f64(bp),
                   q_positions=f64(qpos), rope_theta=theta)
    qk = biggest = 0.0
    S, R = tn.shape[0], q.shape[0] // tn.shape[0] * q.shape[1] // c.H
    for s in range(S):
        L = min(max(int(ln[s]), 0), tn.shape[1] * c.P)
        rows = np.abs(np.nan_to_num(O.gather(K, tn, ln, s, 0, L)))
        if L:
            qs = np.abs(f64(q)[s * (q.shape[0] // S):(s + 1) * (q.shape[0] // S)])
            qs = qs + np.roll(qs, c.d // 2, axis=-1) if theta else qs
            qk = max(qk, max((qs[:, h] @ rows[h // (q.shape[1] // c.H)].T).max() for h in range(q.shape[1])))
    fine = f64(lse)[np.isfinite(f64(lse))]
    biggest = 2 * max(np.abs(fine).max(initial=0.0), (scale or c.d ** -0.5) * qk)
    off = (scale or c.d ** -0.5) * qk * (2 * c.d * 2.0 ** -24 + (4e-7 if theta else 0.0)) + 2 * biggest * 2.0 ** -24 + 2.0 ** -22
    added = np.abs(ref - f64(c.scores))
    g = f64(got)
    assert np.array_equal(np.isnan(g), np.isnan(ref))
    excess = np.nanmax(np.abs(g - ref) - off * np.minimum(R, added + f64(c.scores)) - (R + 1) * 2.0 ** -24 * np.abs(ref))
    log(f"  score worst excess {excess:.3e}, of a weight {off:.2e}")
    assert excess <= 0.0
    return got


@pytest.mark.parametrize("kind,mode", [(BF16, BF16), (FP32, FP32), (E8, BF16), (E8, FP32)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq", [(1, 1), (2, 1), (4, 1), (1, 3), (5, 1), (2, 4), (7, 1), (3, 3), (3, 5), (8, 4), (17, 1), (1, 32)])
def test_score_rows_and_widths(kind, mode, d, group, nq):
    log(f"score kind={kind} mode={mode} d={d} group={group} nq={nq}")
    c = Paged8(50, [1200, 77, 0, 3], 2, d, 32)
    check_score(c, c.rows(4 * nq, mode, heads=2 * group), kind, causal=nq > 1, known=torch.tensor([1199, 70, 0, 0], dtype=torch.int32))


@pytest.mark.parametrize("kind,mode", [(BF16, BF16), (FP32, FP32), (E8, BF16), (E8, FP32)])
@pytest.mark.parametrize("P,n", [(16, 1), (16, 16), (64, 129), (16, 511), (16, 513), (4096, 4097)])
def test_score_lengths_rotated(kind, mode, P, n):
    log(f"score lengths kind={kind} P={P} n={n}")
    c = Paged8(51, [n, max(n - 1, 0), 1], 2, 128, P)
    check_score(c, c.rows(6, mode, heads=8), kind, causal=True, qpos=131000.0 + torch.arange(6, dtype=torch.float64), theta=1e6)


@pytest.mark.parametrize("seqs,longest", [(1, 40000), (300, 500), (70, 3000)])
def test_score_of_many_and_long_sequences(seqs, longest):
    rng = np.random.default_rng(seqs)
    lens = rng.integers(0, min(longest, 200), seqs)
    lens[seqs // 2] = longest
    c = Paged8(52, lens, 1, 64, 64)
    check_score(c, c.rows(seqs, heads=2), E8)


def test_score_of_more_chunks_than_workgroups():
    """More pairs of a sequence and a head than workgroups a chunk each: they loop."""
    c = Paged8(53, [1100] * 65, 65, 64, 16, beta=False, spare=0)
    got = check_score(c, c.rows(65, heads=65), E8, beta=False)
    assert torch.isfinite(got).all()


def test_score_leaves_what_no_row_sees():
    """Slots behind the lengths, absent pages, rows whose sum is empty; NaN where nothing is read."""
    c = Paged8(54, [37, 0, 40, 20], 2, 64, 16, width=5)
    c.table[2, 1] = -1
    c.beta[int(c.table[0, 2]), :, 5:] = float("nan")
    c.scores[int(c.table[0, 2]), :, 5:] = float("nan")
    c.scores[int(c.table[0, 4])] = float("nan")
    c.scores[int(c.table[3, 1]), :, 3] = float("nan")      # of an entry that is new
    c.beta[int(c.table[3, 0])] = float("-inf")
    c.beta[int(c.table[3, 1])] = float("-inf")             # nothing left: the row's lse is minus infinity
    got = check_score(c, c.rows(4, heads=4), E8, known=torch.tensor([37, 0, 40, 19], dtype=torch.int32))
    assert torch.isnan(got[int(c.table[0, 2]), :, 5:]).all() and not got[int(c.table[3, 1]), :, 3].any()


def test_score_takes_what_attention_gives():
    """The lse of paged8_attend and of paged_attend; the weights of a row sum to 1."""
    for kind in (E8, BF16, FP32):
        mode = BF16 if kind == E8 else kind
        c = Paged8(55, [900, 40], 2, 128, 16)
        k, v, ks, vs = (None if x is None else x.cuda() for x in as_type(c, kind))
        q, lse = c.rows(2, mode, heads=8).cuda(), torch.empty(2, 8, device="cuda")
        seqs = (c.table.cuda(), c.lens.cuda())
        if kind == E8:
            binding.paged8_attend(q, k, v, ks, vs, *seqs, lse=lse)
        else:
            binding.paged_attend(q, k, v, *seqs, lse=lse)
        scores = torch.zeros_like(c.scores).cuda()
        binding.paged_score(q, lse, k, scores, *seqs, k_scales=ks)
        for s, n in enumerate(c.lens_list):
            total = scores[c.table[s].long().cuda()].double().sum(dim=(0, 2))
            # 4 rows; a weight's relative error is that of its logit against the one in the lse
            assert (total - 4.0).abs().max() < 4 * 1e-5, total


def test_score_is_the_same_every_time():
    c = Paged8(56, [3000, 17], 2, 128, 32).cuda()
    q, lse = c.rows(2, heads=8).cuda(), torch.randn(2, 8, generator=c.g).cuda() + 5
    outs = []
    for _ in range(5):
        s = c.scores.clone()
        binding.paged_score(q, lse, c.k, s, c.table, c.lens, k_scales=c.ks, beta_pages=c.beta)
        outs.append(s)
    assert all(torch.equal(o, outs[0]) for o in outs)


# ---- eviction -------------------------------------------------------------------

def check_evict(c, kind, keep, first=0, recent=0, shared=False, beta=True, lens=None):
    lens = c.lens if lens is None else lens
    pools = as_type(c, kind)
    tn, ln = c.table.cpu().numpy(), lens.cpu().numpy()
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    k, v, ks, vs = (None if x is None else x.cuda().clone() for x in pools)
    scores, bp = c.scores.cuda().clone(), dev(c.beta.clone()) if beta else None
    kept, new = binding.paged_evict(k, v, c.table.cuda(), lens.cuda(), scores, keep, first=first, recent=recent, shared=shared,
                                    k_scales=ks, v_scales=vs, beta_pages=bp)
    torch.cuda.synchronize()
    ids, lengths = O8.evict(tn, ln, f64(c.scores).astype(np.float32), keep, first, recent, shared)
    np.testing.assert_array_equal(kept.cpu().numpy(), ids)
    np.testing.assert_array_equal(new.cpu().numpy(), lengths)
    for name, got, was in (("scores", scores, c.scores), ("beta", bp, c.beta if beta else None)):
        if was is not None:
            np.testing.assert_array_equal(f64(got), O8.move(f64(was), tn, ids), err_msg=name)
    for name, got, scale, was, had in (("k", k, ks, pools[0], pools[2]), ("v", v, vs, pools[1], pools[3])):
        if had is None:
            np.testing.assert_array_equal(f64(got), O8.move(f64(was), tn, ids), err_msg=name)
            continue
        want, now = O8.move8(f64(was), f64(had), tn, ids)
        np.testing.assert_array_equal(f64(scale), now, err_msg=name + " scales")
        np.testing.assert_array_equal(f64(got), want, err_msg=name)
    return kept, new


KINDS = [BF16, FP32, E8]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,H,P", [(64, 1, 16), (128, 3, 64), (256, 2, 32), (64, 2, 4096)])
@pytest.mark.parametrize("shared", [False, True])
def test_evict_types_and_widths(kind, d, H, P, shared):
    log(f"evict kind={kind} d={d} H={H} P={P} shared={shared}")
    c = Paged8(60, [700, 333, 200, 5, 0, 201], H, d, P)
    check_evict(c, kind, 200, first=4, recent=30, shared=shared)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (16, 0, 0), (17, 3, 14), (63, 0, 63), (64, 64, 0),
                                               (299, 0, 0), (300, 1, 1), (5000, 4000, 1000)])
def test_evict_how_many(kind, keep, first, recent):
    """One entry, none to choose, all but one, more than there are."""
    c = Paged8(61, [300, 299, 1, 64], 2, 64, 16)
    check_evict(c, kind, keep, first, recent)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("seqs,n,keep", [(1, 9000, 4000), (1, 17000, 900), (1, 40000, 123), (40, 600, 512), (3, 5000, 4999),
                                         (3, 9000, 8000), (33, 17000, 100)])
def test_evict_long_and_many(kind, seqs, n, keep):
    """Lists by 256 and by 1024 threads, moves in column pieces and in several chunks."""
    log(f"evict kind={kind} {seqs} of {n} to {keep}")
    c = Paged8(62, [n - 7 * s for s in range(seqs)], 2, 64, 64, spare=1)
    check_evict(c, kind, keep, first=4, recent=min(64, keep // 4), shared=seqs == 3)


def test_evict_long_lists_of_equal_scores():
    """Ties across threads, waves and rounds; more keys than are put aside share the bits found."""
    c = Paged8(67, [40000, 12000], 1, 64, 64, spare=1)
    c.scores = (torch.arange(c.n_pages * 64) * 7919 % 5).float().reshape(c.n_pages, 1, 64) / 4 + 1
    check_evict(c, BF16, 20000, shared=True)
    check_evict(c, BF16, 11000)
    c.scores.fill_(1.0)
    check_evict(c, E8, 9000, first=3, recent=50)


def test_evict_equal_and_odd_scores():
    """Ties go to the earlier entry; zeros of both signs are equal; NaN and minus infinity come last, infinity first."""
    c = Paged8(63, [500, 500, 500, 500], 1, 64, 16)
    for s, x in enumerate((torch.zeros(500), (torch.arange(500) % 3).float(), torch.full((500,), float("nan")), torch.randn(500, generator=c.g))):
        x = torch.cat([x, torch.zeros(12)])
        if s == 0:
            x[::2] = -0.0
        if s == 3:
            x[5::7], x[6::7], x[0::7], x[1::7] = float("nan"), float("-inf"), float("inf"), 2.0 ** -140
        c.scores[c.table[s].long()] = x.reshape(32, 1, 16)
    for keep in (100, 167, 400):
        check_evict(c, BF16, keep)
    check_evict(c, E8, 300, first=1, recent=1, shared=True)


def test_evict_absent_pages():
    """Entries on them come last and move as zeros; places on them are not written."""
    c = Paged8(64, [160, 160, 40], 2, 64, 16, spare=4)
    c.table[0, 3], c.table[0, 7], c.table[1, 0], c.table[2, 1] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31
    for kind in KINDS:
        check_evict(c, kind, 120, recent=40)
        check_evict(c, kind, 140)


def test_evict_of_absent_entries_leaves_positive_scales():
    """A block whose entries all lay on absent pages: zeros, of the smallest scale, to which a later append adds."""
    c = Paged8(68, [320, 200], 2, 64, 16, spare=4)
    c.table[0, 17:20] = -1
    kept, new = check_evict(c, E8, 100, recent=64)
    c.cuda()
    binding.paged_evict(c.k, c.v, c.table, c.lens, c.scores, 100, recent=64, k_scales=c.ks, v_scales=c.vs, beta_pages=c.beta,
                        new_lens=c.lens)
    of = c.table[0, :7].long()
    assert (c.ks > 0).all() and (c.vs > 0).all()
    assert (c.ks[of[4:]] == 2.0 ** -100).all() and (c.vs[of[4:]] == 2.0 ** -100).all()
    K, V = binding.paged8_gather(*c.pages(), 0, 100)
    assert K[:, :52].any() and not K[:, 52:].any() and not V[:, 52:].any()
    was = f64(c.ks), f64(c.k)
    lens, row = (c.lens + 5)[:1], c.rows(5).cuda()
    binding.paged8_append(row, row, *c.pools(), c.table[:1], lens, beta_pages=c.beta)
    want = O8.append(f64(row), f64(row), was[1], was[1], was[0], was[0], c.table[:1].cpu().numpy(), lens.cpu().numpy())
    np.testing.assert_array_equal(f64(c.k), want[0])
    np.testing.assert_array_equal(f64(c.ks), want[2])


def test_evict_lengths_outside_the_table_and_in_place():
    c = Paged8(65, [100, 50], 2, 64, 16, width=8)
    lens = torch.tensor([10 ** 6, -4], dtype=torch.int32)
    check_evict(c, BF16, 30, lens=lens)
    c.cuda()
    lens = lens.cuda()
    kept, new = binding.paged_evict(c.k, c.v, c.table, lens, c.scores, 30, k_scales=c.ks, v_scales=c.vs, new_lens=lens)
    assert new is lens and lens.tolist() == [30, 0] and kept.shape == (2, 2, 30)
    assert (kept[1] == -1).all()


def test_evict_nothing_changes_nothing():
    c = Paged8(66, [100, 64], 2, 64, 16).cuda()
    before = [x.clone() for x in (*c.pools(), c.scores, c.beta)]
    check_evict(c, E8, 100)
    for a, b in zip((*c.pools(), c.scores, c.beta), before):
        assert equal(a, b) if a.dtype == E4M3 else torch.equal(a, b)


def test_evict_past_four_gib():
    H, d, P = 8, 256, 4096
    k, v = (torch.zeros(260, H, P, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))   # 4.06 GiB each
    scores = torch.rand(260, H, P, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    table, lens = torch.tensor([[259, 3]], dtype=torch.int32, device="cuda"), torch.tensor([4200], dtype=torch.int32, device="cuda")
    rows = torch.randn(4200, H, d, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    binding.paged_append(rows, -rows, k, v, table, lens)
    K, _ = binding.paged_gather(k, v, table, lens, 0, 4200)
    kept, new = binding.paged_evict(k, v, table, lens, scores, 500, recent=100)
    K2, V2 = binding.paged_gather(k, v, table, new, 0, 500)
    want = torch.gather(K, 1, kept[0].long()[..., None].expand(H, 500, d))
    assert torch.equal(K2, want) and torch.equal(V2, -want)


# ---- together --------------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
def test_decode_loop_with_eviction_matches_the_oracle(kind):
    """Steps of append, attention, score and, where a sequence grows past its budget, eviction."""
    S, H, group, d, P, theta, keep = 3, 2, 4, 64, 16, 1e6, 60
    mode = BF16 if kind == E8 else kind
    c = Paged8(70, [50, 58, 1], H, d, P, width=6)
    k, v, ks, vs = (None if x is None else x.cuda() for x in as_type(c, kind))
    table, lens = c.table.cuda(), c.lens.cuda()
    scores = torch.rand(c.scores.shape, generator=c.g).cuda()
    pos = torch.tensor([130000.0, 70.0, 1.0], dtype=torch.float64)
    lse = torch.empty(S, H * group, device="cuda")
    known = lens.clone()
    for step in range(24):
        nk, nv, q = c.rows(S, mode), c.rows(S, mode), c.rows(S, mode, heads=H * group)
        lens += 1
        seqs = (table, lens)
        before = [f64(x) for x in (k, v, ks, vs, scores)]
        args = dict(positions=pos.cuda(), rope_theta=theta)
        if kind == E8:
            binding.paged8_append(nk.cuda(), nv.cuda(), k, v, ks, vs, *seqs, **args)
            out = binding.paged8_attend(q.cuda(), k, v, ks, vs, *seqs, q_positions=pos.cuda(), rope_theta=theta, lse=lse)
        else:
            binding.paged_append(nk.cuda(), nv.cuda(), k, v, *seqs, **args)
            out = binding.paged_attend(q.cuda(), k, v, *seqs, q_positions=pos.cuda(), rope_theta=theta, lse=lse)
        binding.paged_score(q.cuda(), lse, k, scores, *seqs, k_scales=ks, known=known, q_positions=pos.cuda(), rope_theta=theta)
        tn, ln = table.cpu().numpy(), lens.cpu().numpy()
        if kind == E8:
            want = O8.append(f64(nk), f64(nv), *before[:4], tn, ln, positions=pos.numpy(), rope_theta=theta)
            for a, b in zip((k, v, ks, vs), want):
                np.testing.assert_array_equal(f64(a), b)
        K, V = (O8.values(f64(x), f64(y)) if kind == E8 else f64(x) for x, y in ((k, ks), (v, vs)))
        ref = O.attend(f64(q), K, V, tn, ln, q_positions=pos.numpy(), rope_theta=theta)
        assert np.linalg.norm(f64(out) - ref) <= (2.5e-3 if mode == BF16 else 1e-5) * np.linalg.norm(ref)
        rs = O8.score(f64(q), O8.lse(f64(q), K, tn, ln, q_positions=pos.numpy(), rope_theta=theta), K, before[4], tn, ln,
                      known.cpu().numpy(), q_positions=pos.numpy(), rope_theta=theta)
        assert np.abs(f64(scores) - rs).max() <= 1e-5 * (1 + np.abs(rs).max())
        pos += 1
        known.copy_(lens)
        if step % 8 == 7:
            ids, lengths = O8.evict(tn, ln, f64(scores).astype(np.float32), keep, 2, 16)
            moved = [O8.move8(f64(a), f64(b), tn, ids) if kind == E8 else (O8.move(f64(a), tn, ids), None)
                     for a, b in ((k, ks), (v, vs))]
            kept, _ = binding.paged_evict(k, v, table, lens, scores, keep, first=2, recent=16, k_scales=ks, v_scales=vs, new_lens=lens)
            np.testing.assert_array_equal(kept.cpu().numpy(), ids)
            np.testing.assert_array_equal(lens.cpu().numpy(), lengths)
            for (a, b), x, y in zip(moved, (k, v), (ks, vs)):
                np.testing.assert_array_equal(f64(x), a)
                assert y is None or np.array_equal(f64(y), b)
            known.copy_(lens)


def test_step_with_eviction_captured_in_a_graph():
    """append, attention, score and eviction in place, captured once, replayed with eager work between."""
    S, H, group, d, P, keep = 3, 2, 4, 128, 16, 96
    c = Paged8(71, [100, 60, 95], H, d, P, width=8).cuda()
    nk, nv, q = c.rows(S).cuda(), c.rows(S).cuda(), c.rows(S, heads=H * group).cuda()
    lse = torch.empty(S, H * group, device="cuda")
    ws = torch.empty(binding.STILL_PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    kept = torch.empty(S, H, keep, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    state = [*c.pools(), c.scores, c.lens]
    other = [x.clone() for x in state]

    def step(k, v, ks, vs, scores, lens, out, kept):
        known = lens.clone()
        lens.add_(1)
        binding.paged8_append(nk, nv, k, v, ks, vs, c.table, lens)
        binding.paged8_attend(q, k, v, ks, vs, c.table, lens, workspace=ws, out=out, lse=lse)
        binding.paged_score(q, lse, k, scores, c.table, lens, k_scales=ks, known=known)
        binding.paged_evict(k, v, c.table, lens, scores, keep, first=2, recent=8, k_scales=ks, v_scales=vs, kept=kept, new_lens=lens)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step(*state, out, kept)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(6):
        eager_out, eager_kept = torch.empty_like(out), torch.empty_like(kept)
        step(*other, eager_out, eager_kept)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager_out) and torch.equal(kept, eager_kept), f"replay {rep}"
        assert all(equal(a, b) if a.dtype == E4M3 else torch.equal(a, b) for a, b in zip(state, other)), f"replay {rep}"
        for x in (nk, nv):
            x.copy_(c.rows(S))
        q.copy_(c.rows(S, heads=H * group))


def test_evict_of_long_lists_captured_with_one_workspace():
    """Few long lists, whose keys and counts lie in the caller's workspace: captured for two layers that share
    it and the lengths, replayed with new scores, whatever it holds, eager calls between."""
    H, d, P, keep = 2, 64, 64, 1500
    layers = [Paged8(74 + i, [30000, 900, 21000], H, d, P, spare=1).cuda() for i in range(2)]
    table, lens = layers[0].table, layers[0].lens
    size = binding.still_paged_evict_workspace_size(
        binding.still_paged_cache(H, d, P, layers[0].n_pages, BF16, 16, 16, None),
        binding.still_paged_seqs(3, table.shape[1], table.shape[1], table.data_ptr(), lens.data_ptr()),
        binding.still_paged_evict_config(keep, 4, 100, 0))
    assert size > 0
    ws = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
    kept = [torch.empty(3, H, keep, dtype=torch.int32, device="cuda") for _ in layers]
    new = [torch.empty(3, dtype=torch.int32, device="cuda") for _ in layers]

    def step(caches, kept, new, ws):
        for x, ids, n in zip(caches, kept, new):
            binding.paged_evict(x[0], x[1], table, lens, x[4], keep, first=4, recent=100, k_scales=x[2], v_scales=x[3], kept=ids,
                                new_lens=n, workspace=ws)

    state = [[*x.pools(), x.scores] for x in layers]
    start = [[y.clone() for y in x] for x in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step(state, kept, new, ws)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        for x, y in zip(state, start):
            y[4].copy_(torch.rand(y[4].shape, generator=layers[0].g) ** (2 * rep + 1))
            for a, b in zip(x, y):
                a.view(torch.uint8).copy_(b.view(torch.uint8))
        lens.copy_(torch.tensor([30000 - 9000 * rep, 900 + rep * 500, 21000], dtype=torch.int32))
        other = [[y.clone() for y in x] for x in start]
        ids, n = [torch.empty_like(x) for x in kept], [torch.empty_like(x) for x in new]
        step(other, ids, n, None)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(kept[i], ids[i]) and torch.equal(new[i], n[i]), f"replay {rep}"
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(state[i], other[i])), f"replay {rep}"
        want = O8.evict(table.cpu().numpy(), lens.cpu().numpy(), start[1][4].cpu().numpy(), keep, 4, 100)
        np.testing.assert_array_equal(kept[1].cpu().numpy(), want[0])
        ws.fill_(rep)


def test_evict_on_another_stream_and_two_at_once():
    c = [Paged8(72 + i, [900, 300], 2, 64, 16).cuda() for i in range(2)]
    want = []
    for x in c:
        y = [t.clone() for t in (*x.pools(), x.scores)]
        want.append((y, binding.paged_evict(y[0], y[1], x.table, x.lens, y[4], 200, recent=10, k_scales=y[2], v_scales=y[3])))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for x, st in zip(c, streams):
        with torch.cuda.stream(st):
            got.append(binding.paged_evict(x.k, x.v, x.table, x.lens, x.scores, 200, recent=10, k_scales=x.ks, v_scales=x.vs))
    torch.cuda.synchronize()
    for x, (y, ref), have in zip(c, want, got):
        assert torch.equal(have[0], ref[0]) and torch.equal(have[1], ref[1])
        assert equal(x.k, y[0]) and equal(x.v, y[1]) and torch.equal(x.scores, y[4])


@pytest.mark.parametrize("with_head", [False, True])
def test_compact_paged_of_8_bit_pages(with_head):
    """Two layers' pages of a sequence, cut by a shared eviction, then compacted where they are: what the dense
    calls make of their rows, appended."""
    w = configs.shrink(configs.get_workload(1), n_tokens=200, t=32)
    H, d, P, n, t, start, end = w.cfg.n_kv_heads, w.cfg.head_dim, 16, 150, 32, 6, 130
    wts = [weights_to_device(synth.make_weights(w, l, t=t), BF16) for l in range(2)]
    wb = [dev_tensor(synth.make_beta_weight(w, l), BF16) for l in range(2)]
    layers = [Paged8(80, [30, 200], H, d, P, width=14).cuda() for _ in range(2)]
    c = layers[0]
    layers[1].k, layers[1].v = layers[1].v, layers[1].k
    layers[1].ks, layers[1].vs = layers[1].vs, layers[1].ks
    positions = torch.arange(200, dtype=torch.float64, device="cuda") + 1000
    for x in layers:
        kept, new = binding.paged_evict(x.k, x.v, c.table, c.lens, x.scores, n, first=4, recent=20, shared=True, k_scales=x.ks,
                                        v_scales=x.vs, beta_pages=x.beta)
    assert new.tolist() == [30, n]
    lens, pos = new, positions[kept[1, 0].long()]
    row, to = c.table[1:2], [torch.tensor([x], dtype=torch.int32, device="cuda") for x in (start + t, n - (end - start) + t)]
    want = []
    for x, W, b in zip(layers, wts, wb):
        K, V, bias = binding.paged8_gather(*x.pools(), c.table, lens, 1, n, beta_pages=x.beta)
        cut = (w.cfg, [W], [K[:, start:end].contiguous()], [V[:, start:end].contiguous()], pos[start:end].contiguous(),
               w.rope_theta, t)
        if with_head:
            (Ck,), (Cv,), pq, (beta,) = binding.compact_model_beta(*cut, [b], 2.0, 0.5)
        else:
            ((Ck,), (Cv,), pq), beta = binding.compact_model(*cut), torch.zeros(H, t, device="cuda")
        y = [z.clone() for z in (*x.pools(), x.beta)]
        binding.paged8_append(Ck.transpose(0, 1), Cv.transpose(0, 1), *y[:4], row, to[0], beta=beta.t(), beta_pages=y[4])
        binding.paged8_append(K[:, end:].transpose(0, 1), V[:, end:].transpose(0, 1), *y[:4], row, to[1], beta=bias[:, end:].t(),
                              beta_pages=y[4])
        want.append(y)
    kw = dict(w_beta=wb, beta_max=2.0, mass_alpha=0.5) if with_head else {}
    now = binding.compact_paged(w.cfg, wts, [x.k for x in layers], [x.v for x in layers], c.table, lens, 1, n, pos, w.rope_theta,
                                t, start=start, end=end, beta_pages=[x.beta for x in layers],
                                scales=[(x.ks, x.vs) for x in layers], **kw)
    assert lens.tolist() == [30, n - (end - start) + t] and torch.equal(now, torch.cat([pos[:start], pq, pos[end:]]))
    for x, y in zip(layers, want):
        assert equal(x.k, y[0]) and equal(x.v, y[1])
        assert torch.equal(x.ks, y[2]) and torch.equal(x.vs, y[3]) and torch.equal(x.beta, y[4])
