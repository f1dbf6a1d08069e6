"""The paged cache on the CPU: pins of its oracle against something other than
itself, and the refusals of its entry points (none reaches a device)."""
import ctypes
import re

import numpy as np
import pytest
import torch

from oracle import compactor, consumer, paged as O
from paper_2606_07878_amd import binding, configs
from tests.paged_cases import Paged

FAKE = 0x10000   # never dereferenced: validation fails before any device access


# ---- oracle ----------------------------------------------------------------

@pytest.mark.parametrize("nq,group,causal", [(1, 4, False), (3, 2, True)])
def test_attend_matches_the_dense_oracle(nq, group, causal):
    c = Paged(1, [37, 16, 50], 2, 64, 16, configs.MODE_FP32)
    k, v, b, table, lens = c.f64()
    q = c.rng.standard_normal((3 * nq, 2 * group, 64))
    pos = 1000.0 + np.arange(3 * nq)
    got = O.attend(q, k, v, table, lens, causal=causal, beta_pages=b, q_positions=pos, rope_theta=1e4)
    for s, n in enumerate(lens):
        K, V, B = (O.gather(x, table, lens, s, 0, n) for x in (k, v, b))
        # the dense oracle's compact part with its bias, and the entries a causal query may not see as suffix
        qs = q[s * nq:(s + 1) * nq].transpose(1, 0, 2)
        t = n - nq if causal else n
        if causal:   # the bias of the suffix part folded into the key it belongs to is not expressible: take it as 0
            B[:, t:] = 0.0
        want = consumer.attend(qs, K[:, :t], V[:, :t], B[:, :t], K[:, t:], V[:, t:], group=group, causal=causal,
                               q_positions=pos[s * nq:(s + 1) * nq], rope_theta=1e4)
        if causal:
            bz = b.copy()
            for j in range(t, n):
                p, o = O.slot(table, s, j, 16, k.shape[0])
                bz[p, :, o] = 0.0
            got = O.attend(q, k, v, table, lens, causal=True, beta_pages=bz, q_positions=pos, rope_theta=1e4)
        np.testing.assert_allclose(got[s * nq:(s + 1) * nq].transpose(1, 0, 2), want, rtol=1e-12, atol=1e-12)


def test_append_then_gather_returns_the_rotated_rows():
    c = Paged(2, [20, 40], 2, 64, 16, configs.MODE_FP32)
    k, v, b, table, lens = c.f64()
    nk, nv, nb = c.rng.standard_normal((9, 2, 64)), c.rng.standard_normal((9, 2, 64)), c.rng.standard_normal((9, 2))
    pos = np.arange(9.0) + 77
    kp, vp, bp = O.append(nk, nv, k, v, table, lens, [0, 4, 9], pos, 1e4, nb, b)
    got = O.gather(kp, table, lens, 1, 35, 5)
    for h in range(2):
        np.testing.assert_allclose(got[h], compactor.rope(nk[4:, h], pos[4:], 1e4), rtol=0, atol=1e-14)
    np.testing.assert_array_equal(O.gather(vp, table, lens, 0, 16, 4), nv[:4].transpose(1, 0, 2))
    np.testing.assert_array_equal(O.gather(bp, table, lens, 0, 16, 4), nb[:4].T)
    np.testing.assert_array_equal(O.gather(kp, table, lens, 0, 0, 16), O.gather(k, table, lens, 0, 0, 16))
    assert (kp != k).any(axis=(1, 3)).sum() == 9   # nine entries, nothing else


def test_absent_pages_and_lengths_out_of_range():
    c = Paged(3, [40], 1, 64, 16, configs.MODE_FP32)
    k, v, b, table, lens = c.f64()
    table[0, 1] = -1
    assert not O.gather(k, table, lens, 0, 16, 16).any()
    kp, _, _ = O.append(np.ones((40, 1, 64)), np.ones((40, 1, 64)), k, v, table, lens)
    assert (kp == 1.0).all(axis=(1, 3)).sum() == 24
    q = c.rng.standard_normal((1, 1, 64))
    one = O.attend(q, k, v, table, lens)
    both = O.attend(q, k, v, np.delete(table, 1, axis=1), np.array([24]))
    np.testing.assert_allclose(one, both, rtol=1e-14, atol=1e-14)
    assert not O.attend(q, k, v, table, np.array([-3])).any()
    np.testing.assert_array_equal(O.attend(q, k, v, table, np.array([4000])), O.attend(q, k, v, table, np.array([48])))


# ---- refusals of the C entry points -----------------------------------------

def _cache(**kw):
    base = dict(n_kv_heads=8, head_dim=128, page_size=16, n_pages=100, mode=configs.MODE_BF16, k=FAKE, v=FAKE, beta=None)
    base.update(kw)
    return binding.still_paged_cache(**base)


def _seqs(**kw):
    base = dict(n_seqs=4, max_pages=10, table_stride=10, table=FAKE, lens=FAKE)
    base.update(kw)
    return binding.still_paged_seqs(**base)


def _tokens(**kw):
    base = dict(n_tokens=4, k=FAKE, v=FAKE, k_token_stride=1024, k_head_stride=128, v_token_stride=1024,
                v_head_stride=128)
    base.update(kw)
    return binding.still_paged_tokens(**base)


def _acfg(**kw):
    base = dict(group=4, n_queries=1, causal=0, scale=0.0, rope_theta=0.0, q_stride=0)
    base.update(kw)
    return binding.still_paged_attend_config(**base)


def _attend(cache=None, seqs=None, cfg=None, q=FAKE, pos=None, out=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return binding.still_paged_attend(cache or _cache(), seqs or _seqs(), cfg or _acfg(), q, pos, out, ws, ws_bytes,
                                      None)


BAD_CACHE = [(dict(mode=7), -3), (dict(head_dim=96), -5), (dict(n_kv_heads=0), -2), (dict(n_kv_heads=65536), -5),
             (dict(n_pages=0), -2), (dict(page_size=8), -5), (dict(page_size=48), -5), (dict(page_size=0), -5),
             (dict(page_size=8192), -5), (dict(page_size=-16), -5), (dict(k=None), -1), (dict(v=FAKE + 8), -1),
             (dict(beta=FAKE + 2), -1)]
BAD_SEQS = [(dict(n_seqs=0), -2), (dict(n_seqs=65536), -5), (dict(max_pages=0), -2), (dict(table_stride=9), -2),
            (dict(max_pages=1 << 27, table_stride=1 << 27), -5),
            (dict(n_seqs=65535, max_pages=1 << 15, table_stride=1 << 15), -5), (dict(table=None), -1), (dict(lens=FAKE + 1), -1)]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_bad_cache(kw, status):
    c = _cache(**kw)
    assert _attend(cache=c) == status
    assert binding.still_paged_append(c, _seqs(), _tokens(), None) == status
    assert binding.still_paged_gather(c, _seqs(), 0, 0, 5, FAKE, FAKE, None, None) == status
    assert binding.still_last_error()


@pytest.mark.parametrize("kw,status", BAD_SEQS)
def test_bad_sequences(kw, status):
    q = _seqs(**kw)
    assert _attend(seqs=q) == status
    assert binding.still_paged_append(_cache(), q, _tokens(), None) == status
    assert binding.still_paged_gather(_cache(), q, 0, 0, 5, FAKE, FAKE, None, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(n_tokens=-1), -2), (dict(n_tokens=5), -2), (dict(k=None), -1), (dict(v=FAKE + 4), -1),
    (dict(k_token_stride=1020), -2), (dict(v_head_stride=4), -2), (dict(beta=FAKE), -1), (dict(offsets=FAKE + 2), -1),
    (dict(rope_theta=1e6), -1), (dict(rope_theta=1e6, positions=FAKE + 4), -1), (dict(rope_theta=-1.0), -1),
    (dict(rope_theta=float("inf"), positions=FAKE), -1), (dict(rope_theta=float("nan"), positions=FAKE), -1)])
def test_bad_tokens(kw, status):
    assert binding.still_paged_append(_cache(), _seqs(), _tokens(**kw), None) == status
    assert binding.still_last_error()


def test_no_tokens_and_no_entries_are_fine_without_buffers():
    assert binding.still_paged_append(_cache(), _seqs(), _tokens(n_tokens=0, k=None, v=None), None) == 0
    assert binding.still_paged_gather(_cache(), _seqs(), 0, 160, 0, None, None, None, None) == 0


@pytest.mark.parametrize("args,status", [
    ((4, 0, 5, FAKE, FAKE, None), -2), ((-1, 0, 5, FAKE, FAKE, None), -2), ((0, -1, 5, FAKE, FAKE, None), -2),
    ((0, 0, -5, FAKE, FAKE, None), -2), ((0, 156, 5, FAKE, FAKE, None), -2),
    ((0, 2**31 - 1, 2**31 - 1, FAKE, FAKE, None), -2), ((0, 0, 5, None, FAKE, None), -1),
    ((0, 0, 5, FAKE, FAKE + 8, None), -1), ((0, 0, 5, FAKE, FAKE, FAKE), -1)])
def test_bad_gather(args, status):
    assert binding.still_paged_gather(_cache(), _seqs(), *args, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(group=0), -2), (dict(n_queries=0), -2), (dict(n_queries=9), -5), (dict(group=1 << 30, n_queries=4), -5),
    (dict(causal=2), -1), (dict(scale=float("nan")), -1), (dict(scale=-1.0), -1), (dict(rope_theta=1e6), -1),
    (dict(rope_theta=-1.0), -1), (dict(q_stride=4100), -2), (dict(q_stride=-4096), -2)])
def test_bad_attend(kw, status):
    assert _attend(cfg=_acfg(**kw)) == status
    assert binding.still_last_error()


def test_attend_pointers_and_workspace():
    assert _attend(q=None) == -1
    assert _attend(out=FAKE + 8) == -1
    assert _attend(cfg=_acfg(rope_theta=1e6), pos=FAKE + 4) == -1
    assert _attend(ws=None) == -4
    need = binding.still_paged_attend_workspace_size(_cache(), _acfg())
    assert need > 0
    assert _attend(ws_bytes=need - 1) == -4
    assert binding.still_paged_attend_workspace_size(_cache(), _acfg(n_queries=9)) == 0
    assert binding.still_paged_attend_workspace_size(_cache(page_size=3), _acfg()) == 0


@pytest.mark.parametrize("H", [1, 3, 8, 100, 1024, 2000, 65535])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_workspace_serves_every_call(H, d):
    for group, nq in ((1, 1), (4, 1), (8, 4), (32, 1), (1, 32)):
        n = binding.still_paged_attend_workspace_size(_cache(n_kv_heads=H, head_dim=d), _acfg(group=group, n_queries=nq))
        assert 0 < n <= binding.STILL_PAGED_WORKSPACE_BYTES


def test_workspace_bound_matches_the_header():
    from tests.test_abi import HEADER
    m = re.search(r"STILL_PAGED_WORKSPACE_BYTES\s*=\s*(\d+)\s*<<\s*(\d+)", open(HEADER).read())
    assert m and int(m.group(1)) << int(m.group(2)) == binding.STILL_PAGED_WORKSPACE_BYTES


def test_null_structs():
    lib, null = binding.lib(), None
    c, s, t, a = _cache(), _seqs(), _tokens(), _acfg()
    r = ctypes.byref
    assert lib.still_paged_append(null, r(s), r(t), null) == -1
    assert lib.still_paged_append(r(c), null, r(t), null) == -1
    assert lib.still_paged_append(r(c), r(s), null, null) == -1
    assert lib.still_paged_gather(null, r(s), 0, 0, 1, FAKE, FAKE, null, null) == -1
    assert lib.still_paged_attend(r(c), r(s), null, FAKE, null, FAKE, FAKE, 1 << 30, null) == -1
    assert lib.still_paged_attend_workspace_size(null, r(a)) == 0


# ---- refusals of the binding -------------------------------------------------

def _refused(status, f, *args, **kw):
    with pytest.raises(binding.StillError) as e:
        f(*args, **kw)
    assert e.value.status == status, str(e.value)


def test_binding_refuses_what_does_not_fit():
    c = Paged(4, [20, 30], 2, 64, 16, configs.MODE_BF16)
    q, k = c.rows(2, 4), c.rows(2)
    P = c.pages()
    assert c.k.device.type == "cpu"
    _refused(-1, binding.paged_attend, q, *P)                                    # no GPU tensors
    _refused(-1, binding.paged_append, k, k, *P)
    _refused(-1, binding.paged_gather, *P, 0, 5)
    _refused(-2, binding.paged_attend, q, c.k[0], *P[1:])
    _refused(-2, binding.paged_attend, q, c.k, c.v[:3], c.table, c.lens)
    _refused(-3, binding.paged_attend, q, c.k, c.v.float(), c.table, c.lens)
    _refused(-3, binding.paged_attend, q, c.k.half(), c.v.half(), c.table, c.lens)
    _refused(-1, binding.paged_attend, q, c.k.transpose(1, 2).contiguous().transpose(1, 2), c.v, c.table, c.lens)
    _refused(-2, binding.paged_attend, q, c.k, c.v, c.table.long(), c.lens)
    _refused(-2, binding.paged_attend, q, c.k, c.v, c.table.t().contiguous().t(), c.lens)
    _refused(-2, binding.paged_attend, q, c.k, c.v, c.table, c.lens[:1])
    _refused(-3, binding.paged_attend, q, c.k, c.v, c.table, c.lens.long())
    _refused(-2, binding.paged_attend, q, *P, beta_pages=c.beta[:, :1].contiguous())
    _refused(-3, binding.paged_attend, q, *P, beta_pages=c.beta.double())


@pytest.mark.skipif(torch.cuda.is_available(), reason="CPU refusals only")
def test_compact_paged_refuses_bad_ranges():
    c = Paged(5, [20, 30], 2, 64, 16, configs.MODE_BF16)
    w = configs.get_workload(1)
    pos = torch.arange(30, dtype=torch.float64)
    args = (w.cfg, [{}], [c.k], [c.v], c.table, c.lens)
    _refused(-1, binding.compact_paged, *args, 1, 30, pos, 1e6, 8, start=10, end=10)
    _refused(-1, binding.compact_paged, *args, 1, 30, pos, 1e6, 8, start=0, end=31)
    _refused(-2, binding.compact_paged, *args, 2, 30, pos, 1e6, 8)
    _refused(-2, binding.compact_paged, *args, 1, 30, pos, 1e6, 100)             # does not fit the pages
    _refused(-2, binding.compact_paged, w.cfg, [{}, {}], [c.k], [c.v], c.table, c.lens, 1, 30, pos, 1e6, 8)
    _refused(-1, binding.compact_paged, *args, 1, 30, pos, 1e6, 8, w_beta=[pos])
    _refused(-2, binding.compact_paged, *args, 1, 30, pos[:5], 1e6, 8)


@pytest.mark.skipif(torch.cuda.is_available(), reason="CPU refusals only")
def test_compact_paged_checks_every_layer_before_any_changes():
    w = configs.get_workload(1)
    c = Paged(6, [20, 30], w.cfg.n_kv_heads, w.cfg.head_dim, 16, configs.MODE_BF16)
    pos = torch.arange(30, dtype=torch.float64)

    def refused(status, k2, v2, seq_len=30, **kw):
        _refused(status, binding.compact_paged, w.cfg, [{}, {}], [c.k, k2], [c.v, v2], c.table, c.lens, 1, seq_len, pos,
                 1e6, 8, **kw)

    refused(-1, c.k, c.v)                                                        # no GPU tensors
    refused(-3, c.k.float(), c.v.float())                                        # layers of two types
    refused(-2, c.k[:, :1], c.v[:, :1])
    refused(-2, c.k[:, :, :8], c.v[:, :, :8])                                    # layer 1's pages hold less
    refused(-1, c.k, c.v, w_beta=[pos, pos], beta_pages=[c.beta, None])
    refused(-2, c.k[0], c.v[0])


@pytest.mark.skipif(torch.cuda.is_available(), reason="CPU refusals only")
def test_binding_refuses_table_rows_too_far_apart():
    c = Paged(7, [20, 30], 2, 64, 16, configs.MODE_BF16)
    far = torch.empty_strided((2, 2), (1 << 31, 1), dtype=torch.int32, device="meta")
    _refused(-2, binding.paged_attend, c.rows(2, 4), c.k, c.v, far, c.lens)


def test_workspace_bound_is_near_what_the_largest_call_needs():
    """A loop holds one such buffer per stream: no more than a sixteenth of it is spare."""
    most = max(binding.still_paged_attend_workspace_size(_cache(n_kv_heads=H, head_dim=d), _acfg(group=group))
               for H in (*range(1, 520), 65535) for d in (64, 128, 256) for group in (1, 16, 17, 32))
    assert 15 / 16 * binding.STILL_PAGED_WORKSPACE_BYTES < most <= binding.STILL_PAGED_WORKSPACE_BYTES


@pytest.mark.skipif(torch.cuda.is_available(), reason="CPU refusals only")
@pytest.mark.parametrize("shape", [((1 << 32) + 2, 2), (1, (1 << 32) + 2)])
def test_binding_refuses_table_sizes_past_32_bits(shape):
    """Their low 32 bits say 2."""
    c = Paged(8, [20, 30], 2, 64, 16, configs.MODE_BF16)
    table = torch.empty(shape, dtype=torch.int32, device="meta")
    lens = torch.empty(shape[:1], dtype=torch.int32, device="meta")
    _refused(-2, binding.paged_attend, c.rows(2, 4), c.k, c.v, table, lens)
    _refused(-2, binding.paged_gather, c.k, c.v, table, lens, 0, 5)


@pytest.mark.skipif(torch.cuda.is_available(), reason="CPU refusals only")
def test_compact_paged_refuses_a_table_of_other_dimensions():
    c = Paged(9, [20, 30], 2, 64, 16, configs.MODE_BF16)
    w = configs.get_workload(1)
    pos = torch.arange(30, dtype=torch.float64)
    for table in (c.table[0], c.table[None], torch.tensor(3, dtype=torch.int32)):
        _refused(-2, binding.compact_paged, w.cfg, [{}], [c.k], [c.v], table, c.lens, 0, 20, pos, 1e6, 8)
