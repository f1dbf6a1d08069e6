"""The oracle of the 8-bit paged cache against independent facts, and the refusals of its
entry points (no GPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged as O, paged8 as O8
from paper_2606_07878_amd import binding, configs
from tests.paged8_cases import E4M3, Paged8, f64
from tests.test_paged_pins import BAD_CACHE, BAD_SEQS, FAKE, _acfg, _seqs, _tokens


def test_e4m3_is_what_torch_rounds_to():
    x = torch.cat([torch.randn(20000, generator=torch.Generator().manual_seed(1)) * s for s in (1e-3, 0.02, 1.0, 90.0)])
    x = torch.cat([x.clamp(-448, 448), torch.tensor([0.0, -0.0, 448.0, -448.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 17.0, 19.0, 432.0])])
    np.testing.assert_array_equal(O8.e4m3(f64(x)), f64(x.to(E4M3)))
    assert np.isnan(O8.e4m3([math.inf, -math.inf, math.nan])).all()


@pytest.mark.parametrize("top", [448.0, 448.5, 447.9, 1.75, 1.7500001, 1e-40, 3e38, 1.0, 2.0 ** -92, 0.0])
def test_scale_is_the_smallest_power_that_serves(top):
    s = O8.scale_for(top)
    assert math.frexp(s)[0] == 0.5 and 448 * s >= top
    assert s == 2.0 ** -100 or 448 * s / 2 < top


def test_append_to_8_bits_grows_and_starts_anew():
    c = Paged8(1, [21], 2, 64, 16, beta=False)
    k, v, _, _ = (f64(x) for x in c.pools())
    x = np.ones((3, 2, 64))
    x[1] = 1000.0
    kp, vp, ks, vs, _ = O8.append(x, x * 0.5, k, v, f64(c.ks), f64(c.vs), c.table.numpy(), c.lens.numpy())
    page = int(c.table[0, 1])
    assert (ks[page] == np.maximum(f64(c.ks)[page], 4.0)).all()           # 1000 = 250 * 4
    before = O8.values(k, f64(c.ks))[page, :, :2]
    after = O8.values(kp, ks)[page]
    assert np.abs(after[:, :2] - before).max() <= 4.0 * 2.0 ** -10        # what fell below the smallest code
    assert (after[:, 3] == O8.e4m3(250.0) * 4).all() and (after[:, 2] == 1.0).all()
    # a first slot starts anew, whatever the scale was
    kp, _, ks, _, _ = O8.append(x[:1], x[:1], k, v, np.full_like(f64(c.ks), 1e6), f64(c.vs), c.table.numpy(), np.array([17]))
    assert (ks[page] == O8.scale_for(1.0)).all()
    assert (O8.values(kp, ks)[page, :, 0] == 1.0).all()


def test_weights_sum_to_the_rows_and_lse_is_their_normalizer():
    c = Paged8(2, [40, 0, 7], 2, 64, 16)
    k, _ = c.values()
    q, t, n = f64(c.rows(6, heads=4)), c.table.numpy(), c.lens.numpy()
    row = O8.lse(q, k, t, n, causal=True, beta_pages=f64(c.beta))
    assert np.isneginf(row[2:4]).all() and np.isfinite(row[[0, 1, 4, 5]]).all()
    zero = np.zeros(f64(c.scores).shape)
    got = O8.score(q, row, k, zero, t, n, causal=True, beta_pages=f64(c.beta))
    np.testing.assert_allclose(got.sum(axis=(0, 2)), [8.0, 8.0], rtol=1e-13)   # 2 sequences x 2 queries x 2 heads
    # the same attention output from them
    out = O.attend(q, k, c.values()[1], t, n, causal=True, beta_pages=f64(c.beta))
    assert np.isfinite(out).all()


def test_evict_keeps_the_largest_in_order():
    x = [0.0, 5.0, 5.0, math.nan, 1.0, 7.0, 0.0]
    assert O8.keep_entries(x, 7, 3, 0, 0).tolist() == [1, 2, 5]
    assert O8.keep_entries(x, 7, 3, 1, 1).tolist() == [0, 5, 6]
    assert O8.keep_entries(x, 7, 2, 0, 0).tolist() == [1, 5]
    assert O8.keep_entries(x, 7, 6, 0, 0).tolist() == [0, 1, 2, 4, 5, 6]
    assert O8.keep_entries(x, 7, 9, 0, 0).tolist() == list(range(7))


# ---- refusals ----------------------------------------------------------------

def _cache8(**kw):
    base = dict(n_kv_heads=8, head_dim=128, page_size=16, n_pages=100, mode=configs.MODE_BF16, k=FAKE, v=FAKE,
                k_scale=FAKE, v_scale=FAKE, beta=None)
    base.update(kw)
    return binding.still_paged8_cache(**base)


def _attend8(cache=None, seqs=None, cfg=None, q=FAKE, pos=None, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 30):
    return binding.still_paged8_attend(cache or _cache8(), seqs or _seqs(), cfg or _acfg(), q, pos, out, lse, ws,
                                       ws_bytes, None)


@pytest.mark.parametrize("kw,status", BAD_CACHE + [(dict(k_scale=None), -1), (dict(v_scale=FAKE + 4), -1)])
def test_bad_cache(kw, status):
    c = _cache8(**kw)
    assert _attend8(cache=c) == status
    assert binding.still_paged8_append(c, _seqs(), _tokens(), None) == status
    assert binding.still_paged8_gather(c, _seqs(), 0, 0, 5, FAKE, FAKE, None, None) == status
    assert binding.still_last_error()


@pytest.mark.parametrize("kw,status", BAD_SEQS)
def test_bad_sequences(kw, status):
    q = _seqs(**kw)
    assert _attend8(seqs=q) == status
    assert binding.still_paged8_append(_cache8(), q, _tokens(n_tokens=q.n_seqs), None) == status
    assert binding.still_paged8_gather(_cache8(), q, 0, 0, 5, FAKE, FAKE, None, None) == status


def test_attend_pointers_workspace_and_nothing_to_do():
    assert _attend8(q=None) == -1 and _attend8(out=FAKE + 8) == -1 and _attend8(lse=FAKE + 2) == -1
    assert _attend8(ws=None) == -4 and _attend8(ws_bytes=100) == -4
    assert _attend8(cfg=_acfg(group=5, n_queries=7)) == -5 and _attend8(cfg=_acfg(rope_theta=1e6)) == -1
    assert binding.still_paged_attend_lse(binding.still_paged_cache(8, 128, 16, 100, 0, FAKE, FAKE, None), _seqs(), _acfg(),
                                          FAKE, None, FAKE, FAKE + 1, FAKE, 1 << 30, None) == -1
    need = binding.still_paged8_attend_workspace_size(_cache8(), _acfg())
    assert 0 < need <= binding.STILL_PAGED_WORKSPACE_BYTES
    assert binding.still_paged8_attend_workspace_size(_cache8(head_dim=96), _acfg()) == 0
    assert binding.still_paged8_append(_cache8(), _seqs(), _tokens(n_tokens=0, k=None, v=None), None) == 0
    assert binding.still_paged8_gather(_cache8(), _seqs(), 0, 0, 0, None, None, None, None) == 0


@pytest.mark.parametrize("H", [1, 2, 3, 8, 64, 300, 65535])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_workspace_serves_every_call(H, d):
    for mode in (configs.MODE_BF16, configs.MODE_FP32):
        for rows in (1, 16, 17, 32):
            need = binding.still_paged8_attend_workspace_size(_cache8(n_kv_heads=H, head_dim=d, mode=mode), _acfg(group=rows))
            assert 0 < need <= binding.STILL_PAGED_WORKSPACE_BYTES


def test_null_structs():
    lib, c, s = binding.lib(), ctypes.byref(_cache8()), ctypes.byref(_seqs())
    assert lib.still_paged8_append(None, s, ctypes.byref(_tokens()), None) == -1
    assert lib.still_paged8_append(c, None, ctypes.byref(_tokens()), None) == -1
    assert lib.still_paged8_append(c, s, None, None) == -1
    assert lib.still_paged8_gather(None, s, 0, 0, 1, FAKE, FAKE, None, None) == -1
    assert lib.still_paged8_attend(None, s, ctypes.byref(_acfg()), FAKE, None, FAKE, None, FAKE, 1 << 30, None) == -1
    assert lib.still_paged8_attend(c, s, None, FAKE, None, FAKE, None, FAKE, 1 << 30, None) == -1
    assert lib.still_paged8_attend_workspace_size(None, ctypes.byref(_acfg())) == 0


def _raises(status, call, *args, **kw):
    with pytest.raises(binding.StillError) as e:
        call(*args, **kw)
    assert e.value.status == status, str(e.value)


def test_binding_refuses_what_does_not_fit():
    c = Paged8(3, [40, 7], 2, 64, 16)
    k, v, ks, vs, table, lens = c.pages()
    rows = c.rows(2)
    good = (k, v, ks, vs, table, lens)

    def each(status, *pages):
        _raises(status, binding.paged8_append, rows, rows, *pages)
        _raises(status, binding.paged8_gather, *pages, 0, 5)
        _raises(status, binding.paged8_attend, c.rows(2, heads=4), *pages)

    each(-1, *good)                                                       # CPU tensors: a GPU is needed
    each(-3, k.view(torch.uint8), v, ks, vs, table, lens)
    each(-3, k.float(), v, ks, vs, table, lens)
    each(-3, k, v.view(torch.uint8), ks, vs, table, lens)
    each(-2, k[0], v, ks, vs, table, lens)
    each(-2, k, v[:1], ks, vs, table, lens)
    each(-2, k, v, ks[..., :0], vs, table, lens)
    each(-2, k, v, ks, vs.repeat(1, 1, 2), table, lens)
    each(-3, k, v, ks.double(), vs, table, lens)
    each(-1, k, v, ks, vs.transpose(0, 1).contiguous().transpose(0, 1), table, lens)
    each(-2, k, v, ks, vs, table.long(), lens)
    each(-2, k, v, ks, vs, table, lens[:1])
    _raises(-3, binding.paged8_append, rows.half(), rows.half(), *good)
    _raises(-3, binding.paged8_gather, *good, 0, 5, dtype=torch.float16)
    _raises(-3, binding.paged8_attend, c.rows(2, heads=4).double(), *good)


# ---- scores and eviction -----------------------------------------------------

def _ecfg(**kw):
    base = dict(keep=64, first=4, recent=16, shared=0)
    base.update(kw)
    return binding.still_paged_evict_config(**base)


def _plain(**kw):
    base = dict(n_kv_heads=8, head_dim=128, page_size=16, n_pages=100, mode=configs.MODE_BF16, k=FAKE, v=FAKE, beta=None)
    base.update(kw)
    return binding.still_paged_cache(**base)


def _score(cache=None, seqs=None, cfg=None, q=FAKE, pos=None, lse=FAKE, known=None, scores=FAKE):
    return binding.still_paged_score(cache or _cache8(), seqs or _seqs(), cfg or _acfg(), q, pos, lse, known, scores, None)


def _evict(cache=None, seqs=None, cfg=None, scores=FAKE, kept=FAKE, new_lens=FAKE, ws=None, ws_bytes=0):
    return binding.still_paged_evict(cache or _cache8(), seqs or _seqs(), cfg or _ecfg(), scores, kept, new_lens, ws, ws_bytes,
                                     None)


@pytest.mark.parametrize("make", [_cache8, _plain])
def test_score_and_evict_refuse(make):
    for kw, status in BAD_CACHE:
        if "v" not in kw:
            assert _score(cache=make(**kw)) == status
        assert _evict(cache=make(**kw)) == status
    for kw, status in BAD_SEQS:
        assert _score(cache=make(), seqs=_seqs(**kw)) == status
        assert _evict(cache=make(), seqs=_seqs(**kw)) == status
    for kw in (dict(q=None), dict(lse=None), dict(lse=FAKE + 2), dict(known=FAKE + 1), dict(scores=None), dict(scores=FAKE + 4)):
        assert _score(cache=make(), **kw) == -1
    for kw, status in ((dict(group=33), -5), (dict(n_queries=0), -2), (dict(causal=2), -1), (dict(scale=-1.0), -1),
                       (dict(rope_theta=1e6), -1), (dict(q_stride=4), -2)):
        assert _score(cache=make(), cfg=_acfg(**kw)) == status
    for kw in (dict(scores=None), dict(scores=FAKE + 8), dict(kept=None), dict(kept=FAKE + 2), dict(new_lens=None), dict(new_lens=FAKE + 3)):
        assert _evict(cache=make(), **kw) == -1
    for kw, status in ((dict(keep=0), -2), (dict(keep=-5), -2), (dict(first=-1), -2), (dict(recent=-1), -2),
                       (dict(first=50, recent=15), -2), (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), -2), (dict(shared=2), -1),
                       (dict(keep=2 ** 30 + 1), -5), (dict(keep=2 ** 31 - 1), -5)):
        assert _evict(cache=make(), cfg=_ecfg(**kw)) == status


def test_score_and_evict_null_structs_and_scales():
    assert _score(cache=_cache8(k_scale=None)) == -1 and _evict(cache=_cache8(v_scale=FAKE + 4)) == -1
    lib, s = binding.lib(), ctypes.byref(_seqs())
    for c in (None, ctypes.byref(_cache8())):
        assert lib.still_paged8_evict(c, s if c is None else None, ctypes.byref(_ecfg()), FAKE, FAKE, FAKE, None, 0, None) == -1
        assert lib.still_paged8_score(c, s if c is None else None, ctypes.byref(_acfg()), FAKE, None, FAKE, None, FAKE, None) == -1
    assert lib.still_paged8_evict(ctypes.byref(_cache8()), s, None, FAKE, FAKE, FAKE, None, 0, None) == -1
    assert lib.still_paged_evict(None, s, ctypes.byref(_ecfg()), FAKE, FAKE, FAKE, None, 0, None) == -1
    assert lib.still_paged_score(None, s, ctypes.byref(_acfg()), FAKE, None, FAKE, None, FAKE, None) == -1


def test_evict_workspace():
    """The lists' keys and counts where few long tables are given, 96 MiB at most; none for others."""
    size = binding.still_paged_evict_workspace_size
    assert size(_plain(), _seqs(max_pages=512, table_stride=512), _ecfg()) == 0
    long = _seqs(max_pages=1200, table_stride=1200)
    each = 19200 * 4 + 5 * 2048 * 4
    assert size(_plain(), long, _ecfg()) == 4 * 8 * each and size(_plain(), long, _ecfg(shared=1)) == 4 * each
    assert size(_plain(), _seqs(max_pages=600, table_stride=600), _ecfg()) == 0
    assert size(_plain(), _seqs(max_pages=600, table_stride=600), _ecfg(shared=1)) > 0
    assert size(_plain(), _seqs(n_seqs=60, max_pages=600, table_stride=600), _ecfg()) == 0
    for pages in (1 << 16, 1 << 20, 1 << 26):
        assert size(_plain(), _seqs(max_pages=pages, table_stride=pages), _ecfg(shared=1)) <= 96 << 20
    assert size(_plain(head_dim=96), long, _ecfg()) == 0 and size(_plain(), long, _ecfg(keep=0)) == 0
    assert _evict(seqs=long) == -4 and _evict(seqs=long, ws=FAKE, ws_bytes=1000) == -4
    assert _evict(seqs=long, ws=FAKE + 4, ws_bytes=1 << 30) == -1


def test_binding_refuses_scores_that_do_not_fit():
    c = Paged8(4, [40, 7], 2, 64, 16)
    k, v, ks, vs, table, lens = c.pages()
    q, lse = c.rows(2, heads=4), torch.zeros(2, 4)
    _raises(-1, binding.paged_score, q, lse, k, c.scores, table, lens, k_scales=ks)       # CPU tensors: a GPU is needed
    _raises(-3, binding.paged_score, q, lse, k, c.scores, table, lens)
    _raises(-1, binding.paged_score, q, lse, k.bfloat16(), c.scores, table, lens, k_scales=ks)
    _raises(-1, binding.paged_evict, k, v, table, lens, c.scores, 8, k_scales=ks, v_scales=vs)
    _raises(-1, binding.paged_evict, k, v, table, lens, c.scores, 8, k_scales=ks)
    _raises(-1, binding.paged_evict, k.float(), v.float(), table, lens, c.scores, 8)
    _raises(-1, binding.compact_paged, configs.get_workload(1).cfg, [None], [k], [v], table, lens, 0, 40, None, 1e6, 8,
            scales=[None])
