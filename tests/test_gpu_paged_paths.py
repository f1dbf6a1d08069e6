"""The kernels of the paged attention that a call reaches by its table's
capacity, against the fp64 oracle: entries split over workgroups and joined,
with ordinary and streaming loads, at every width, type and row count; their
addresses past 4 GiB; and captured, on a workspace that other calls use too.
"""
import pytest
import torch

from paper_2606_07878_amd import configs
from tests.helpers import log
from tests.paged_cases import Paged
from tests.test_gpu_paged import check_attend

pytestmark = pytest.mark.gpu

BF16, FP32 = configs.MODE_BF16, configs.MODE_FP32
STREAM_BYTES = 256 << 20    # a table that can hold more than this takes streaming loads


def columns(c, streaming):
    """Table columns that take the split kernel (above 1024 entries), below or above the streaming line."""
    row = 2 * len(c.lens_list) * c.H * c.d * (4 if c.mode == FP32 else 2) * c.P
    n = STREAM_BYTES // row + 1 if streaming else max(c.table.shape[1], 1024 // c.P + 1)
    assert (n * row > STREAM_BYTES) == streaming and n * c.P > 1024
    return n


def widened(c, streaming):
    """c's table with absent pages behind."""
    table = torch.full((c.table.shape[0], columns(c, streaming)), -1, dtype=torch.int32)
    table[:, : c.table.shape[1]] = c.table.cpu()
    return table


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("group,nq", [(4, 1), (3, 8), (4, 8)])
@pytest.mark.parametrize("streaming", [False, True])
def test_split_sequences(mode, d, group, nq, streaming):
    """A sequence over many workgroups, one of a chunk, one of none; rotated, causal, with bias."""
    log(f"split mode={mode} d={d} group={group} nq={nq} streaming={streaming}")
    c = Paged(70, [2100, 0, 37, 700], 2, d, 32, mode)
    n = 4 * nq
    pos = torch.from_numpy(c.rng.uniform(0, 1e5, n))
    check_attend(c, c.rows(n, 2 * group), causal=nq > 1, qpos=pos, theta=1e6, table=widened(c, streaming))


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("streaming", [False, True])
def test_split_kernels_past_four_gib(mode, streaming):
    """Pages whose byte and element offsets pass 32 bits, read by the split kernels."""
    from paper_2606_07878_amd import binding
    H, P, d = 8, 16, 128
    pages = (1 << 32) // (H * P * d * 2) + 40          # more than 2^31 elements, 2^32 bytes
    c = Paged(71, [600, 90], H, d, P, mode)
    small = c.n_pages
    k = torch.zeros(pages, H, P, d, dtype=c.k.dtype, device="cuda")
    v = torch.zeros_like(k)
    beta = torch.zeros(pages, H, P, device="cuda")
    k[pages - small:], v[pages - small:], beta[pages - small:] = c.k.cuda(), c.v.cuda(), c.beta.cuda()
    table = widened(c, streaming)
    q = c.rows(2, 32)
    want = check_attend(c, q, table=table)
    far = torch.where(table >= 0, table + (pages - small), table)
    got = binding.paged_attend(q.cuda(), k, v, far.cuda(), c.lens.cuda(), beta_pages=beta)
    assert torch.equal(got, want)


def test_split_steps_in_a_graph_share_a_workspace_with_other_calls():
    """A split call, captured once: its grid stays while sequences go from
    split to whole to empty and back; the workspace starts as 0xFF bytes, and
    between the replays other shapes use it, among them one whose joins are
    planned per workgroup (more sequences than workgroups of a head)."""
    from paper_2606_07878_amd import binding
    c = Paged(72, [5000, 300, 0, 40], 2, 128, 16, BF16, width=400)
    q = c.rows(4, 8)
    many = Paged(73, [int(x) for x in torch.randint(0, 90, (600,), generator=c.g)], 1, 64, 16, BF16, width=6)
    many.table = torch.cat([many.table, torch.full((600, 60), -1, dtype=torch.int32)], 1)
    many.lens[300] = 66 * 16
    many.table[300] = torch.arange(66, dtype=torch.int32)
    mq = many.rows(600, 8)
    few = Paged(74, [1500, 20], 3, 256, 32, FP32)
    fq = few.rows(2 * 4, 12)
    others = [(x, y, z, check_attend(x, y, causal=z)) for x, y, z in ((many, mq, False), (few, fq, True))]
    c.cuda(), many.cuda(), few.cuda()
    q, mq, fq = q.cuda(), mq.cuda(), fq.cuda()
    ws = torch.full((binding.STILL_PAGED_WORKSPACE_BYTES,), 255, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            binding.paged_attend(q, *c.pages(), beta_pages=c.beta, workspace=ws, out=out)
    torch.cuda.current_stream().wait_stream(side)
    for lens in ([5000, 300, 0, 40], [10, 6000, 300, 0], [0, 0, 0, 0], [6400, 6400, 1, 2000], [30, 30, 30, 30],
                 [5000, 300, 0, 40]):
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for other, oq, causal, want in others:
            got = binding.paged_attend(oq.cuda(), *other.pages(), causal=causal, beta_pages=other.beta, workspace=ws)
            torch.cuda.synchronize()
            assert torch.equal(got, want)
            out.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, check_attend(c, q)), lens


# ---- calls that the documentation allows -----------------------------------------

def test_strides_of_dimensions_of_one_mean_nothing():
    """One query head (a transposed [1, T, d]), one KV head, one token: their strides address nothing."""
    from paper_2606_07878_amd import binding
    c = Paged(75, [20, 33, 5], 1, 64, 16, BF16)
    heads_first = torch.randn(1, 3, 64, generator=c.g).bfloat16()
    q = heads_first.cuda().transpose(0, 1)
    assert q.shape == (3, 1, 64) and q.stride(1) != 64
    assert torch.equal(check_attend(c, q), check_attend(c, q.contiguous()))
    rows = torch.randn(3 * 64 + 8, generator=c.g).bfloat16().cuda()
    odd = rows.as_strided((3, 1, 64), (64, 5, 1))                       # the one head's stride
    one = rows.as_strided((1, 1, 64), (7, 3, 1))                        # the one token's, too
    c.cuda()
    for k, table, lens in ((odd, c.table, c.lens), (one, c.table[:1], c.lens[:1])):
        pages = [[x.clone() for x in (c.k, c.v)] for _ in range(2)]
        binding.paged_append(k, k, *pages[0], table, lens)
        dense = k.reshape(-1).clone().view(k.shape)
        binding.paged_append(dense, dense, *pages[1], table, lens)
        assert torch.equal(pages[0][0], pages[1][0]) and torch.equal(pages[0][1], pages[1][1])
        assert not torch.equal(pages[0][0], c.k)


# ---- compact_paged ---------------------------------------------------------------

def two_layers(t=32, n=100):
    from paper_2606_07878_amd import synth
    from tests.helpers import weights_to_device
    w = configs.shrink(configs.get_workload(1), n_tokens=n, t=t)
    c = Paged(76, [n, 50], w.cfg.n_kv_heads, w.cfg.head_dim, 16, BF16).cuda()
    W = weights_to_device(synth.make_weights(w, 0, t=t), BF16)
    pages = [[x.clone() for x in (c.k, c.v, c.beta)] for _ in range(2)]
    return w, c, [W, W], pages, torch.arange(n, dtype=torch.float64, device="cuda")


def test_compact_paged_changes_nothing_where_a_layers_bias_pages_are_not_aligned():
    from paper_2606_07878_amd import binding
    w, c, W, pages, pos = two_layers()
    odd = torch.empty(c.beta.numel() + 4, device="cuda")[1: 1 + c.beta.numel()].view(c.beta.shape)
    odd.copy_(c.beta)
    assert odd.is_contiguous() and odd.data_ptr() % 16 == 4
    with pytest.raises(binding.StillError) as e:
        binding.compact_paged(w.cfg, W, [p[0] for p in pages], [p[1] for p in pages], c.table, c.lens, 0, 100, pos,
                              w.rope_theta, 32, beta_pages=[pages[0][2], odd])
    assert e.value.status == -1
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for p in pages for x, y in zip(p, (c.k, c.v, c.beta))) and c.lens.tolist() == [100, 50]


def test_compact_paged_allocates_nothing_once_pages_change(monkeypatch):
    """What could run out of memory comes before the first page changes."""
    from paper_2606_07878_amd import binding
    w, c, W, pages, pos = two_layers()
    count = lambda: torch.cuda.memory_stats()["allocation.all.allocated"]  # noqa: E731
    seen, append = [], binding.paged_append

    def counted(*args, **kw):
        seen.append(count())
        append(*args, **kw)

    monkeypatch.setattr(binding, "paged_append", counted)
    binding.compact_paged(w.cfg, W, [p[0] for p in pages], [p[1] for p in pages], c.table, c.lens, 0, 100, pos,
                          w.rope_theta, 32, start=10, end=60, beta_pages=[p[2] for p in pages])
    assert len(seen) == 4 and seen[0] == count()


@pytest.mark.parametrize("with_head", [False, True])
def test_compact_paged_of_entries_that_carry_bias(with_head):
    """A sequence whose first 20 entries (an earlier compaction's) carry bias.
    Behind them a compaction leaves them alone; over them it gives what it gives
    without their bias, or, asked not to drop it, nothing changes."""
    from paper_2606_07878_amd import binding, synth
    from tests.helpers import dev_tensor
    w, c, W, pages, pos = two_layers()
    kw = {}
    if with_head:
        head = dev_tensor(synth.make_beta_weight(w, 0), BF16)
        kw = dict(w_beta=[head, head], beta_max=2.0, mass_alpha=0.5)

    def compact(pages, lens, **more):
        return binding.compact_paged(w.cfg, W, [p[0] for p in pages], [p[1] for p in pages], c.table, lens, 0, 100, pos,
                                     w.rope_theta, 32, beta_pages=[p[2] for p in pages], **kw, **more)

    for p in pages:   # bias on entries 0 .. 19 alone
        keep = [binding.paged_gather(*p[:2], c.table, c.lens, 0, 20, beta_pages=p[2])[2]]
        p[2].zero_()
        k, v, _ = binding.paged_gather(*p[:2], c.table, c.lens, 0, 20, beta_pages=p[2])
        binding.paged_append(k.transpose(0, 1), v.transpose(0, 1), *p[:2], c.table[:1],
                             torch.tensor([20], dtype=torch.int32, device="cuda"), beta=keep[0].t(), beta_pages=p[2])
    before = [[x.clone() for x in p] for p in pages]
    with pytest.raises(binding.StillError) as e:
        compact(pages, c.lens, drop_bias=False)
    assert e.value.status == -5 and "layer 0" in str(e.value)
    with pytest.raises(binding.StillError) as e:
        compact(pages, c.lens, start=19, drop_bias=False)
    assert e.value.status == -5
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for p, b in zip(pages, before) for x, y in zip(p, b)) and c.lens.tolist() == [100, 50]

    bare = [[p[0].clone(), p[1].clone(), torch.zeros_like(p[2])] for p in pages]
    over = [[x.clone() for x in p] for p in pages]
    lens = [c.lens.clone() for _ in range(3)]
    assert torch.equal(compact(bare, lens[0], drop_bias=False), compact(over, lens[1]))
    for x, y in zip(bare, over):
        got, want = (binding.paged_gather(*p[:2], c.table, lens[0], 0, 32, beta_pages=p[2]) for p in (x, y))
        assert all(torch.equal(g, r) for g, r in zip(got, want))
    compact(pages, lens[2], start=20, drop_bias=False)
    assert lens[2].tolist() == [52, 50]
    for p, b in zip(pages, before):
        got, want = (binding.paged_gather(*x[:2], c.table, c.lens, 0, 20, beta_pages=x[2]) for x in (p, b))
        assert all(torch.equal(g, r) for g, r in zip(got, want)) and got[2].any()


@pytest.mark.parametrize("mode", [BF16, FP32])
@pytest.mark.parametrize("streaming", [None, False])
def test_a_logit_of_minus_infinity_leaves_its_entry_out(mode, streaming):
    """An infinite key whose product is minus infinity is the same as a bias of
    minus infinity, bit for bit; a query whose product is plus infinity, and an
    infinite value, come out non-finite."""
    from paper_2606_07878_amd import binding
    c = Paged(77, [40, 90], 2, 64, 16, mode)
    q = c.rows(2, 4)
    q[:, :, 0] = -q[:, :, 0].abs() - 0.5
    q[1, 1, 0] = 0.5
    table = c.table if streaming is None else widened(c, streaming)
    page, at = int(c.table[1, 2]), 5

    def run(k, v, b):
        return binding.paged_attend(q.cuda(), k.cuda(), v.cuda(), table.cuda(), c.lens.cuda(), beta_pages=b.cuda())

    k, v, b = c.k.clone(), c.v.clone(), c.beta.clone()
    b[page, 0, at] = float("-inf")
    want = run(k, v, b)
    k[page, 0, at, 0] = float("inf")
    got = run(k, v, c.beta)
    same = torch.ones(2, 4, dtype=torch.bool)
    same[1, :2] = False                    # the query, and the other one of its sequence and KV head
    assert torch.isfinite(want).all() and not torch.isfinite(got[1, 1]).any()
    assert torch.equal(got[same.cuda()], want[same.cuda()])
    q[1, 1, 0] = -0.5
    assert torch.equal(run(k, v, c.beta), run(c.k, v, b))
    v[page, 0, at, 3] = float("inf")
    assert not torch.isfinite(run(c.k, v, b)[1, :2, 3]).any()


def test_append_of_more_tokens_than_a_grid_has_threads_for():
    """2^26 tokens and some: 64 threads each pass 2^32, which one dimension of a grid cannot hold."""
    from paper_2606_07878_amd import binding
    n, P = (1 << 26) + 5000, 4096
    pages = -(-n // P)
    log(f"{n} tokens, {pages} pages, {3 * pages * P * 128 / 2**30:.1f} GiB")
    k = torch.empty(n, 1, 64, dtype=torch.bfloat16, device="cuda")
    k.view(torch.int16).copy_(torch.arange(n, device="cuda", dtype=torch.int32).to(torch.int16)[:, None, None])
    pool = [torch.zeros(pages, 1, P, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    binding.paged_append(k, k, *pool, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    for x in pool:
        rows = x.view(torch.int16).view(pages * P, 64)
        assert torch.equal(rows[:n], k.view(torch.int16)[:, 0]) and not rows[n:].any()
    del k, pool, x, rows
    torch.cuda.empty_cache()


def test_gather_of_as_many_entries_as_a_table_holds():
    """2^30 entries, 2^24 blocks of 256 threads: their number passes 32 bits too.  Keys and values, the
    same, go into one buffer (128 GiB), the table repeats a few pages."""
    from paper_2606_07878_amd import binding
    P, pages, n = 4096, 5, 1 << 30
    width = n // P
    pool = torch.randint(-32768, 32767, (pages, 1, P, 64), dtype=torch.int16, device="cuda").view(torch.bfloat16)
    table = (torch.arange(width, dtype=torch.int32, device="cuda") % pages)[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    out = torch.empty(n, 64, dtype=torch.bfloat16, device="cuda")
    chunks = out.view(torch.int16).view(width, P * 64)
    chunks[-1] = 7
    cache = binding.still_paged_cache(1, 64, P, pages, BF16, pool.data_ptr(), pool.data_ptr(), None)
    seqs = binding.still_paged_seqs(1, width, width, table.data_ptr(), lens.data_ptr())
    assert binding.still_paged_gather(cache, seqs, 0, 0, n, out, out, None, torch.cuda.current_stream().cuda_stream) == 0
    rows = pool.view(torch.int16).view(pages, P * 64)
    for i in (*range(0, width, 9973), width - 2, width - 1):
        assert torch.equal(chunks[i], rows[i % pages]), i
    del out, chunks
    torch.cuda.empty_cache()
