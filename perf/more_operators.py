"""A paged cache held in 8 bits, and eviction from a paged cache by accumulated attention weight.

Five operators, each through a public entry point of ``binding``:

* ``append8``  new keys and values of several sequences into pages of 8-bit
               floating point (e4m3) with a scale for each block of 16 entries
               and head, the keys rotated on the way (``binding.paged8_append``);
* ``gather8``  a range of one sequence out of such pages, as the dense rows the
               compactor reads (``binding.paged8_gather``);
* ``attend8``  attention of the newest query rows over such pages, with the log
               of each row's sum of exponentials (``binding.paged8_attend``);
* ``score``    the attention weights of the newest query rows, summed over the
               rows of a KV head, added to what the entries have gathered so
               far (``binding.paged_score``);
* ``evict``    the entries of largest score, the first and the most recent ones
               kept, the others dropped, inside the pages (``binding.paged_evict``).

Pages are [n_pages, H, P, d], scales [n_pages, H, P / 16], bias and scores
[n_pages, H, P] float32; a table [n_seqs, pages] of page numbers and the lengths
say which entries a sequence has.  An entry of 8 bits stands for its code times its
block's scale, a power of two: the smallest with which no number of the block exceeds
448, the largest e4m3 number.  A block that grows keeps its scale if that still
serves; otherwise its codes are rescaled.  Page sizes, head shapes and lengths are those of
the caches that the repository compacts.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
SIZES = {"bf16": 2, "fp32": 4, "fp8": 1}
WORKSPACE_BYTES = 24 << 20      # a serving program's one buffer, enough for every call
BLOCK = 16                      # entries that share a scale
LEAST = 2.0 ** -100             # the smallest scale


# ----------------------------------------------------------------------------
# The cases
# ----------------------------------------------------------------------------

def _append(name, seqs, lo, hi, new_lo, new_hi, H, d, P, rows="bf16", rotate=True, beta=False, layout="token"):
    return dict(name=name, op="append8", seqs=seqs, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, H=H, group=4, d=d, P=P,
                rows=rows, cache="fp8", rotate=rotate, beta=beta, layout=layout)


def _gather(name, n, start, H, d, P, rows="bf16", beta=False):
    return dict(name=name, op="gather8", n=n, start=start, H=H, d=d, P=P, rows=rows, cache="fp8", beta=beta)


def _attend(name, seqs, lo, hi, H, group, d, P, nq=1, causal=False, rows="bf16", rotate=False, beta=False, empty=0):
    return dict(name=name, op="attend8", seqs=seqs, lo=lo, hi=hi, H=H, group=group, d=d, P=P, nq=nq, causal=causal,
                rows=rows, cache="fp8", rotate=rotate, beta=beta, empty=empty)


def _score(name, seqs, lo, hi, H, group, d, P, nq=1, causal=False, cache="fp8", rows="bf16", rotate=False, beta=False,
           empty=0):
    return dict(name=name, op="score", seqs=seqs, lo=lo, hi=hi, H=H, group=group, d=d, P=P, nq=nq, causal=causal,
                rows=rows, cache=cache, rotate=rotate, beta=beta, empty=empty)


def _evict(name, seqs, lo, hi, keep, first, recent, H, d, P, cache="fp8", shared=False, beta=False):
    return dict(name=name, op="evict", seqs=seqs, lo=lo, hi=hi, keep=keep, first=first, recent=recent, H=H, d=d, P=P,
                rows="fp32" if cache == "fp32" else "bf16", cache=cache, shared=shared, beta=beta)


def listed():
    return [
        # one token of one conversation behind its compact entries, inside a block: the smallest append
        _append("append8_step_1", 1, 727, 727, 1, 1, 8, 128, 16),
        # prompts of 13 sequences of odd lengths in one call, about 8k tokens, wide heads
        _append("append8_prompts_d256", 13, 2000, 9000, 37, 2000, 8, 256, 32, beta=True),
        # the fresh tokens behind a preserved prefix, an odd count that starts inside a block
        _gather("gather8_1k", 1087, 37, 8, 128, 16),
        # a long wide-headed cache on its way into the compactor: the largest copy
        _gather("gather8_64k_d256", 65536, 0, 8, 256, 64),
        # one decode step of one conversation: 655 compact entries with their bias and 64 fresh ones
        _attend("attend8_step_compact", 1, 719, 719, 8, 4, 128, 16, beta=True),
        # the same step over an uncompacted 128k cache
        _attend("attend8_step_128k", 1, 131136, 131136, 8, 4, 128, 64),
        # a decode step of 64 conversations between a word and 16k tokens, queries rotated here,
        # the last rows of the batch padding
        _attend("attend8_batch_ragged", 64, 5, 16384, 8, 4, 128, 16, rotate=True, beta=True, empty=3),
        # 8 new tokens each (a checked draft), causal, wide heads: 16 query rows per KV head
        _attend("attend8_block_causal", 12, 1500, 20011, 8, 2, 256, 128, nq=8, causal=True, rotate=True),
        # the weights of that batch's decode step, for a later eviction
        _score("score_batch_ragged", 64, 5, 16384, 8, 4, 128, 16, rotate=True, beta=True, empty=3),
        # the last 8 tokens of a long prompt over an ordinary cache: what of it they look at
        _score("score_prompt_bf16", 1, 65536, 65536, 8, 4, 128, 64, nq=8, causal=True, cache="bf16"),
        # 64 conversations back to 1024 entries each, every head its own, 64 tokens after the last time
        _evict("evict_batch", 64, 1088, 1088, 1024, 4, 64, 8, 128, 64),
        # one long prompt down to 4096 entries, the same for all heads (so that it can be compacted)
        _evict("evict_prompt_bf16", 1, 65536, 65536, 4096, 4, 256, 8, 128, 64, cache="bf16", shared=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: 1 to 256 sequences, 1 to 131136 entries, every type,
    the widths and page sizes the kernels take, up to 32 query rows."""
    op = rng.choice(["append8", "gather8", "attend8", "attend8", "score", "evict"])
    H, d, P = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([64, 128, 256]), rng.choice([16, 32, 64, 128, 256])
    rows = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    beta = rng.random() < 0.5
    row = 4 * H * d                                                  # bytes of one entry in 16 bits
    if op == "gather8":
        n = min(_log(rng, 1, 131072), int(2.5e8 / row))
        return dict(_gather("", n, rng.choice([0, rng.randrange(0, 5000)]), H, d, P, rows, beta), name="gather8")
    seqs = _log(rng, 1, 256)
    if op == "append8":
        most = max(1, min(8192, int(1.2e8 / row / seqs)))
        new = _log(rng, 1, most)
        new_lo = rng.choice([new, rng.randint(1, new)])
        lo = new + rng.randrange(0, 2000)
        return dict(_append("", seqs, lo, lo + rng.randrange(0, 4000), new_lo, new, H, d, P, rows,
                            rng.random() < 0.7, beta, rng.choice(["token", "head"])), name="append8")
    hi = min(_log(rng, 1, 131136), max(1, int((5e8 if op == "attend8" else 1.3e8) / row / seqs)))
    lo = min(hi, rng.choice([hi, _log(rng, 1, hi)]))
    cache = rng.choice(["fp8", "fp8", rows])
    if op == "evict":
        keep = _log(rng, 1, hi)
        first = rng.choice([0, rng.randint(0, min(keep, 16))])
        return dict(_evict("", seqs, lo, hi, keep, first, rng.choice([0, rng.randint(0, keep - first)]), H, d, P, cache,
                           rng.random() < 0.4, beta), name="evict")
    group = rng.choice([1, 2, 3, 4, 8])
    nq = rng.choice([1, 1, 1, rng.randint(1, 32 // group)])
    more = (nq, rng.random() < 0.6)
    empty = rng.choice([0, 0, 1]) if seqs > 1 else 0
    if op == "attend8":
        return dict(_attend("", seqs, lo, hi, H, group, d, P, *more, rows, rng.random() < 0.5, beta, empty), name="attend8")
    return dict(_score("", seqs, lo, hi, H, group, d, P, *more, cache, rows, rng.random() < 0.5, beta, empty), name="score")


def _spread(lo, hi, n, salt):
    """n whole numbers from lo to hi, spread over their logarithm, in no order."""
    x = np.rint(np.geomspace(lo, hi, n) if n > 1 else np.array([hi])).astype(np.int64)
    return np.random.RandomState(salt).permutation(x)


def _lens(case):
    """(entries of each sequence after the call's tokens, new ones among them)."""
    if case["op"] == "gather8":
        return np.array([case["start"] + case["n"]]), np.array([case["n"]])
    n = case["seqs"]
    lens = _spread(case["lo"], case["hi"], n, n)
    if case["op"] == "append8":
        return lens, _spread(case["new_lo"], case["new_hi"], n, n + 1)
    if case.get("empty"):
        lens[n - case["empty"]:] = 0
    return lens, np.full(n, case.get("nq", 0))


def _theta(d):
    return 1e4 if d == 256 else 1e6     # the wide-headed models' base, and the others'


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op, H, d, P, dt = case["op"], case["H"], case["d"], case["P"], DTYPES[case["rows"]]
    lens, new = _lens(case)
    n = len(lens)

    def rand(*shape, dtype=dt):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)

    # a pool a little larger than the sequences need, its pages handed out in no order; the
    # table's entries behind a sequence's last page stay 0
    held = -(-lens // P)
    width, pages = max(1, int(held.max())), int(held.sum()) + 5
    taken = torch.from_numpy(np.arange(width) < held[:, None]).to(DEV)
    table = torch.zeros(n, width, dtype=torch.int32, device=DEV)
    table[taken] = torch.randperm(pages, generator=g, device=DEV)[: int(held.sum())].to(torch.int32)
    s = dict(case=case, H=H, d=d, P=P, table=table, lens=torch.from_numpy(lens.astype(np.int32)).to(DEV),
             theta=_theta(d) if case.get("rotate") else 0.0, beta_pages=None, k_scales=None, v_scales=None)
    eight = case["cache"] == "fp8"
    for x in ("k", "v"):
        if eight:   # blocks of numbers up to about 16 to 448 times scales of 2^-9 to 2^-6
            size = torch.randint(4, 7, (pages, H, P // BLOCK, 1, 1), generator=g, device=DEV)
            codes = torch.randn(pages, H, P // BLOCK, BLOCK, d, generator=g, device=DEV).mul_(torch.exp2(size))
            s[x + "_pages"] = codes.clamp_(-448, 448).to(DTYPES["fp8"]).view(pages, H, P, d)
            s[x + "_scales"] = torch.exp2(-size.view(pages, H, P // BLOCK).float())
            del codes
        else:
            s[x + "_pages"] = rand(pages, H, P, d)
    if case["beta"]:
        s["beta_pages"] = rand(pages, H, P, dtype=torch.float32)
    if op == "gather8":
        s["out"] = tuple(torch.empty(H, case["n"], d, dtype=dt, device=DEV) for _ in range(2))
        if case["beta"]:
            s["out"] += (torch.empty(H, case["n"], device=DEV),)
        return s
    if op in ("score", "evict"):   # sums of a few hundred rows' weights; entries nothing looked at have none
        s["scores"] = torch.exp(2 * rand(pages, H, P, dtype=torch.float32) - 3)
        s["scores"][torch.rand(pages, H, P, generator=g, device=DEV) < 0.03] = 0.0
    if op == "evict":
        s["kept"] = torch.empty(n, 1 if case["shared"] else H, case["keep"], dtype=torch.int32, device=DEV)
        s["new_lens"] = torch.empty(n, dtype=torch.int32, device=DEV)
        return s
    tokens = int(new.sum())
    # rows of the fused projection: query heads, key heads, value heads
    Hq = H * case["group"]
    if case.get("layout") == "head":
        s["k"], s["v"] = (rand(H, tokens, d).transpose(0, 1) for _ in range(2))
    else:
        qkv = rand(tokens, (Hq + 2 * H) * d)
        s["q"] = qkv[:, : Hq * d].view(tokens, Hq, d)
        s["k"] = qkv[:, Hq * d: (Hq + H) * d].view(tokens, H, d)
        s["v"] = qkv[:, (Hq + H) * d:].view(tokens, H, d)
    # logical positions: behind a prefix that was compacted from 128k tokens
    first = np.repeat(lens - new, new)
    within = np.arange(tokens) - np.repeat(np.cumsum(new) - new, new)
    s["positions"] = torch.from_numpy((first + within + 130417).astype(np.float64)).to(DEV) if s["theta"] else None
    if op == "append8":
        s["offsets"] = None
        if new.min() != new.max():
            s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
        s["beta"] = rand(H, tokens, dtype=torch.float32).transpose(0, 1) if case["beta"] else None
        return s
    s["out"] = torch.empty(tokens, Hq, d, dtype=dt, device=DEV)
    s["lse"] = torch.empty(tokens, Hq, device=DEV)
    s["ws"] = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    if op == "score":   # what the step's attention has given out; all but the newest entries have scores
        x = _logits(s)
        m = x.amax(dim=-1, keepdim=True)
        x.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
        s["lse"] = _by_token(s, (torch.log(x.sum(dim=-1)) + m[..., 0])[..., None])[..., 0].contiguous()
        s["known"] = (s["lens"] - 1).clamp_(min=0)
    return s


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"append8": _plain_append, "gather8": _plain_gather, "attend8": _plain_attend, "score": _plain_score,
            "evict": _plain_evict}[op](s)


def _own(s, op):
    from paper_2606_07878_amd import binding
    case = s["case"]
    if op == "append8":
        binding.paged8_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["table"],
                              s["lens"], offsets=s["offsets"], positions=s["positions"], rope_theta=s["theta"],
                              beta=s["beta"], beta_pages=s["beta_pages"])
        return _pools(s)
    if op == "gather8":
        return list(binding.paged8_gather(s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["table"], s["lens"],
                                          0, case["n"], start=case["start"], beta_pages=s["beta_pages"], out=s["out"]))
    if op == "attend8":
        binding.paged8_attend(s["q"], s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["table"], s["lens"],
                              causal=case["causal"], beta_pages=s["beta_pages"], q_positions=s["positions"],
                              rope_theta=s["theta"], workspace=s["ws"], out=s["out"], lse=s["lse"])
        return [s["out"], s["lse"]]
    if op == "score":
        binding.paged_score(s["q"], s["lse"], s["k_pages"], s["scores"], s["table"], s["lens"], causal=case["causal"],
                            k_scales=s["k_scales"], beta_pages=s["beta_pages"], known=s["known"],
                            q_positions=s["positions"], rope_theta=s["theta"])
        return s["scores"]
    binding.paged_evict(s["k_pages"], s["v_pages"], s["table"], s["lens"], s["scores"], case["keep"], first=case["first"],
                        recent=case["recent"], shared=case["shared"], k_scales=s["k_scales"], v_scales=s["v_scales"],
                        beta_pages=s["beta_pages"], kept=s["kept"], new_lens=s["new_lens"])
    return [s["kept"], s["new_lens"]] + _pools(s) + [s["scores"]]


def _pools(s):
    return [s[x] for x in ("k_pages", "v_pages", "k_scales", "v_scales", "beta_pages") if s[x] is not None]


def _rotated(x, positions, theta):
    """x [tokens, heads, d] rotated at the tokens' positions in 64 bits (a scale depends on which side
    of a border the largest number of a block lies), as 32 bits."""
    if not theta:
        return x.float()
    x = x.double()
    half = x.shape[-1] // 2
    inv = torch.pow(torch.tensor(theta, dtype=torch.float64, device=DEV),
                    -torch.arange(half, dtype=torch.float64, device=DEV) / half)
    angle = positions[:, None] * inv
    c, sn = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * sn, b * c + a * sn], dim=-1).float()


def _scale_for(top):
    """The smallest power of two whose 448-fold reaches top, at least LEAST."""
    m, e = torch.frexp(top)     # top = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    return torch.where(top > 0, torch.ldexp(torch.ones_like(top), e - 9 + (m > 0.875)), LEAST).clamp_(min=LEAST)


def _plain_append(s):
    P, H, d, n, tokens = s["P"], s["H"], s["d"], s["table"].shape[0], s["k"].shape[0]
    i = torch.arange(tokens, device=DEV)
    if s["offsets"] is None:
        seq = i // (tokens // n)
        start, end = seq * (tokens // n), (seq + 1) * (tokens // n)
    else:
        seq = torch.searchsorted(s["offsets"], i.to(torch.int32), right=True) - 1
        start, end = s["offsets"][seq], s["offsets"][seq + 1]
    j = (s["lens"][seq] - end + i).long()
    first = s["lens"][seq] - end + start                     # the call's first entry of the sequence
    slot = j % P
    at = s["table"][seq, j // P].long() * (P // BLOCK) + slot // BLOCK
    blocks, to = torch.unique(at, return_inverse=True)       # blocks that get entries, each token's among them
    page, b = blocks // (P // BLOCK), blocks % (P // BLOCK)
    # entries that a block holds already: those in front of the call's first one
    old = torch.zeros(len(blocks), dtype=torch.long, device=DEV)
    old.scatter_reduce_(0, to, (first - (j - j % BLOCK)).clamp(0, BLOCK).long(), "amax")
    for_old = torch.arange(BLOCK, device=DEV) < old[:, None]
    for x in ("k", "v"):
        y = _rotated(s[x], s["positions"], s["theta"] if x == "k" else 0.0)
        top = torch.zeros(len(blocks), H, device=DEV)
        top.scatter_reduce_(0, to[:, None].expand(tokens, H), y.abs().amax(dim=-1), "amax")
        scales = s[x + "_scales"]
        before = torch.where(old[:, None] > 0, scales[page, :, b], 0.0)
        now = torch.maximum(before, _scale_for(top))
        codes = s[x + "_pages"].view(torch.uint8).view(-1, H, P // BLOCK, BLOCK, d)
        had = codes[page, :, b]
        again = (had.view(DTYPES["fp8"]).float() * (before / now)[:, :, None, None]).to(DTYPES["fp8"]).view(torch.uint8)
        codes[page, :, b] = torch.where(for_old[:, None, :, None], again, had)
        codes[page[to], :, b[to], slot % BLOCK] = (y / now[to][:, :, None]).to(DTYPES["fp8"]).view(torch.uint8)
        scales[page, :, b] = now
    if s["beta_pages"] is not None:
        s["beta_pages"][page[to], :, slot] = s["beta"]
    return _pools(s)


def _entries(s, pages, scales, table):
    """The entries of these pages in 32 bits, [..., H, P, d]."""
    if scales is None:
        return pages[table].float()
    x = pages.view(torch.uint8)[table].view(DTYPES["fp8"]).float()
    return x * scales[table].repeat_interleave(BLOCK, dim=-1)[..., None]


def _plain_gather(s):
    n, start, P = s["case"]["n"], s["case"]["start"], s["P"]
    a, z = start // P, -(-(start + n) // P)
    pages = s["table"][0, a:z].long()
    there = torch.arange(n, device=DEV) + start < s["lens"][0]
    got = []
    for x in ("k", "v"):
        y = _entries(s, s[x + "_pages"], s[x + "_scales"], pages).transpose(0, 1).reshape(s["H"], -1, s["d"])
        got.append(torch.where(there[:, None], y[:, start - a * P: start - a * P + n], 0.0).to(s["out"][0].dtype))
    if s["beta_pages"] is not None:
        y = s["beta_pages"][pages].transpose(0, 1).reshape(s["H"], -1)
        got.append(torch.where(there, y[:, start - a * P: start - a * P + n], 0.0))
    return got


def _logits(s):
    """[n_seqs, H, group * n_queries, entries] in 32 bits, minus infinity where a row does not see."""
    n, width = s["table"].shape
    H, d, P, group, nq = s["H"], s["d"], s["P"], s["case"]["group"], s["case"]["nq"]
    table = s["table"].long()
    k = _entries(s, s["k_pages"], s["k_scales"], table).transpose(1, 2).reshape(n, H, width * P, d)
    q = _rotated(s["q"], s["positions"], s["theta"]).reshape(n, nq, H, group, d).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.reshape(n, H, group * nq, d), k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    del k
    if s["beta_pages"] is not None:
        x += s["beta_pages"][table].transpose(1, 2).reshape(n, H, 1, width * P)
    # row (g, i) sits at entry lens - nq + i and, where causal, sees entries up to its own
    last = s["lens"][:, None] - (nq if s["case"]["causal"] else 1)
    last = last + torch.arange(nq, device=DEV) if s["case"]["causal"] else last.expand(n, nq)
    last = last[:, None, None, :, None].expand(n, 1, group, nq, 1).reshape(n, 1, group * nq, 1)
    return x.masked_fill_(torch.arange(width * P, device=DEV) > last, -math.inf)


def _by_token(s, x):
    """[n_seqs, H, group * n_queries, y] as [tokens, H * group, y]."""
    n, H, group, nq = s["table"].shape[0], s["H"], s["case"]["group"], s["case"]["nq"]
    return x.reshape(n, H, group, nq, -1).permute(0, 3, 1, 2, 4).reshape(n * nq, H * group, -1)


def _plain_attend(s):
    n, width = s["table"].shape
    x = _logits(s)
    m = x.amax(dim=-1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    del x
    total = e.sum(dim=-1, keepdim=True)
    v = _entries(s, s["v_pages"], s["v_scales"], s["table"].long()).transpose(1, 2).reshape(n, s["H"], width * s["P"], s["d"])
    o = torch.matmul(e, v) / torch.where(total > 0, total, 1.0)
    return [_by_token(s, o).to(s["q"].dtype), _by_token(s, torch.log(total) + m)[..., 0]]


def _plain_score(s):
    n, width = s["table"].shape
    H, P = s["H"], s["P"]
    lse = s["lse"].view(n, s["case"]["nq"], H, s["case"]["group"]).permute(0, 2, 3, 1).reshape(n, H, -1, 1)
    x = _logits(s)
    w = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)).sum(dim=2)
    j = torch.arange(width * P, device=DEV)
    old = s["scores"][s["table"].long()].transpose(1, 2).reshape(n, H, width * P)
    w = w + torch.where(j < s["known"][:, None, None], old, 0.0)
    there = (j < s["lens"][:, None]).view(n, width, P)
    seq, t, slot = there.nonzero(as_tuple=True)
    s["scores"][s["table"][seq, t].long(), :, slot] = w.view(n, H, width, P)[seq, :, t, slot]
    return s["scores"]


def _plain_evict(s):
    n, width = s["table"].shape
    H, P, d, case = s["H"], s["P"], s["d"], s["case"]
    keep, lens = case["keep"], s["lens"].long()
    j = torch.arange(width * P, device=DEV)
    table = s["table"].long()
    x = s["scores"][table].transpose(1, 2).reshape(n, H, width * P)
    if case["shared"]:
        x = torch.cumsum(x.double(), dim=1)[:, -1:].float()       # (in 64 bits: no order of the heads matters)
    x = torch.where(x.isnan(), -math.inf, x) + 0.0
    bits = x.view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)       # the numbers' order as whole numbers
    end = lens[:, None, None]
    key = torch.where((j < case["first"]) | (j >= end - case["recent"]), 1 << 33, key)
    key = torch.where(j < end, key, -(1 << 33))
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1]
    if keep > width * P:
        order = torch.cat([order, order.new_full((n, order.shape[1], keep - width * P), width * P)], dim=-1)
    kept = order[..., :keep]
    kept = torch.sort(torch.where(kept < end, kept, width * P), dim=-1)[0]
    there = kept < end
    kept = torch.where(there, kept, -1)
    new_lens = torch.clamp(lens, max=keep)
    # every kept entry to its place, in order
    src, there = kept.clamp(min=0).expand(n, H, keep), there.expand(n, H, keep)
    seq, head, dst = there.nonzero(as_tuple=True)
    src = src[seq, head, dst]
    page, slot = table[seq, src // P], src % P
    to, place = table[seq, dst // P], dst % P
    for x in ("k", "v"):
        pages, scales = s[x + "_pages"], s[x + "_scales"]
        if scales is None:
            pages[to, head, place] = pages[page, head, slot]
            continue
        mine = scales[page, head, slot // BLOCK]
        block = ((seq * H + head) * -(-keep // BLOCK)) + dst // BLOCK
        top = torch.zeros(n * H * -(-keep // BLOCK), device=DEV).scatter_reduce_(0, block, mine, "amax")[block]
        codes = pages.view(torch.uint8)
        moved = (codes[page, head, slot].view(DTYPES["fp8"]).float() * (mine / top)[:, None]).to(DTYPES["fp8"])
        codes[to, head, place] = moved.view(torch.uint8)
        scales[to, head, place // BLOCK] = top
    for x in (s["beta_pages"], s["scores"]):
        if x is not None:
            x[to, head, place] = x[page, head, slot]
    return [kept.to(torch.int32), new_lens.to(torch.int32)] + _pools(s) + [s["scores"]]


# ----------------------------------------------------------------------------
# The definition in 64 bits
# ----------------------------------------------------------------------------

def _turned(x, positions, theta):
    """The rotation of the pairs (e, e + d/2) as a product of complex numbers, in 64 bits."""
    x = x.double()
    if not theta:
        return x
    d = x.shape[-1]
    freq = torch.exp(torch.arange(d // 2, dtype=torch.float64, device=DEV) * (-2.0 * math.log(theta) / d))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), positions.unsqueeze(1) * freq).unsqueeze(1)
    z = torch.complex(x[..., : d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
    return torch.cat([z.real, z.imag], dim=-1)


def _e4m3(x):
    """The nearest e4m3 number, ties to the even one: 3 bits behind the leading one, steps of 2^-9 at least."""
    size = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(size - 3)
    return torch.round(x / step) * step


def _power(top):
    k = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))
    return torch.exp2(k).clamp(min=LEAST)


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _lens(case)
    op, P, H, d = case["op"], s["P"], s["H"], s["d"]
    table = s["table"].cpu().numpy()
    scales = dict(k=s["k_scales"], v=s["v_scales"])

    def rows(pages, b, first, count, scale=None):
        """Entries [first, first + count) of sequence b, [H, count, ...]."""
        a, z = first // P, -(-(first + count) // P)
        at = torch.from_numpy(table[b, a:z].astype(np.int64)).to(DEV)
        x = (pages if scale is None else pages.view(torch.uint8))[at]
        x = x.double() if scale is None else x.view(DTYPES["fp8"]).double()
        if scale is not None:
            x = (x.view(len(at), H, P // BLOCK, BLOCK, d) * scale[at].double()[..., None, None]).view(len(at), H, P, d)
        return x.transpose(0, 1).reshape(H, (z - a) * P, *x.shape[3:])[:, first - a * P: first - a * P + count]

    if op == "gather8":
        out = [rows(s[x + "_pages"], 0, case["start"], case["n"], scales[x]) for x in "kv"]
        return out + ([rows(s["beta_pages"], 0, case["start"], case["n"])] if case["beta"] else [])
    if op == "append8":
        return _exact_append(s, table, lens, new)
    if op == "evict":
        return _exact_evict(s, table, lens)
    nq, group = case["nq"], case["group"]
    q = _turned(s["q"], s["positions"], s["theta"])
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    total = s["scores"].double() if op == "score" else None
    for b in range(len(lens)):
        length = int(lens[b])
        if length == 0:
            continue
        k = rows(s["k_pages"], b, 0, length, scales["k"])
        v = rows(s["v_pages"], b, 0, length, scales["v"]) if op == "attend8" else None
        bias = rows(s["beta_pages"], b, 0, length) if case["beta"] else torch.zeros(H, length, dtype=torch.float64, device=DEV)
        weight = torch.zeros(H, length, dtype=torch.float64, device=DEV)
        for i in range(nq):
            seen = length - nq + i + 1 if case["causal"] else length
            if seen <= 0:
                continue
            row = q[b * nq + i].reshape(H, group, d)
            x = torch.matmul(row, k[:, :seen].transpose(1, 2).contiguous()) / math.sqrt(d) + bias[:, None, :seen]
            if op == "score":
                weight[:, :seen] += torch.softmax(x, dim=-1).sum(dim=1)
                continue
            lse[b * nq + i] = torch.logsumexp(x, dim=-1).reshape(-1)
            out[b * nq + i] = torch.matmul(torch.softmax(x, dim=-1), v[:, :seen].contiguous()).reshape(H * group, d)
        if op == "score":
            known = max(length - 1, 0)
            weight[:, :known] += rows(total, b, 0, length)[:, :known]
            for a in range(0, length, P):
                total[int(table[b, a // P]), :, : min(P, length - a)] = weight[:, a: a + P]
    return total if op == "score" else [out, lse]


def _exact_append(s, table, lens, new):
    P, H, d = s["P"], s["H"], s["d"]
    page, slot, block, old, at = [], [], [], [], []
    for b in range(len(lens)):
        j = np.arange(lens[b] - new[b], lens[b])
        page.append(table[b, j // P])
        slot.append(j % P)
        block.append(page[-1].astype(np.int64) * (P // BLOCK) + j % P // BLOCK)
        first = np.unique(j // BLOCK)
        at.append(table[b, first * BLOCK // P].astype(np.int64) * (P // BLOCK) + first * BLOCK % P // BLOCK)
        old.append(np.maximum(lens[b] - new[b] - first * BLOCK, 0))
    page, slot, block, old, at = (torch.from_numpy(np.concatenate(x).astype(np.int64)).to(DEV) for x in (page, slot, block, old, at))
    count = torch.zeros(s["k_pages"].shape[0] * (P // BLOCK), dtype=torch.int64, device=DEV)
    count[at] = old
    touched = torch.zeros_like(count, dtype=torch.bool)
    touched[at] = True
    pools, scales = [], []
    for x in ("k", "v"):
        y = (_turned(s[x], s["positions"], s["theta"]) if x == "k" else s[x].double()).float().double()
        pages = s[x + "_pages"].double().view(-1, H, P // BLOCK, BLOCK, d)
        scale = s[x + "_scales"].double().transpose(1, 2).reshape(-1, H)          # [blocks, H]
        top = torch.zeros(len(count), H, dtype=torch.float64, device=DEV)
        top.scatter_reduce_(0, block[:, None].expand(-1, H), y.abs().amax(dim=2), "amax")
        need = _power(top)
        now = torch.where((count > 0)[:, None], torch.maximum(scale, need), need)
        now = torch.where(touched[:, None], now, scale)
        ratio = torch.where(touched[:, None] & (count > 0)[:, None], scale / now, 1.0)
        by_page = ratio.view(-1, P // BLOCK, H).transpose(1, 2)[..., None, None]
        pages = _e4m3(pages * by_page).view(-1, H, P, d)
        pages[page, :, slot] = _e4m3(y / now[block][:, :, None])
        pools.append(pages)
        scales.append(now.view(-1, P // BLOCK, H).transpose(1, 2))
    if s["beta_pages"] is None:
        return pools + scales
    bias = s["beta_pages"].double()
    bias[page, :, slot] = s["beta"].double()
    return pools + scales + [bias]


def _exact_evict(s, table, lens):
    case, P, H, d = s["case"], s["P"], s["H"], s["d"]
    keep, alone = case["keep"], 1 if case["shared"] else H
    score = s["scores"].cpu().numpy()
    kept = np.full((len(lens), alone, keep), -1, dtype=np.int64)
    for b, n in enumerate(lens):
        n = int(n)
        x = score[table[b, : -(-n // P)]].transpose(1, 0, 2).reshape(H, -1)[:, :n].astype(np.float64)
        if case["shared"]:
            x = x.sum(axis=0, keepdims=True).astype(np.float32)
        for h in range(alone):
            left = max(0, min(n, keep) - min(n, case["first"]) - min(max(n - case["first"], 0), case["recent"]))
            inside = np.arange(min(n, case["first"]), max(n - case["recent"], min(n, case["first"])))
            best = inside[np.lexsort((inside, -x[h, inside]))[:left]]
            fixed = np.setdiff1d(np.arange(n), inside)
            ids = np.sort(np.concatenate([fixed, best])) if n > keep else np.arange(n)
            kept[b, h, : len(ids)] = ids
    out = [torch.from_numpy(kept).to(DEV), torch.from_numpy(np.minimum(lens, keep)).to(DEV)]
    # the moved entries: flat places of rows [page][head][slot]
    src, dst, block = [], [], []
    for b in range(len(lens)):
        for h in range(H):
            ids = kept[b, h % alone]
            ids = ids[ids >= 0]
            to = np.arange(len(ids))
            src.append((table[b, ids // P].astype(np.int64) * H + h) * P + ids % P)
            dst.append((table[b, to // P].astype(np.int64) * H + h) * P + to % P)
    src, dst = (torch.from_numpy(np.concatenate(x)).to(DEV) for x in (src, dst))
    factors = {}
    for x in ("k", "v"):
        pages = s[x + "_pages"].double().view(-1, d)
        moved = pages[src]
        if s["k_scales"] is not None:
            scale = s[x + "_scales"].double().view(-1)
            now = scale.clone()
            now[dst // BLOCK] = 0.0
            now.scatter_reduce_(0, dst // BLOCK, scale[src // BLOCK], "amax")
            moved = _e4m3(moved * (scale[src // BLOCK] / now[dst // BLOCK])[:, None])
            factors[x] = now.view(s[x + "_scales"].shape)
        pages[dst] = moved
        out.append(pages.view(s[x + "_pages"].shape))
    out += list(factors.values())
    for x in (s["beta_pages"], s["scores"]):
        if x is not None:
            y = x.double().view(-1)
            y[dst] = y[src]
            out.append(y.view(x.shape))
    return out


# ----------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------

def work(case):
    op, H, d = case["op"], case["H"], case["d"]
    held, given = SIZES[case["cache"]], SIZES[case["rows"]]
    lens, new = _lens(case)
    scale = 4 / BLOCK if case["cache"] == "fp8" else 0
    side = H * (d * held + scale)                                # one entry's keys or values
    bias = 4 * H if case["beta"] else 0
    if op in ("append8", "gather8"):
        rotate = 8 if case.get("rotate") else 0
        return {"bytes": int(int(new.sum()) * (2 * side + 2 * H * d * given + 2 * bias + rotate)),
                "flops": int(new.sum()) * H * d * (5 if rotate else 2)}
    total = int(lens.sum())
    if op == "evict":
        few = np.minimum(lens, case["keep"])
        moved = int(few[lens > case["keep"]].sum()) - case["first"] * int((lens > case["keep"]).sum())
        read = int(lens[lens > case["keep"]].sum()) * H * 4
        return {"bytes": int(read + 2 * moved * (2 * side + bias + 4 * H) + int(few.sum()) * 4 * (1 if case["shared"] else H)),
                "flops": int(lens.sum()) * H}
    rows = case["group"] * case["nq"]
    q = len(lens) * rows * H * (d * given + 4)
    if op == "attend8":
        return {"bytes": int(total * (2 * side + bias) + q + len(lens) * rows * H * d * given), "flops": 4 * total * H * d * rows}
    return {"bytes": int(total * (side + bias + 8 * H) + q), "flops": 2 * total * H * d * rows}
