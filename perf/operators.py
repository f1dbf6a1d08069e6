"""The paged key-value cache: appending to it, reading it back, attention over it.

Three operators, each through a public entry point of ``binding``:

* ``append``  new keys and values of several sequences into their pages, the
              keys rotated by the base model's RoPE on the way
              (``binding.paged_append``);
* ``gather``  a range of one sequence out of its pages, as the dense rows the
              compactor reads (``binding.paged_gather``);
* ``attend``  attention of the newest query rows of several sequences over
              their pages (``binding.paged_attend``).

Pages are [n_pages, H, P, d], the bias of compact entries [n_pages, H, P]
float32; a table [n_seqs, pages] of page numbers and the lengths say which
entries a sequence has.  The page size, head shapes and lengths are those of
the caches that the repository compacts: 8 KV heads of width 128 (4 query
heads each) and of width 256 (2 each), 655 or 1024 compact entries of 8k to
128k tokens, fresh tokens behind them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
WORKSPACE_BYTES = 80 << 20      # a serving program's one buffer, enough for every call


# ----------------------------------------------------------------------------
# The cases
# ----------------------------------------------------------------------------

def _append(name, seqs, lo, hi, new_lo, new_hi, H, d, P, dtype="bf16", rotate=True, beta=False, layout="token"):
    return dict(name=name, op="append", seqs=seqs, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, H=H, group=4, d=d, P=P,
                dtype=dtype, rotate=rotate, beta=beta, layout=layout)


def _gather(name, n, start, H, d, P, dtype="bf16", beta=False):
    return dict(name=name, op="gather", n=n, start=start, H=H, d=d, P=P, dtype=dtype, beta=beta)


def _attend(name, seqs, lo, hi, H, group, d, P, nq=1, causal=False, dtype="bf16", rotate=False, beta=False, empty=0):
    return dict(name=name, op="attend", seqs=seqs, lo=lo, hi=hi, H=H, group=group, d=d, P=P, nq=nq, causal=causal,
                dtype=dtype, rotate=rotate, beta=beta, empty=empty)


def listed():
    return [
        # one token of one conversation behind its compact entries: the smallest append
        _append("append_step_1", 1, 719, 719, 1, 1, 8, 128, 16),
        # a decode step of 64 conversations, k and v as slices of the fused projection's rows
        _append("append_step_64", 64, 700, 9000, 1, 1, 8, 128, 64),
        # prompts of 13 sequences of odd lengths in one call, about 8k tokens, wide heads, into a
        # cache that keeps the bias of compact entries
        _append("append_prompts_d256", 13, 2000, 9000, 37, 2000, 8, 256, 32, beta=True),
        # a layer's compact entries [H, t, d] with their bias, installed as they are, fp32
        _append("append_compact_fp32", 1, 1024, 1024, 1024, 1024, 8, 128, 16, dtype="fp32", rotate=False, beta=True,
                layout="head"),
        # the fresh tokens behind a preserved prefix, an odd count that starts inside a page
        _gather("gather_1k", 1087, 37, 8, 128, 16),
        # a long wide-headed cache on its way into the compactor: the largest copy
        _gather("gather_64k_d256", 65536, 0, 8, 256, 64),
        # one decode step of one conversation: 655 compact entries with their bias and 64 fresh ones,
        # the smallest call
        _attend("attend_step_compact", 1, 719, 719, 8, 4, 128, 16, beta=True),
        # the same step over an uncompacted 128k cache
        _attend("attend_step_128k", 1, 131136, 131136, 8, 4, 128, 64),
        # a decode step of 64 conversations between a word and 16k tokens, queries rotated here,
        # the last rows of the batch padding
        _attend("attend_batch_ragged", 64, 5, 16384, 8, 4, 128, 16, rotate=True, beta=True, empty=3),
        # a decode step of 48 conversations that are compacted every 8k tokens, wide heads
        _attend("attend_batch_d256", 48, 1024, 9216, 8, 2, 256, 32, beta=True),
        # 8 new tokens each (a checked draft), causal: 32 query rows per KV head
        _attend("attend_block_causal", 5, 1500, 20011, 8, 4, 128, 128, nq=8, causal=True, rotate=True),
        # the validation mode, narrow heads
        _attend("attend_fp32_d64", 7, 1, 3001, 2, 3, 64, 16, nq=2, causal=True, dtype="fp32", beta=True, empty=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: 1 to 256 sequences, 1 to 131136 entries, both
    types, the widths and page sizes the kernels take, up to 32 query rows."""
    op = rng.choice(["append", "gather", "attend", "attend", "attend"])
    H, d, P = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([64, 128, 256]), rng.choice([16, 32, 64, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    beta = rng.random() < 0.5
    row = 2 * H * d * (2 if dtype == "bf16" else 4)                  # bytes of one entry
    if op == "gather":
        n = min(_log(rng, 1, 131072), int(2.5e8 / row))
        return dict(_gather("", n, rng.choice([0, rng.randrange(0, 5000)]), H, d, P, dtype, beta), name="gather")
    seqs = _log(rng, 1, 256)
    if op == "append":
        most = max(1, min(8192, int(1.2e8 / row / seqs)))
        new = _log(rng, 1, most)
        new_lo = rng.choice([new, rng.randint(1, new)])
        lo = new + rng.randrange(0, 2000)
        return dict(_append("", seqs, lo, lo + rng.randrange(0, 4000), new_lo, new, H, d, P, dtype,
                            rng.random() < 0.7, beta, rng.choice(["token", "head"])), name="append")
    hi = min(_log(rng, 1, 131136), max(1, int(5e8 / row / seqs)))
    lo = min(hi, rng.choice([hi, _log(rng, 1, hi)]))
    group = rng.choice([1, 2, 3, 4, 8])
    nq = rng.choice([1, 1, 1, rng.randint(1, 32 // group)])
    return dict(_attend("", seqs, lo, hi, H, group, d, P, nq, rng.random() < 0.6, dtype, rng.random() < 0.5, beta,
                        rng.choice([0, 0, 1]) if seqs > 1 else 0), name="attend")


def _spread(lo, hi, n, salt):
    """n whole numbers from lo to hi, spread over their logarithm, in no order."""
    x = np.rint(np.geomspace(lo, hi, n) if n > 1 else np.array([hi])).astype(np.int64)
    return np.random.RandomState(salt).permutation(x)


def _lens(case):
    """(entries of each sequence after the call, new ones among them)."""
    if case["op"] == "gather":
        return np.array([case["start"] + case["n"]]), np.array([case["n"]])
    n = case["seqs"]
    lens = _spread(case["lo"], case["hi"], n, n)
    if case["op"] == "attend":
        if case["empty"]:
            lens[n - case["empty"]:] = 0
        return lens, np.full(n, case["nq"])
    return lens, _spread(case["new_lo"], case["new_hi"], n, n + 1)


def _theta(d):
    return 1e4 if d == 256 else 1e6     # the wide-headed models' base, and the others'


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    H, d, P, dt = case["H"], case["d"], case["P"], DTYPES[case["dtype"]]
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
             theta=_theta(d) if case.get("rotate") else 0.0, beta_pages=None)
    if case["op"] == "append":
        s.update(k_pages=torch.zeros(pages, H, P, d, dtype=dt, device=DEV),
                 v_pages=torch.zeros(pages, H, P, d, dtype=dt, device=DEV))
        if case["beta"]:
            s["beta_pages"] = torch.zeros(pages, H, P, device=DEV)
    else:
        s.update(k_pages=rand(pages, H, P, d), v_pages=rand(pages, H, P, d))
        if case["beta"]:
            s["beta_pages"] = rand(pages, H, P, dtype=torch.float32)
    if case["op"] == "gather":
        s["out"] = (torch.empty(H, case["n"], d, dtype=dt, device=DEV), torch.empty(H, case["n"], d, dtype=dt, device=DEV))
        if case["beta"]:
            s["out"] += (torch.empty(H, case["n"], device=DEV),)
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
    if case["op"] == "append":
        s["offsets"] = None
        if new.min() != new.max():
            s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
        s["beta"] = rand(H, tokens, dtype=torch.float32).transpose(0, 1) if case["beta"] else None
    else:
        s["scale"] = 1.0 / math.sqrt(d)
        s["out"] = torch.empty(tokens, Hq, d, dtype=dt, device=DEV)
        s["ws"] = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    return s


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"append": _plain_append, "gather": _plain_gather, "attend": _plain_attend}[op](s)


def _own(s, op):
    from paper_2606_07878_amd import binding
    if op == "append":
        binding.paged_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lens"], offsets=s["offsets"],
                             positions=s["positions"], rope_theta=s["theta"], beta=s["beta"],
                             beta_pages=s["beta_pages"])
        return [x for x in (s["k_pages"], s["v_pages"], s["beta_pages"]) if x is not None]
    if op == "gather":
        return list(binding.paged_gather(s["k_pages"], s["v_pages"], s["table"], s["lens"], 0, s["case"]["n"],
                                         start=s["case"]["start"], beta_pages=s["beta_pages"], out=s["out"]))
    return binding.paged_attend(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], causal=s["case"]["causal"],
                                beta_pages=s["beta_pages"], q_positions=s["positions"], rope_theta=s["theta"],
                                workspace=s["ws"], out=s["out"])


def _rotated(x, positions, theta):
    """x [tokens, heads, d] in 32 bits, rotated at the tokens' positions (angles in 64 bits)."""
    x = x.float()
    if not theta:
        return x
    half = x.shape[-1] // 2
    inv = torch.pow(torch.tensor(theta, dtype=torch.float64, device=DEV),
                    -torch.arange(half, dtype=torch.float64, device=DEV) / half)
    angle = positions[:, None] * inv
    c, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)


def _plain_append(s):
    P, n, tokens = s["P"], s["table"].shape[0], s["k"].shape[0]
    i = torch.arange(tokens, device=DEV)
    if s["offsets"] is None:
        seq = i // (tokens // n)
        end = (seq + 1) * (tokens // n)
    else:
        seq = torch.searchsorted(s["offsets"], i.to(torch.int32), right=True) - 1
        end = s["offsets"][seq + 1]
    j = s["lens"][seq] - end + i
    page, slot = s["table"][seq, j // P].long(), j % P
    s["k_pages"][page, :, slot] = _rotated(s["k"], s["positions"], s["theta"]).to(s["k"].dtype)
    s["v_pages"][page, :, slot] = s["v"]
    if s["beta_pages"] is None:
        return [s["k_pages"], s["v_pages"]]
    s["beta_pages"][page, :, slot] = s["beta"]
    return [s["k_pages"], s["v_pages"], s["beta_pages"]]


def _plain_gather(s):
    j = torch.arange(s["case"]["n"], device=DEV) + s["case"]["start"]
    page, slot = s["table"][0, j // s["P"]].long(), j % s["P"]
    there = j < s["lens"][0]
    got = [s["k_pages"][page, :, slot], s["v_pages"][page, :, slot]]
    got = [torch.where(there[:, None, None], x, 0.0).transpose(0, 1).contiguous() for x in got]
    if s["beta_pages"] is not None:
        got.append(torch.where(there[:, None], s["beta_pages"][page, :, slot], 0.0).t().contiguous())
    return got


def _plain_attend(s):
    n, width = s["table"].shape
    H, d, P = s["H"], s["d"], s["P"]
    group, nq = s["case"]["group"], s["case"]["nq"]
    table = s["table"].long()
    k = s["k_pages"][table].float().transpose(1, 2).reshape(n, H, width * P, d)
    q = _rotated(s["q"], s["positions"], s["theta"]).reshape(n, nq, H, group, d).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.reshape(n, H, group * nq, d), k.transpose(2, 3)) * s["scale"]
    del k
    if s["beta_pages"] is not None:
        x += s["beta_pages"][table].transpose(1, 2).reshape(n, H, 1, width * P)
    # row (g, i) sits at entry lens - nq + i and, where causal, sees entries up to its own
    last = s["lens"][:, None] - (nq if s["case"]["causal"] else 1)
    if s["case"]["causal"]:
        last = last + torch.arange(nq, device=DEV)
    else:
        last = last.expand(n, nq)
    last = last[:, None, None, :, None].expand(n, 1, group, nq, 1).reshape(n, 1, group * nq, 1)
    hidden = torch.arange(width * P, device=DEV) > last
    x.masked_fill_(hidden, -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    total = e.sum(dim=-1, keepdim=True)
    del x
    v = s["v_pages"][table].float().transpose(1, 2).reshape(n, H, width * P, d)
    o = torch.matmul(e, v) / torch.where(total > 0, total, 1.0)
    o = o.reshape(n, H, group, nq, d).permute(0, 3, 1, 2, 4)
    return o.reshape(n * nq, H * group, d).to(s["q"].dtype)


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


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _lens(case)
    P, H, d = s["P"], s["H"], s["d"]
    table = s["table"].cpu().numpy()

    def rows(pages, b, first, count):
        """Entries [first, first + count) of sequence b, [H, count, ...]."""
        a, z = first // P, -(-(first + count) // P)
        x = pages[torch.from_numpy(table[b, a:z].astype(np.int64)).to(DEV)].double()
        return x.transpose(0, 1).reshape(H, (z - a) * P, *x.shape[3:])[:, first - a * P: first - a * P + count]

    if case["op"] == "gather":
        pools = [s["k_pages"], s["v_pages"]] + ([s["beta_pages"]] if case["beta"] else [])
        return [rows(x, 0, case["start"], case["n"]) for x in pools]
    if case["op"] == "append":
        news = [(s["k_pages"], _turned(s["k"], s["positions"], s["theta"])), (s["v_pages"], s["v"].double())]
        if case["beta"]:
            news.append((s["beta_pages"], s["beta"].double()))
        out = []
        for pool, x in news:
            pool, at = pool.double(), 0
            for b in range(len(lens)):
                done = 0
                while done < new[b]:
                    j = int(lens[b] - new[b]) + done
                    step = int(min(P - j % P, new[b] - done))
                    pool[int(table[b, j // P]), :, j % P: j % P + step] = x[at + done: at + done + step].transpose(0, 1)
                    done += step
                at += int(new[b])
            out.append(pool)
        return out
    nq, group = case["nq"], case["group"]
    q = _turned(s["q"], s["positions"], s["theta"])
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    for b in range(len(lens)):
        length = int(lens[b])
        if length == 0:
            continue
        k, v = rows(s["k_pages"], b, 0, length), rows(s["v_pages"], b, 0, length)
        bias = rows(s["beta_pages"], b, 0, length) if case["beta"] else torch.zeros(H, length, dtype=torch.float64, device=DEV)
        for i in range(nq):
            seen = length - nq + i + 1 if case["causal"] else length
            if seen <= 0:
                continue
            row = q[b * nq + i].reshape(H, group, d)
            x = torch.matmul(row, k[:, :seen].transpose(1, 2).contiguous()) / math.sqrt(d) + bias[:, None, :seen]
            w = torch.softmax(x, dim=-1)
            out[b * nq + i] = torch.matmul(w, v[:, :seen].contiguous()).reshape(H * group, d)
    return out


def work(case):
    H, d = case["H"], case["d"]
    size = 2 if case["dtype"] == "bf16" else 4
    lens, new = _lens(case)
    entry = H * (2 * d * size + (4 if case["beta"] else 0))      # one entry's key, value and bias
    if case["op"] != "attend":
        extra = 8 if case.get("rotate") else 0
        return {"bytes": int(new.sum()) * (2 * entry + extra), "flops": int(new.sum()) * (3 * H * d if extra else 0)}
    rows, total = case["group"] * case["nq"], int(lens.sum())
    return {"bytes": total * entry + len(lens) * rows * H * d * size * 2, "flops": 4 * total * H * d * rows}
