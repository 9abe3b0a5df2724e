"""The calls around a decode loop that a serving program makes, as cases to be timed: prompts and caches in pages.

* ``prompt``      hill_prompt_attn: causal attention over packed prompts of different lengths, each perhaps behind
                  earlier context of its own, everything visible or the first ``sinks`` tokens and the newest ``window``;
* ``importance``  hill_prompt_importance: the attention weights that the prompts' tokens receive, summed over the
                  queries (all, or the ``newest`` of each prompt) and added to a running importance;
* ``paged``       hill_paged_attn: one query token per sequence over a cache stored in pages, in 16 bits or in E4M3
                  with a scale per row, with or without the attention weights added to the running importance;
* ``write``       hill_paged_write: new tokens into their pages, quantised on the way where the cache is held in E4M3,
                  then hill_paged_read: the same rows as the cache stands for them.

A row of an E4M3 cache has the codes e4m3(x * (448 / amax)), amax = max |x|, and the scale amax / 448; scales
[pages][Hkv][page][2] holds (K scale, V scale).  Where ``own`` is false every case runs in elementary torch operations
in 32 bits, the sequences side by side, padded to the longest.
"""
from __future__ import annotations

import math
import random
import zlib

import torch

own = False

D = 128
ALL = 1 << 30   # a window that hides nothing; all queries
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
BASE = dict(op="prompt", batch=1, heads=32, kv_heads=8, tokens=4096, past=0, ragged=False, dtype="bf16", sinks=0,
            window=ALL, newest=ALL, kvh=False, accum=False, page=64, e4m3=False)


def _case(name, **over):
    return dict(BASE, name=name, **over)


def listed():
    return [
        # the smallest prompt: one chat turn of a grouped-query model, an odd length
        _case("prompt-1x131-gqa", tokens=131),
        # a batch of requests of different lengths, packed
        _case("prompt-8x2k-gqa-ragged", batch=8, tokens=2048, ragged=True),
        # the next chunk of long documents behind what is cached of them, 4 sinks and a window of 4096 tokens
        _case("prompt-2x2k-past14k-window4k", batch=2, heads=64, tokens=2048, past=14336, sinks=4, window=4096),
        # the largest: a long document of a 32-head model
        _case("prompt-1x16k-mha", kv_heads=32, tokens=16384, dtype="fp16"),
        # first weights of a batch's tokens from the last 64 queries of each prompt, every KV head with its own
        _case("importance-4x4k-newest64-kvh", op="importance", batch=4, tokens=4096, ragged=True, newest=64, kvh=True),
        # first weights of a long document's tokens from all of its queries
        _case("importance-1x8k-gqa", op="importance", tokens=8192),
        # the smallest decode: one chat turn over small pages, an odd length
        _case("paged-1x4k-gqa", op="paged", tokens=4001, page=16),
        # long documents of different lengths of a grouped-query model
        _case("paged-8x32k-gqa", op="paged", batch=8, tokens=32768, ragged=True),
        # the smallest decode from E4M3
        _case("paged_e4m3-1x4k-gqa", op="paged", tokens=4001, page=16, e4m3=True),
        # long documents of a 32-head model in E4M3, the weights accumulated for a later eviction
        _case("paged_e4m3-4x32k-mha-accum", op="paged", batch=4, kv_heads=32, tokens=32768, ragged=True, dtype="fp16",
              accum=True, e4m3=True),
        # one decode step of a batch into an E4M3 cache, and the step's rows read back
        _case("write_e4m3-16x1", op="write", batch=16, tokens=1, past=4096, page=16, e4m3=True),
        # the prompts of a batch into an E4M3 cache, and what it then stands for
        _case("write_e4m3-4x16k-prompt", op="write", batch=4, tokens=16411, ragged=True, e4m3=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges: 1 to 16 sequences, every head layout; prompts of one token to 16K, alone or
    behind up to 16K tokens; caches of up to 128K tokens, pages of 16 to 256, windows from 64 tokens to everything."""
    while True:
        c = dict(BASE, op=rng.choice(["prompt", "prompt", "importance", "paged", "paged", "write"]))
        c["heads"], c["kv_heads"] = rng.choice([(32, 32), (32, 8), (32, 8), (64, 8), (28, 4), (40, 40), (32, 1)])
        c["batch"] = _log(rng, 1, 16)
        c["dtype"] = rng.choice(["fp16", "bf16"])
        c["ragged"] = rng.random() < 0.5
        c["sinks"] = rng.choice([0, 0, 4, 16, 61])
        c["page"] = rng.choice([16, 16, 32, 64, 112, 256])
        c["e4m3"] = rng.random() < 0.5
        if c["op"] in ("prompt", "importance"):
            c["tokens"] = _log(rng, 1, 16384)
            c["past"] = rng.choice([0, 0, _log(rng, 1, 16384)])
            if rng.random() < 0.3:
                c["window"] = _log(rng, 64, max(64, c["tokens"] + c["past"]))
            if c["op"] == "importance":
                c["kvh"] = rng.random() < 0.5
                c["newest"] = rng.choice([ALL, 16, 64, 200])
            most = 1 << 33 if c["op"] == "prompt" else 1 << 31
            if c["batch"] * c["heads"] * c["tokens"] * (c["tokens"] + c["past"]) > most:
                continue
            if c["batch"] * (c["tokens"] + c["past"]) * c["kv_heads"] > 1 << 20:
                continue
        elif c["op"] == "paged":
            c["tokens"] = _log(rng, 200, 131072)
            c["accum"] = rng.random() < 0.4
            c["kvh"] = rng.random() < 0.3
            if rng.random() < 0.5:
                c["window"] = _log(rng, 64, c["tokens"])
            rows = c["batch"] * c["tokens"] * c["kv_heads"]
            if rows > (8 << 20 if c["e4m3"] else 4 << 20) or c["batch"] * c["tokens"] * c["heads"] > 64 << 20:
                continue
        else:
            c["tokens"] = rng.choice([1, _log(rng, 1, 16384)])
            c["past"] = rng.choice([0, _log(rng, 1, 16384)])
            if c["batch"] * (c["tokens"] + c["past"]) * c["kv_heads"] > 1 << 20:
                continue
        return c


# ---------------------------------------------------------------- inputs
def _lengths(case):
    """New tokens of every sequence (of ``paged`` cases: cached ones); ragged: the longest, and others down to a half."""
    n, B = case["tokens"], case["batch"]
    if not case["ragged"]:
        return [n] * B
    r = random.Random(zlib.crc32(repr(sorted((k, v) for k, v in case.items() if k != "name")).encode()))
    return [n] + [r.randint(max(1, n // 2), n) for _ in range(B - 1)]


def _starts(lengths):
    return [sum(lengths[:b]) for b in range(len(lengths) + 1)]


def _generator(seed, what):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((int(seed), what)).encode()))


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _channels(g, Hkv):
    """Per KV head and channel: a spread and an offset; a few channels are far larger, as keys have them."""
    spread = 0.5 + torch.rand(Hkv, D, generator=g, device="cuda")
    offset = torch.randn(Hkv, D, generator=g, device="cuda")
    loud = torch.rand(Hkv, D, generator=g, device="cuda") < 0.03
    return spread * (1 + 2 * loud), offset * (0.2 + 3 * loud)


def _rows(g, n, spread, offset):
    return torch.randn(n, *spread.shape, generator=g, device="cuda") * spread + offset


def _keys(g, n, ch, u):
    """Keys [n][Hkv][d] of which one in 64 points along the query direction u: the heavy hitters of real attention."""
    heavy = (torch.rand(n, 1, 1, generator=g, device="cuda") < 1 / 64) * torch.rand(n, 1, 1, generator=g, device="cuda")
    return _rows(g, n, *ch) + heavy * 0.35 * u


def _queries(g, n, H, u, dt):
    return (u.repeat_interleave(H // u.shape[0], 0) + 0.25 * torch.randn(n, H, D, generator=g, device="cuda")).to(dt)


def _quantise(x):
    """E4M3 codes and scales of rows x (last axis 128)."""
    amax = x.abs().amax(-1, keepdim=True)
    codes = torch.where(amax > 0, x * (448 / amax), 0.0).clamp(-448, 448).to(torch.float8_e4m3fn)
    return codes, (amax / 448)[..., 0]


def prepare(case, seed):
    B, H, Hkv, dt, op = case["batch"], case["heads"], case["kv_heads"], DTYPES[case["dtype"]], case["op"]
    g = _generator(seed, "inputs")
    ck, cv = _channels(g, Hkv), _channels(g, Hkv)
    u = torch.randn(Hkv, D, generator=g, device="cuda")
    new = _lengths(case)
    s = {"case": case}
    if op in ("prompt", "importance"):
        held = [n + case["past"] for n in new]
        s["q_start"], s["k_start"] = _ints(_starts(new)), _ints(_starts(held))
        s["q"] = _queries(g, sum(new), H, u, dt)
        s["k"], s["v"] = _keys(g, sum(held), ck, u).to(dt), _rows(g, sum(held), *cv).to(dt)
        s["cap"] = max(held)
        if op == "prompt":
            s["out"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(sum(new), H, device="cuda")
        else:
            s["lse"] = _plain_prompt(s, case)[1]
            s["accum"] = torch.rand(B, *([Hkv] if case["kvh"] else []), s["cap"], generator=g, device="cuda")
        if own:
            from paper_2602_18750_gb300 import hill

            hill.load()
            s["desc"] = hill.make_packed(s["q"], s["k"], s["v"], B)
            s["ws"] = hill.alloc_prompt_workspace(s["desc"]) if op == "importance" else None
        return s
    # a pool of pages, somewhat more than are in use, handed out in any order
    held = new if op == "paged" else [n + case["past"] for n in new]
    page = case["page"]
    cols = -(-max(held) // page)
    used = [-(-n // page) for n in held]
    pages = sum(used) + 8
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    s["table"] = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    for b, at in enumerate(_starts(used)[:-1]):
        s["table"][b, :used[b]] = order[at:at + used[b]]
    s["k_pool"], s["v_pool"] = (torch.zeros(pages, Hkv, page, D, dtype=torch.float8_e4m3fn if case["e4m3"] else dt, device="cuda")
                                for _ in range(2))
    s["scales"] = torch.zeros(pages, Hkv, page, 2, device="cuda") if case["e4m3"] else None
    cap = s["cap"] = cols * page
    if op == "paged" or case["past"]:   # the pages as earlier calls left them
        each = max(1, (1 << 24) // (Hkv * page * D))
        for p0 in range(0, pages, each):
            n = min(each, pages - p0)
            rows = [x.view(n, page, Hkv, D).transpose(1, 2) for x in (_keys(g, n * page, ck, u).to(dt), _rows(g, n * page, *cv).to(dt))]
            for i, (x, pool) in enumerate(zip(rows, (s["k_pool"], s["v_pool"]))):
                if case["e4m3"]:
                    codes, s["scales"][p0:p0 + n, ..., i] = _quantise(x.float())
                    pool[p0:p0 + n].view(torch.uint8).copy_(codes.view(torch.uint8))
                else:
                    pool[p0:p0 + n] = x
    if op == "paged":
        s["q"] = _queries(g, B, H, u, dt)
        s["lens"] = _ints([[n] * Hkv for n in held] if case["kvh"] else held)
        s["out"] = torch.zeros(B, H, D, device="cuda")
        s["accum"] = torch.rand(B, *([Hkv] if case["kvh"] else []), cap, generator=g, device="cuda") * (H / cap) if case["accum"] else None
    else:
        s["k_new"], s["v_new"] = _keys(g, sum(new), ck, u).to(dt), _rows(g, sum(new), *cv).to(dt)
        s["starts"], s["begin"], s["end"] = _ints(_starts(new)), _ints([case["past"]] * B), _ints(held)
        s["K"], s["V"] = (torch.zeros(B, Hkv, cap, D, dtype=dt, device="cuda") for _ in range(2))
    if own:
        from paper_2602_18750_gb300 import hill

        hill.load()
        s["pages"] = hill.make_pages(s["k_pool"], s["v_pool"], s["table"], s["scales"])
        if op == "paged":
            s["desc"] = hill.make_desc_paged(s["q"], s["pages"])
            s["ws"] = hill.alloc_window_workspace(s["desc"], case["accum"])
        else:
            s["desc"] = hill.make_desc(torch.empty(B, H, D, dtype=dt, device="cuda"), s["K"], s["V"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"prompt": _plain_attn, "importance": _plain_importance, "paged": _plain_paged, "write": _plain_write}[case["op"]](s, case)


def _run_own(s, case):
    from paper_2602_18750_gb300 import hill

    op = case["op"]
    if op == "prompt":
        hill.hill_prompt_attn(s["desc"], s["q"], s["k"], s["v"], s["q_start"], s["k_start"], case["sinks"], case["window"],
                              s["out"], lse=s["lse"])
    elif op == "importance":
        hill.hill_prompt_importance(s["desc"], s["q"], s["k"], s["lse"], s["q_start"], s["k_start"], case["sinks"],
                                    case["window"], case["newest"], s["accum"], kvh=case["kvh"], ws=s["ws"])
    elif op == "paged":
        hill.hill_paged_attn(s["desc"], s["q"], s["pages"], s["lens"], case["sinks"], case["window"], s["out"],
                             accum=s["accum"], kvh=case["kvh"], ws=s["ws"])
    else:
        hill.hill_paged_write(s["desc"], s["pages"], s["k_new"], s["v_new"], s["starts"], s["begin"])
        hill.hill_paged_read(s["desc"], s["pages"], s["begin"], s["end"], case["tokens"], s["K"], s["V"])
    return _outputs(s, case)


def _outputs(s, case):
    names = {"prompt": ("out", "lse"), "importance": ("accum",), "paged": ("out", "accum") if case["accum"] else ("out",),
             "write": ("K", "V")}[case["op"]]
    return {n: s[n] for n in names}


def _padded(x, start, n):
    """Packed rows [T][...] as [B][n][...], places past a sequence's own holding any row."""
    at = start[:-1, None].long() + torch.arange(n, device="cuda")
    return x[at.clamp(max=max(0, x.shape[0] - 1))]


def _packed(x, start):
    """[B][n][...] back to packed rows."""
    lens = (start[1:] - start[:-1])[:, None]
    return x[torch.arange(x.shape[1], device="cuda") < lens]


def _logits(s, case):
    """Base-e logits [B][Hkv][G][nq][nk] of padded prompts, -inf where a query does not look (or is none)."""
    B, H, Hkv = case["batch"], case["heads"], case["kv_heads"]
    nq, nk = case["tokens"], case["tokens"] + case["past"]
    q = _padded(s["q"], s["q_start"], nq).float().view(B, nq, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    k = _padded(s["k"], s["k_start"], nk).float().permute(0, 2, 3, 1)
    z = (q @ k).div_(math.sqrt(D)).view(B, Hkv, H // Hkv, nq, nk)
    lq, lk = ((x[1:] - x[:-1]).long()[:, None, None] for x in (s["q_start"], s["k_start"]))
    i, j = torch.arange(nq, device="cuda")[:, None], torch.arange(nk, device="cuda")
    pos = i + (lk - lq)
    seen = (i < lq) & (j <= pos) & ((j < case["sinks"]) | (j > pos - case["window"]))
    return z.masked_fill_(~seen[:, None, None], -math.inf)


def _plain_prompt(s, case):
    """(out, lse) of packed rows."""
    B, H = case["batch"], case["heads"]
    z = _logits(s, case)
    top = z.amax(-1, keepdim=True).clamp_min(-3e38)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = _padded(s["v"], s["k_start"], z.shape[-1]).float().transpose(1, 2)
    o = (p.flatten(2, 3) @ v).view(*p.shape[:4], D) / total.clamp_min(1e-30)
    lse = (top + total.log())[..., 0]
    return (_packed(o.permute(0, 3, 1, 2, 4).reshape(B, -1, H, D), s["q_start"]),
            _packed(lse.permute(0, 3, 1, 2).reshape(B, -1, H), s["q_start"]))


def _plain_attn(s, case):
    out, lse = _plain_prompt(s, case)
    s["out"].copy_(out)
    s["lse"].copy_(lse)
    return _outputs(s, case)


def _plain_importance(s, case):
    B, H, Hkv = case["batch"], case["heads"], case["kv_heads"]
    z = _logits(s, case)
    lse = _padded(s["lse"], s["q_start"], z.shape[3]).view(B, -1, Hkv, H // Hkv).permute(0, 2, 3, 1)
    i, lq = torch.arange(z.shape[3], device="cuda"), (s["q_start"][1:] - s["q_start"][:-1])[:, None]
    counts = (i < lq) & (i >= lq - case["newest"])
    p = z.sub_(lse[..., None]).exp_().mul_(counts[:, None, None, :, None])
    s["accum"] += p.sum((2, 3)) if case["kvh"] else p.sum((1, 2, 3))
    return _outputs(s, case)


def _slots(s, cols):
    """Rows of the pools (pages and slots flat) of positions cols [..][n], and of each sequence."""
    page = s["k_pool"].shape[2]
    table = s["table"].view(s["table"].shape[0], *[1] * (cols.dim() - 2), -1).expand(*cols.shape[:-1], -1)
    return table.gather(-1, cols // page).long().clamp_min(0), cols % page


def _held(pool, scales, pg, slot, Hkv):
    """Values [B][Hkv][n][d] in 32 bits of the rows (pg, slot) [B][Hkv][n]."""
    h = torch.arange(Hkv, device="cuda")[:, None]
    if scales is None:
        return pool[pg, h, slot].float()
    return pool.view(torch.uint8)[pg, h, slot].view(torch.float8_e4m3fn).float() * scales[pg, h, slot][..., None]


def _plain_paged(s, case):
    B, H, Hkv, cap = case["batch"], case["heads"], case["kv_heads"], s["cap"]
    n = s["lens"][..., None].clamp(0, cap).long()   # [rows][1]
    sinks, window = case["sinks"], case["window"]
    if sinks + window >= cap:   # every position is looked at
        cols = torch.arange(cap, device="cuda").expand(*n.shape[:-1], cap)
        valid = (cols < n) & ((cols < sinks) | (cols >= n - window))
    else:
        first, rest = torch.arange(sinks, device="cuda").expand(*n.shape[:-1], sinks), n - window + torch.arange(window, device="cuda")
        valid = torch.cat(((first < n) & (first < n - window), rest >= 0), -1)
        cols = torch.cat((first, rest), -1).clamp(0, cap - 1)
    by_head = (cols if case["kvh"] else cols[:, None]).expand(B, Hkv, cols.shape[-1])
    pg, slot = _slots(s, by_head)
    k, v = (_held(s[p], None if s["scales"] is None else s["scales"][..., i], pg, slot, Hkv) for i, p in enumerate(("k_pool", "v_pool")))
    seen = (valid if case["kvh"] else valid[:, None])[:, :, None]   # [B][Hkv or 1][1][n]
    z = s["q"].float().view(B, Hkv, H // Hkv, D) @ k.transpose(-1, -2) / math.sqrt(D)
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(z - torch.where(top > -math.inf, top, 0.0)), 0.0)
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-30)
    s["out"].copy_((p @ v).view(B, H, D))
    if case["accum"]:
        s["accum"].scatter_add_(-1, cols, p.sum(2) if case["kvh"] else p.sum((1, 2)))
    return _outputs(s, case)


def _plain_write(s, case):
    B, Hkv, page = case["batch"], case["kv_heads"], case["page"]
    T = s["k_new"].shape[0]
    b = torch.searchsorted(s["starts"], torch.arange(T, device="cuda", dtype=torch.int32), right=True) - 1
    at = (s["begin"][b] + torch.arange(T, device="cuda") - s["starts"][b]).long()   # positions
    pg, slot, h = s["table"][b, at // page].long()[:, None], (at % page)[:, None], torch.arange(Hkv, device="cuda")
    put = lambda i, x, pool: pool.index_put_((pg, h, slot), x)
    if case["e4m3"]:
        def put(i, x, pool):
            codes, scale = _quantise(x.float())
            pool.view(torch.uint8).index_put_((pg, h, slot), codes.view(torch.uint8))
            s["scales"][..., i].index_put_((pg, h, slot), scale)
    put(0, s["k_new"], s["k_pool"])
    put(1, s["v_new"], s["v_pool"])
    h, flat = torch.arange(Hkv, device="cuda"), lambda i, p: (s["scales"][..., i] if case["e4m3"] else None)
    for i, (pool, to) in enumerate(((s["k_pool"], s["K"]), (s["v_pool"], s["V"]))):
        held = _held(pool, flat(i, pool), pg.T[None].expand(1, Hkv, T), slot.T[None].expand(1, Hkv, T), Hkv)[0]
        to.index_put_((b[:, None], h, at[:, None]), held.transpose(0, 1).to(to.dtype))
    return _outputs(s, case)


def _pairs(case, n):
    """(query, key) pairs that n new tokens behind ``past`` others look at."""
    w, first = case["window"], case["past"] + max(0, n - case["newest"])
    return sum(min(p + 1, w) + min(case["sinks"], max(0, p + 1 - w)) for p in range(first, case["past"] + n))


def work(case):
    B, H, Hkv, new = case["batch"], case["heads"], case["kv_heads"], _lengths(case)
    row = 2 * ((D + 4) if case["e4m3"] else 2 * D)   # K and V of one token and KV head
    if case["op"] in ("prompt", "importance"):
        pairs = sum(_pairs(case, n) for n in new) * H
        queries = sum(min(n, case["newest"]) for n in new) * H
        keys = sum(n + case["past"] for n in new) * Hkv
        if case["op"] == "prompt":
            return {"bytes": queries * (4 * D + 4) + keys * 4 * D, "flops": 4 * D * pairs}
        return {"bytes": queries * (2 * D + 4) + keys * 2 * D + 8 * (keys if case["kvh"] else keys // Hkv), "flops": 2 * D * pairs}
    if case["op"] == "paged":
        seen = sum(min(n, min(case["sinks"], max(0, n - case["window"])) + case["window"]) for n in new)
        accum = 8 * seen * (Hkv if case["kvh"] else 1) if case["accum"] else 0
        return {"bytes": seen * Hkv * row + accum + 6 * B * H * D, "flops": 4 * H * D * seen}
    rows = sum(new) * Hkv
    return {"bytes": rows * (4 * D + 2 * row + 4 * D), "flops": 4 * D * rows}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"prompt": _exact_prompt, "importance": _exact_prompt, "paged": _exact_paged, "write": _exact_write}[case["op"]](s, case)


def _exact_prompt(s, case):
    """One sequence and query head after another, 2048 queries at a time."""
    H, Hkv, weights = case["heads"], case["kv_heads"], case["op"] == "importance"
    new = _lengths(case)
    out = torch.zeros(sum(new), H, D, dtype=torch.float64, device="cuda") if not weights else None
    lse = s["lse"].double() if weights else torch.zeros(sum(new), H, dtype=torch.float64, device="cuda")
    accum = s["accum"].double() if weights else None
    q0 = k0 = 0
    for b, n in enumerate(new):
        m = n + case["past"]
        j = torch.arange(m, device="cuda")
        first = max(0, n - case["newest"]) if weights else 0
        for h in range(H):
            g = h // (H // Hkv)
            K, V = s["k"][k0:k0 + m, g].double(), s["v"][k0:k0 + m, g].double()
            for i0 in range(first, n, 2048):
                i1 = min(n, i0 + 2048)
                at = torch.arange(i0, i1, device="cuda")[:, None] + case["past"]
                hidden = (j > at) | ((at - j >= case["window"]) & (j >= case["sinks"]))
                z = (s["q"][q0 + i0:q0 + i1, h].double() @ K.T) * D ** -0.5
                z[hidden] = -math.inf
                if weights:
                    to = accum[b, g] if case["kvh"] else accum[b]
                    to[:m] += torch.exp(z - lse[q0 + i0:q0 + i1, h, None]).sum(0)
                else:
                    lse[q0 + i0:q0 + i1, h] = torch.logsumexp(z, 1)
                    out[q0 + i0:q0 + i1, h] = torch.softmax(z, 1) @ V
        q0, k0 = q0 + n, k0 + m
    return {"accum": accum} if weights else {"out": out, "lse": lse}


def _exact_paged(s, case):
    H, Hkv, page = case["heads"], case["kv_heads"], case["page"]
    out = torch.zeros(case["batch"], H, D, dtype=torch.float64, device="cuda")
    accum = s["accum"].double() if case["accum"] else None
    for b, n in enumerate(_lengths(case)):
        shown = list(range(min(case["sinks"], max(0, n - case["window"])))) + list(range(max(0, n - case["window"]), n))
        shown = torch.tensor(shown, dtype=torch.long, device="cuda")
        pg, slot = s["table"][b].long()[torch.div(shown, page, rounding_mode="floor")], shown % page
        for g in range(Hkv):
            k, v = (s[p].view(torch.uint8 if case["e4m3"] else s[p].dtype)[pg, g, slot] for p in ("k_pool", "v_pool"))
            if case["e4m3"]:
                k, v = (x.view(torch.float8_e4m3fn).double() * s["scales"][pg, g, slot, i].double()[:, None] for i, x in enumerate((k, v)))
            h = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
            p = torch.softmax(s["q"][b, h].double() @ k.double().T * D ** -0.5, -1)
            out[b, h] = p @ v.double()
            if accum is not None:
                (accum[b, g] if case["kvh"] else accum[b])[shown] += p.sum(0)
    return {"out": out, "accum": accum} if case["accum"] else {"out": out}


def _exact_write(s, case):
    """The rows that the cache then stands for: the new ones, to the nearest of E4M3's values where it is held so."""
    t = 0
    for b, n in enumerate(_lengths(case)):
        for new, to in ((s["k_new"], s["K"]), (s["v_new"], s["V"])):
            x = new[t:t + n].transpose(0, 1)
            if case["e4m3"]:   # (the codes' own rule is in 32 bits, the values of codes and scales in 64)
                amax = x.float().abs().max(-1, keepdim=True).values
                y = (x.float() * (448 / amax.clamp_min(1e-30))).double()
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))).clamp(-6, 8) - 3)
                x = (torch.round(y / step) * step).clamp(-448, 448) * (amax / 448).double()
            to[b, :, case["past"]:case["past"] + n] = x.to(to.dtype)
        t += n
    return {"K": s["K"].double(), "V": s["V"].double()}
