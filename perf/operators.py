"""The calls that a serving program with a bounded key/value cache makes, as cases to be timed.

* ``attn``       hill_window_attn: one query token per sequence over the visible part of a 16-bit cache (the first
                 ``sinks`` tokens and the newest ``window``), with or without the attention weights added to the
                 running importance;
* ``attn_q4``    hill_window_attn_q4: the same over a cache held in 4 bits;
* ``insert``     hill_cache_insert: new tokens into a 16-bit cache of fixed size; when it is full they take the slots
                 of the least accumulated attention weight;
* ``insert_q4``  hill_cache_insert_q4 into a 4-bit cache, then hill_cache_read_q4: what the cache stands for.

A 4-bit row of 128 channels is 64 bytes (byte i: channel 2i in the low half, 2i + 1 in the high one) with a scale and
a minimum in the cache's 16-bit type; params [B][Hkv][cap32][4] holds (K scale, K min, V scale, V min), cap32 the
capacity rounded up to 32.  Where ``own`` is false every case runs in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random
import zlib

import torch

own = False

D = 128
ALL = 1 << 30   # a window that hides nothing
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
BASE = dict(op="attn", batch=1, heads=32, kv_heads=32, tokens=4096, spare=64, ragged=False, dtype="fp16", sinks=0,
            window=ALL, accum=False, kvh=False, layout="head", new=1, recent=0)


def _case(name, **over):
    return dict(BASE, name=name, **over)


def listed():
    return [
        # the smallest attention: one chat turn of a 32-head model that keeps 4 sinks and the newest 1024 tokens
        _case("attn-1x4k-window1k", sinks=4, window=1024),
        # a batch of long documents of a grouped-query model, 4 sinks and a window of 4096
        _case("attn-8x32k-gqa-window4k", batch=8, kv_heads=8, tokens=32768, ragged=True, dtype="bf16", sinks=4, window=4096),
        # long documents of different lengths, everything visible, the weights accumulated for a later eviction
        _case("attn-4x32k-mha-accum", batch=4, tokens=32768, ragged=True, accum=True),
        # one very long context, eight query heads per KV head, an odd length
        _case("attn-1x128k-gqa8", heads=64, kv_heads=8, tokens=131071, dtype="bf16"),
        # the smallest over 4 bits: one chat turn of a grouped-query model over a whole cache of odd length
        _case("attn_q4-1x4k-gqa", op="attn_q4", kv_heads=8, tokens=4095, dtype="bf16"),
        # long documents of a 32-head model in 4 bits, the weights accumulated
        _case("attn_q4-4x32k-mha-accum", op="attn_q4", batch=4, tokens=32768, ragged=True, accum=True),
        # one very long context of a grouped-query model in 4 bits, importance per KV head
        _case("attn_q4-1x128k-gqa-kvh", op="attn_q4", kv_heads=8, tokens=131072, dtype="bf16", accum=True, kvh=True),
        # the largest: 8 sequences of 64K tokens, 32 KV heads, in 4 bits
        _case("attn_q4-8x64k-mha", op="attn_q4", batch=8, tokens=65536),
        # the smallest insert: one decode step of one sequence into a full cache of 1024 slots
        _case("insert-1x1k-gqa", op="insert", kv_heads=8, tokens=1024, sinks=4, recent=128),
        # one decode step of a batch, every KV head with its own slots
        _case("insert-16x4k-kvh", op="insert", batch=16, kv_heads=8, tokens=4096, dtype="bf16", kvh=True, sinks=4, recent=256),
        # a chunk of a prompt through full caches, ragged chunks, a cache stored token by token
        _case("insert-8x8k-chunk512", op="insert", batch=8, kv_heads=8, tokens=8192, ragged=True, sinks=16, recent=1024,
              new=512, layout="token"),
        # the prompts of a batch into an empty 4-bit cache, and what it then stands for
        _case("insert_q4-4x16k-prompt", op="insert_q4", batch=4, kv_heads=8, tokens=16411, ragged=True, new=16411),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges: 1 to 16 sequences, every head layout, up to 128K tokens (inserts: caches of
    256 to 16K slots), windows from 64 tokens to everything, chunks from one token to the whole cache."""
    while True:
        c = dict(BASE, op=rng.choice(["attn", "attn", "attn_q4", "attn_q4", "insert", "insert_q4"]))
        c["heads"], c["kv_heads"] = rng.choice([(32, 32), (32, 8), (32, 8), (64, 8), (28, 4), (40, 40), (32, 1)])
        c["batch"] = _log(rng, 1, 16)
        c["dtype"] = rng.choice(["fp16", "bf16"])
        c["ragged"] = rng.random() < 0.5
        c["sinks"] = rng.choice([0, 0, 4, 16, 61])
        c["kvh"] = rng.random() < 0.3
        if c["op"].startswith("attn"):
            c["tokens"] = _log(rng, 200, 131072)
            c["accum"] = rng.random() < 0.4
            if rng.random() < 0.5:
                c["window"] = _log(rng, 64, c["tokens"])
            if c["op"] == "attn" and rng.random() < 0.25:
                c["layout"] = "token"
            c["spare"] = rng.choice([0, 1, 64])
            rows = c["batch"] * c["tokens"] * c["kv_heads"]
            if rows > (4 << 20 if c["op"] == "attn" else 16 << 20) or c["batch"] * c["tokens"] * c["heads"] > 64 << 20:
                continue
        else:
            c["tokens"] = _log(rng, 256, 16384)
            c["new"] = rng.choice([1, 1, _log(rng, 2, c["tokens"] // 2)]) if c["op"] == "insert" else _log(rng, 1, c["tokens"])
            c["recent"] = min(rng.choice([0, 32, 128]), c["tokens"] // 8)
            if max(c["new"], c["recent"]) > c["tokens"] - c["sinks"] or c["batch"] * c["tokens"] * c["kv_heads"] > 1 << 20:
                continue
            if c["op"] == "insert" and rng.random() < 0.25:
                c["layout"] = "token"
        return c


# ---------------------------------------------------------------- inputs
def _lengths(case):
    """Cached tokens of every sequence; ragged: the longest, and others between a half of it and it."""
    n, B = case["tokens"], case["batch"]
    if not case["ragged"]:
        return [n] * B
    r = random.Random(zlib.crc32(repr(sorted((k, v) for k, v in case.items() if k != "name")).encode()))
    return [n] + [r.randint(max(1, n // 2), n) for _ in range(B - 1)]


def _generator(seed, what):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((int(seed), what)).encode()))


def _channels(g, Hkv):
    """Per KV head and channel: a spread and an offset; a few channels are far larger, as keys have them."""
    spread = 0.5 + torch.rand(Hkv, 1, D, generator=g, device="cuda")
    offset = torch.randn(Hkv, 1, D, generator=g, device="cuda")
    loud = torch.rand(Hkv, 1, D, generator=g, device="cuda") < 0.03
    return spread * (1 + 2 * loud), offset * (0.2 + 3 * loud)


def _rows(g, Hkv, n, spread, offset):
    return torch.randn(Hkv, n, D, generator=g, device="cuda") * spread + offset


def _keys(g, Hkv, n, ch, u):
    """Keys of which one in 64 points along the query direction u: the heavy hitters of real attention."""
    k = _rows(g, Hkv, n, *ch)
    heavy = (torch.rand(1, n, 1, generator=g, device="cuda") < 1 / 64) * torch.rand(1, n, 1, generator=g, device="cuda")
    return k + heavy * 0.35 * u[:, None, :]


def _encode(x, dtype):
    """4-bit rows of x (last axis 128): (bytes, scales, minima)."""
    mn, mx = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((mx - mn) / 15).to(dtype)
    s = scale.float()
    code = torch.where(s > 0, ((x - mn) / s).round().clamp(0, 15), 0).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale[..., 0], mn[..., 0].to(dtype)


def _q4_attn(case):
    return case["op"] == "attn_q4"


def _token_major(x):
    return x.transpose(1, 2).contiguous().transpose(1, 2)


def prepare(case, seed):
    B, H, Hkv, dt = case["batch"], case["heads"], case["kv_heads"], DTYPES[case["dtype"]]
    attn, q4 = case["op"].startswith("attn"), case["op"].endswith("q4")
    cap = case["tokens"] + (case["spare"] if attn else 0)
    cap32 = (cap + 31) // 32 * 32
    rows = (B, Hkv) if case["kvh"] else (B,)
    g = _generator(seed, "inputs")
    ck, cv = _channels(g, Hkv), _channels(g, Hkv)
    u = torch.randn(Hkv, D, generator=g, device="cuda")
    q = (u.repeat_interleave(H // Hkv, 0) + 0.25 * torch.randn(B, H, D, generator=g, device="cuda")).to(dt)
    s = {"case": case, "q": q}
    lengths = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    if q4:
        s["k4"], s["v4"] = (torch.zeros(B, Hkv, cap, D // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
        s["params"] = torch.zeros(B, Hkv, cap32, 4, dtype=dt, device="cuda")
    else:
        s["K"], s["V"] = (torch.empty(B, Hkv, cap, D, dtype=dt, device="cuda") for _ in range(2))
    for b in range(B):   # the cache as earlier steps left it
        if case["op"] == "insert_q4":
            break
        k, v = _keys(g, Hkv, cap, ck, u).to(dt), _rows(g, Hkv, cap, *cv).to(dt)
        if q4:
            for i, (x, codes) in enumerate(((k, s["k4"]), (v, s["v4"]))):
                codes[b], s["params"][b, :, :cap, 2 * i], s["params"][b, :, :cap, 2 * i + 1] = _encode(x.float(), dt)
        else:
            s["K"][b], s["V"][b] = k, v
    if case["layout"] == "token":
        s["K"], s["V"] = _token_major(s["K"]), _token_major(s["V"])
    if attn:
        s["lens"] = lengths[:, None].expand(rows).contiguous() if case["kvh"] else lengths
        s["out"] = torch.zeros(B, H, D, device="cuda")
        s["accum"] = torch.rand(*rows, cap, generator=g, device="cuda") * (H / cap) if case["accum"] else None
    else:
        T = case["new"]
        fresh = case["op"] == "insert_q4"   # an empty cache; else a full one, some way into the sequence
        s["k_new"] = torch.stack([_keys(g, Hkv, T, ck, u).to(dt) for _ in range(B)])
        s["v_new"] = torch.stack([_rows(g, Hkv, T, *cv).to(dt) for _ in range(B)])
        s["n_new"] = (T - (case["tokens"] - lengths) * T // max(1, case["tokens"])).to(torch.int32) if case["ragged"] else None
        seen = torch.zeros(*rows, dtype=torch.int32, device="cuda") if fresh else torch.full(rows, 3 * cap, dtype=torch.int32, device="cuda")
        s["seen"] = seen
        # what a full cache holds: the sinks, the newest half, and a random set of the positions between
        keep = torch.rand(*rows, 3 * cap, generator=g, device="cuda")
        keep[..., :case["sinks"]] = 2
        keep[..., 3 * cap - cap // 2:] = 2
        pos = keep.topk(cap, -1).indices
        order = torch.rand(*rows, cap, generator=g, device="cuda").argsort(-1)   # slots are reused in any order
        s["pos"] = pos.gather(-1, order).to(torch.int32) if not fresh else torch.zeros(*rows, cap, dtype=torch.int32, device="cuda")
        # accumulated weights fall off like a power of the rank
        s["accum"] = torch.rand(*rows, cap, generator=g, device="cuda").pow(6) * (0 if fresh else 30)
        s["slots"] = torch.full((*rows, T), -1, dtype=torch.int32, device="cuda")
        if q4:
            s["K"], s["V"] = (torch.zeros(B, Hkv, cap, D, dtype=dt, device="cuda") for _ in range(2))
            s["zero"], s["full"] = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), cap, dtype=torch.int32, device="cuda")
    if own:
        from paper_2602_18750_gb300 import hill

        hill.load()
        s["desc"] = hill.make_desc_q4(q, s["k4"]) if _q4_attn(case) else hill.make_desc(q, s["K"], s["V"])
        if attn:
            s["ws"] = hill.alloc_window_workspace(s["desc"], case["accum"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return _plain_attn(s, case) if case["op"].startswith("attn") else _plain_insert(s, case)


def _run_own(s, case):
    from paper_2602_18750_gb300 import hill

    op = case["op"]
    if op == "attn":
        hill.hill_window_attn(s["desc"], s["q"], s["K"], s["V"], s["lens"], case["sinks"], case["window"], s["out"],
                              accum=s["accum"], kvh=case["kvh"], ws=s["ws"])
    elif op == "attn_q4":
        hill.hill_window_attn_q4(s["desc"], s["q"], s["k4"], s["v4"], s["params"], s["lens"], case["sinks"],
                                 case["window"], s["out"], accum=s["accum"], kvh=case["kvh"], ws=s["ws"])
    elif op == "insert":
        hill.hill_cache_insert(s["desc"], s["k_new"], s["v_new"], s["K"], s["V"], s["seen"], s["pos"], s["accum"],
                               case["sinks"], case["recent"], s["slots"], n_new=s["n_new"], kvh=case["kvh"])
    else:
        hill.hill_cache_insert_q4(s["desc"], s["k_new"], s["v_new"], s["k4"], s["v4"], s["params"], s["seen"], s["pos"],
                                  s["accum"], case["sinks"], case["recent"], s["slots"], n_new=s["n_new"], kvh=case["kvh"])
        hill.hill_cache_read_q4(s["desc"], s["k4"], s["v4"], s["params"], s["zero"], s["full"], case["tokens"], s["K"], s["V"])
    return _outputs(s, case)


def _outputs(s, case):
    if case["op"].startswith("attn"):
        return {"out": s["out"], "accum": s["accum"]} if case["accum"] else {"out": s["out"]}
    return {n: s[n] for n in ("K", "V", "pos", "accum", "seen", "slots")}


def _decode(codes, scale, mn):
    """The values of 4-bit rows, in the type of scale and mn."""
    x = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return mn[..., None] + scale[..., None] * x


def _take(x, cols):
    """Rows cols [..][n] of x [B][Hkv][cap][w]."""
    return x.gather(2, cols[..., None].expand(*cols.shape, x.shape[-1]))


def _plain_attn(s, case):
    B, H, Hkv, q4 = case["batch"], case["heads"], case["kv_heads"], _q4_attn(case)
    cap = (s["k4"] if q4 else s["K"]).shape[2]
    n = s["lens"][..., None].clamp(0, cap).long()   # [rows][1]
    sinks, window = case["sinks"], case["window"]
    if sinks + window >= cap:   # every slot is looked at
        cols = torch.arange(cap, device="cuda").expand(*n.shape[:-1], cap)
        valid = (cols < n) & ((cols < sinks) | (cols >= n - window))
        pick = lambda x: x[:, :, :cap]
    else:
        first, rest = torch.arange(sinks, device="cuda").expand(*n.shape[:-1], sinks), n - window + torch.arange(window, device="cuda")
        valid = torch.cat(((first < n) & (first < n - window), rest >= 0), -1)
        cols = torch.cat((first, rest), -1).clamp(0, cap - 1)
        by_head = (cols if case["kvh"] else cols[:, None]).expand(B, Hkv, cols.shape[-1])
        pick = lambda x: _take(x, by_head)
    if q4:
        pr = pick(s["params"]).float()
        k = _decode(pick(s["k4"]), pr[..., 0], pr[..., 1])
        v = _decode(pick(s["v4"]), pr[..., 2], pr[..., 3])
    else:
        k, v = pick(s["K"]).float(), pick(s["V"]).float()
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


def _plain_insert(s, case):
    B, Hkv, T, cap, kvh = case["batch"], case["kv_heads"], case["new"], case["tokens"], case["kvh"]
    seen = s["seen"][..., None].long()   # [rows][1]
    t = torch.full((B,), T, device="cuda") if s["n_new"] is None else s["n_new"].long().clamp(0, T)
    t = (t[:, None, None] if kvh else t[:, None]).expand(seen.shape)
    slot = torch.arange(cap, device="cuda").expand(*seen.shape[:-1], cap)
    held = seen.clamp(max=cap)
    free = torch.minimum(t, cap - held)
    # the last ones in the order (weight descending, slot ascending) go first
    can = (slot < held) & (s["pos"] >= case["sinks"]) & (s["pos"] < seen + t - case["recent"])
    order = torch.where(can, s["accum"], math.inf).flip(-1).sort(stable=True, dim=-1).indices
    rank = torch.empty_like(order).scatter_(-1, order, slot).flip(-1)
    victim = rank < t - free
    # token i goes to slot held + i, or to the victims in ascending order
    token = torch.where(victim, free + victim.cumsum(-1) - 1, torch.where((slot >= held) & (slot < held + free), slot - held, T))
    to = torch.full((*seen.shape[:-1], T + 1), -1, device="cuda").scatter_(-1, token, slot)[..., :T]
    s["slots"].copy_(to)
    put = token < T
    s["pos"].copy_(torch.where(put, seen + token, s["pos"]))
    s["accum"].copy_(torch.where(put, 0.0, s["accum"]))
    s["seen"].add_(t[..., 0].to(torch.int32))
    # places past a sequence's new tokens repeat its last one; with none, slot 0 keeps what it has
    i = torch.minimum(torch.arange(T, device="cuda"), t - 1).clamp_min(0)
    i, at, some = ((x if kvh else x[:, None]).expand(B, Hkv, x.shape[-1]) for x in (i, to.gather(-1, i).clamp_min(0), t > 0))
    scatter = lambda x, new: x.scatter_(2, at[..., None].expand(B, Hkv, T, x.shape[-1]), torch.where(some[..., None], _take(new, i), x[:, :, :1]))
    if case["op"] == "insert":
        scatter(s["K"], s["k_new"])
        scatter(s["V"], s["v_new"])
    else:
        k, ks, km = _encode(s["k_new"].float(), s["params"].dtype)
        v, vs, vm = _encode(s["v_new"].float(), s["params"].dtype)
        scatter(s["k4"], k)
        scatter(s["v4"], v)
        scatter(s["params"], torch.stack((ks, km, vs, vm), -1))
        p = s["params"][:, :, :cap].float()
        s["K"].copy_(_decode(s["k4"], p[..., 0], p[..., 1]))
        s["V"].copy_(_decode(s["v4"], p[..., 2], p[..., 3]))
    return _outputs(s, case)


def work(case):
    B, H, Hkv, T = case["batch"], case["heads"], case["kv_heads"], case["new"]
    rows = B * (Hkv if case["kvh"] else 1)
    if case["op"].startswith("attn"):
        seen = sum(min(n, min(case["sinks"], max(0, n - case["window"])) + case["window"]) for n in _lengths(case))
        row = 2 * (D // 2 + 4 if _q4_attn(case) else 2 * D)
        accum = 8 * seen * (Hkv if case["kvh"] else 1) if case["accum"] else 0
        return {"bytes": seen * Hkv * row + accum + 6 * B * H * D, "flops": 4 * H * D * seen}
    new = sum(T - (case["tokens"] - n) * T // max(1, case["tokens"]) for n in _lengths(case)) if case["ragged"] else B * T
    state = 16 * new * rows // B   # slot, position and weight written, one of them counted
    if case["op"] == "insert":
        return {"bytes": new * Hkv * 2 * 4 * D + state + 8 * rows * case["tokens"], "flops": rows * case["tokens"]}
    cache = B * Hkv * case["tokens"]   # read back whole
    return {"bytes": new * Hkv * 2 * (2 * D + D // 2 + 4) + state + cache * 2 * (2 * D + D // 2 + 4), "flops": 8 * D * new * Hkv}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attn(s, case) if case["op"].startswith("attn") else _exact_insert(s, case)


def _values64(codes, scale, mn):
    low, high = (codes % 16).double(), torch.div(codes, 16, rounding_mode="floor").double()
    return torch.stack((low, high), -1).reshape(*codes.shape[:-1], D) * scale.double()[..., None] + mn.double()[..., None]


def _exact_attn(s, case):
    H, Hkv = case["heads"], case["kv_heads"]
    out = torch.zeros(case["batch"], H, D, dtype=torch.float64, device="cuda")
    accum = s["accum"].double() if case["accum"] else None
    for b, n in enumerate(_lengths(case)):
        shown = [j for j in range(min(case["sinks"], max(0, n - case["window"])))]
        shown = torch.tensor(shown, dtype=torch.long, device="cuda")
        shown = torch.cat((shown, torch.arange(max(0, n - case["window"]), n, device="cuda")))
        for g in range(Hkv):
            if _q4_attn(case):
                p4 = s["params"][b, g, shown]
                k, v = _values64(s["k4"][b, g, shown], p4[:, 0], p4[:, 1]), _values64(s["v4"][b, g, shown], p4[:, 2], p4[:, 3])
            else:
                k, v = s["K"][b, g, shown].double(), s["V"][b, g, shown].double()
            h = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
            p = torch.softmax(s["q"][b, h].double() @ k.T * D ** -0.5, -1)
            out[b, h] = p @ v
            if accum is not None:
                (accum[b, g] if case["kvh"] else accum[b])[shown] += p.sum(0)
    return {"out": out, "accum": accum} if case["accum"] else {"out": out}


def _exact_insert(s, case):
    cap, T, Hkv = case["tokens"], case["new"], case["kv_heads"]
    K, V, slots = s["K"].double(), s["V"].double(), torch.full_like(s["slots"], -1)
    pos, accum, seen = s["pos"].clone(), s["accum"].double(), s["seen"].clone()
    for b in range(case["batch"]):
        t = T if s["n_new"] is None else int(s["n_new"][b])
        if case["op"] == "insert":
            fresh = [s["k_new"][b, :, :t].double(), s["v_new"][b, :, :t].double()]
        else:
            fresh = []
            for x in (s["k_new"], s["v_new"]):
                x = x[b, :, :t].double()
                lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
                step = ((hi - lo) / 15).to(s["params"].dtype).double()
                fresh.append(lo + step * torch.where(step > 0, (x - lo) / step, 0.0).round().clamp(0, 15))
        for g in range(Hkv if case["kvh"] else 1):
            at = (b, g) if case["kvh"] else (b,)
            before, held = int(seen[at]), min(int(seen[at]), cap)
            to = list(range(held, min(cap, held + t)))
            if len(to) < t:
                w, p = accum[at].tolist(), pos[at].tolist()
                ranked = sorted((j for j in range(held) if case["sinks"] <= p[j] < before + t - case["recent"]), key=lambda j: (w[j], -j))
                to += sorted(ranked[:t - len(to)])
            to = torch.tensor(to, dtype=torch.long, device="cuda")
            slots[at][:t] = to.int()
            pos[at][to] = before + torch.arange(t, dtype=torch.int32, device="cuda")
            accum[at][to] = 0
            seen[at] = before + t
            heads = slice(g, g + 1) if case["kvh"] else slice(0, Hkv)
            for cache, x in ((K, fresh[0]), (V, fresh[1])):
                cache[b, heads, to] = x[heads]
    return {"K": K, "V": V, "pos": pos, "accum": accum, "seen": seen, "slots": slots}
