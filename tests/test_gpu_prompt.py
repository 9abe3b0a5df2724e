"""Attention and importance of packed prompts against plain float64 forms (tests/paged_util.py)."""
import numpy as np
import pytest
import torch

from paged_util import ALL, HALF, importance, prompt

pytestmark = pytest.mark.gpu

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def H():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2602_18750_gb300 import build, hill
    build.build()
    hill.load()
    return hill


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts(lens, first=0):
    return [first + sum(lens[:i]) for i in range(len(lens) + 1)]


def f64(t):
    return t.double().cpu().numpy()


class Case:
    """Sequences of (new, earlier) tokens, `spare` rows of no sequence before the first and behind the last."""

    def __init__(self, H, seqs, Hq, Hkv, dtype="bf16", seed=0, spare=0, layout="row", scale=1.0):
        self.H, self.dt, self.seqs = H, DT[dtype], seqs
        self.q_start = starts([n for n, _ in seqs], spare)
        self.k_start = starts([max(0, n + past) for n, past in seqs], spare)
        T, S, g = self.q_start[-1] + spare, self.k_start[-1] + spare, gen(seed)
        loud = 1 + 5 * (torch.rand(1, Hkv, 128, generator=g, device="cuda") < 0.05)
        make = lambda n, h, by: self.lay(((torch.randn(n, h, 128, generator=g, device="cuda") + 0.3) * by * scale).to(self.dt), layout)
        self.q, self.k, self.v = make(T, Hq, 0.7), make(S, Hkv, loud), make(S, Hkv, loud)
        self.desc = H.make_packed(self.q, self.k, self.v, len(seqs))
        self.out = torch.full((T, Hq, 128), 7.0, dtype=self.dt, device="cuda")
        self.lse = torch.full((T, Hq), 7.0, device="cuda")
        self.qs, self.ks = ints(self.q_start), ints(self.k_start)

    @staticmethod
    def lay(x, layout):
        if layout == "head":      # [heads][rows][d] underneath
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        if layout == "wide":      # a part of a wider row
            w = torch.full((x.shape[0], x.shape[1] + 3, 136), float("nan"), dtype=x.dtype, device="cuda")
            w[:, 1:-2, :128] = x
            return w[:, 1:-2, :128]
        return x

    def attend(self, sinks, window, lse=True, stream=None):
        self.H.hill_prompt_attn(self.desc, self.q, self.k, self.v, self.qs, self.ks, sinks, window, self.out,
                                lse=self.lse if lse else None, stream=stream)
        self.H.hill_sync_status(stream)
        return f64(self.out), f64(self.lse)

    def reference(self, sinks, window):
        return prompt(f64(self.q), f64(self.k), f64(self.v), self.q_start, self.k_start, sinks, window, HALF[self.dt])

    def verify(self, sinks, window):
        out, lse = self.attend(sinks, window)
        ref, rl, bound, lbound = self.reference(sinks, window)
        none = np.isnan(rl)                         # rows of no sequence: as they were
        assert np.all(out[none] == 7) and np.all(lse[none] == 7)
        check(out[~none], ref[~none], bound[~none])
        empty = ~none & np.isneginf(rl)
        assert np.all(np.isneginf(lse[empty])) and np.all(out[empty] == 0)
        check(lse[~none & ~empty], rl[~none & ~empty], lbound[~none & ~empty])
        return out, lse


def check(got, ref, bound):
    assert not np.isnan(got).any()
    err = np.abs(got - ref)
    bad = np.argwhere(err > bound + 1e-30)
    assert not len(bad), (f"{len(bad)} of {err.size} out of bounds; first {bad[0]}: {got[tuple(bad[0])]} for "
                          f"{ref[tuple(bad[0])]}, bound {bound[tuple(bad[0])]}")


SEQS = [(131, 0), (0, 40), (1, 0), (300, 17), (5, 400), (128, 128), (64, -20), (257, 0)]
HEADS = [(4, 4), (8, 2), (7, 1), (12, 1), (32, 1), (10, 2), (3, 3)]
RULES = [(0, ALL), (4, 64), (0, 0), (3, 0), (61, 100), (200, 1), (0, 33), (130, 129)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}x{h[1]}")
def test_attention(H, heads, dtype):
    c = Case(H, SEQS, *heads, dtype, seed=heads[0], spare=3)
    for sinks, window in RULES:
        out, _ = c.verify(sinks, window)
        c.out.fill_(7)
        c.attend(sinks, window, lse=False)   # without the statistics: the same output
        assert np.array_equal(f64(c.out), out)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513])
@pytest.mark.parametrize("heads", [(1, 1), (4, 1), (7, 1)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_lengths(H, n, heads):
    for past in (0, 1, 127, 128, 700):
        Case(H, [(n, past)], *heads, seed=n).verify(0, ALL)


def test_long(H):
    """More tiles than SMs, long rows, chunks behind long contexts."""
    Case(H, [(1500, 0), (700, 2500), (1, 3000), (40, 2990)], 8, 2, seed=1).verify(0, ALL)
    Case(H, [(2600, 0)], 2, 2, "fp16", seed=2).verify(4, 500)
    Case(H, [(300, 3300)], 6, 2, seed=3).verify(150, 700)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,seqs", [((4, 1), [(1, 5000)]), ((8, 2), [(40, 4000), (3, 9000)]), ((8, 8), [(9, 2500)]),
                                        ((16, 2), [(5, 9000), (7, 20), (0, 30), (2, -2)]), ((14, 2), [(90, 3000)])])
def test_few_rows_behind_many_keys(H, heads, seqs, dtype):
    """Clusters share a unit's key tiles; parts without any, of short sequences and windows, among them."""
    c = Case(H, seqs, *heads, dtype, seed=sum(heads), spare=2)
    for sinks, window in [(0, ALL), (4, 1000), (300, 200), (0, 0), (0, 4000)]:
        out, lse = c.verify(sinks, window)
        again, lse2 = c.attend(sinks, window)
        assert np.array_equal(out, again) and np.array_equal(lse, lse2)
    want, wl = c.attend(0, 2000)
    b = max(range(len(seqs)), key=lambda i: seqs[i][0] + seqs[i][1])
    last = c.q_start[b + 1] - 1      # the newest query sees key 100 under no window of 2000
    c.v[c.k_start[b] + 100] = float("nan")
    c.k[c.k_start[b] + 100] = float("nan")
    out, lse = c.attend(0, 2000)
    assert np.array_equal(out, want) and np.array_equal(lse, wl)
    out, _ = c.attend(0, ALL)
    assert np.isnan(out[last]).all()


@pytest.mark.parametrize("B", [31, 32, 33, 70])
def test_many_sequences(H, B):
    """Up to a warp's lanes of sequences, and more; lengths all over, empty ones among them."""
    r = np.random.RandomState(B)
    seqs = [(int(n), int(p)) for n, p in zip(r.choice([0, 1, 2, 30, 64, 65, 150], B), r.choice([0, 0, 5, 140], B))]
    for heads in ((4, 4), (8, 2)):
        c = Case(H, seqs, *heads, seed=B, spare=1)
        c.verify(0, ALL)
        c.verify(3, 50)
    verify_importance(H, c, 0, ALL, 40, True)


def test_groups_past_a_tile(H):
    """More query heads to a KV head than a tile has rows."""
    Case(H, [(3, 20), (130, 0)], 130, 1, seed=4).verify(0, ALL)
    Case(H, [(2, 9)], 300, 2, "fp16", seed=5).verify(2, 5)


@pytest.mark.parametrize("layout", ["head", "wide"])
def test_strides(H, layout):
    Case(H, [(200, 30), (77, 0)], 8, 2, seed=6, layout=layout).verify(0, ALL)
    c = Case(H, [(1, 0)], 1, 1, seed=6, layout=layout)
    c.verify(0, ALL)


def test_expanded_rows_are_refused(H):
    c = Case(H, [(20, 10)], 4, 2, seed=6)
    for q, k in ((c.q[:1].expand(20, -1, -1), c.k), (c.q, c.k[:, :1].expand(-1, 2, -1))):
        desc = H.make_packed(q, k, c.v, 1)
        with pytest.raises(H.HillError) as e:
            H.hill_prompt_attn(desc, q, k, c.v, c.qs, c.ks, 0, ALL, c.out, lse=c.lse)
        assert e.value.status == H.HILL_ERR_UNSUPPORTED


def test_large_logits(H):
    """Logits of hundreds, rising and falling: the running maximum moves often."""
    for dtype in DT:
        c = Case(H, [(300, 500)], 4, 2, dtype, seed=7, scale=2.0)
        order = torch.linspace(0.1, 4, c.k.shape[0], device="cuda")[:, None, None]
        for by in (order, order.flip(0)):
            kept = c.k.clone()
            c.k.copy_((c.k.float() * by).to(c.dt))
            c.verify(0, ALL)
            c.verify(5, 200)
            c.k.copy_(kept)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), "lowest"])
def test_hidden_places_do_not_matter(H, bad):
    """Keys and values that a query does not see hold anything: of other sequences, later ones, out of the window."""
    for dtype, heads in (("bf16", (4, 4)), ("fp16", (8, 1))):
        c = Case(H, [(150, 30), (90, 0), (60, 200)], *heads, dtype, seed=8, spare=5)
        value = torch.finfo(c.dt).min if bad == "lowest" else bad
        for sinks, window in [(0, ALL), (3, 40)]:
            want, wl = c.attend(sinks, window)
            for where in ([0, 1, 2], [c.k_start[1] + 45], [c.k_start[1] - 1], list(range(c.k_start[3], c.k_start[3] + 5)),
                          [c.k_start[2] + 130, c.k_start[2] + 257]):
                kept = c.k.clone(), c.v.clone()
                c.k[where] = value
                c.v[where] = value
                out, lse = c.attend(sinks, window)
                c.k.copy_(kept[0])
                c.v.copy_(kept[1])
                seen = np.zeros(c.q.shape[0], bool)
                for b, (n, past) in enumerate(c.seqs):
                    for w in where:
                        j = w - c.k_start[b]
                        if 0 <= j < n + past:
                            pos = np.arange(n) + past
                            seen[c.q_start[b]:c.q_start[b + 1]] |= (j <= pos) & ((j < sinks) | (j > pos - window))
                assert np.array_equal(out[~seen], want[~seen]) and np.array_equal(lse[~seen], wl[~seen])
                if bad != "lowest":
                    assert not np.isfinite(out[seen]).any()


def test_seen_values_that_are_not_finite(H):
    """A value of infinity shows in the channels that have it, in those rows that see it."""
    for dtype in DT:
        c = Case(H, [(200, 20)], 4, 2, dtype, seed=9)
        want, _ = c.attend(0, ALL)
        c.v[60, 0, 5] = float("inf")
        c.v[61, 1, 7] = float("nan")
        out, lse = c.attend(0, ALL)
        pos = np.arange(200) + 20
        assert np.all(out[pos >= 60][:, :2, 5] == np.inf)
        assert np.isnan(out[pos >= 61][:, 2:, 7]).all()
        mask = np.ones_like(out, bool)
        mask[pos >= 60, :2, 5] = False
        mask[pos >= 61, 2:, 7] = False
        assert np.isfinite(out[mask]).all()
        ref, _, bound, _ = c.reference(0, ALL)
        with np.errstate(invalid="ignore"):
            clean = prompt(f64(c.q), f64(c.k), np.nan_to_num(f64(c.v), posinf=0, nan=0), c.q_start, c.k_start, 0, ALL, HALF[c.dt])
        check(out[mask], clean[0][mask], clean[2][mask])


def test_queries_that_are_not_finite(H):
    c = Case(H, [(140, 0)], 4, 2, seed=10)
    want, wl = c.attend(0, ALL)
    c.q[77, 1] = float("nan")
    out, lse = c.attend(0, ALL)
    rest = np.ones(out.shape[:2], bool)
    rest[77, 1] = False
    assert np.isnan(out[77, 1]).all() and np.isnan(lse[77, 1])
    assert np.array_equal(out[rest], want[rest]) and np.array_equal(lse[rest], wl[rest])


def test_no_keys_and_no_queries(H):
    c = Case(H, [(5, -5), (3, -3)], 4, 2, seed=11)
    out, lse = c.attend(0, ALL)
    assert np.all(out == 0) and np.all(np.isneginf(lse))
    c = Case(H, [(0, 5)], 4, 2, seed=11)
    c.attend(0, ALL)
    H.hill_prompt_attn(H.make_packed(c.q, c.k, c.v, 0), c.q, c.k, c.v, ints([0]), ints([0]), 0, ALL, c.out)


def test_tiles_that_see_nothing_beside_ones_that_do(H):
    """Queries before the first key, in one tile of a unit and not in the other, many units at once."""
    for heads in ((32, 1), (64, 2), (4, 4)):
        c = Case(H, [(40, -20)] * 24 + [(300, -130)], *heads, seed=33)
        for _ in range(5):
            c.out.fill_(7)
            c.verify(0, ALL)


def test_bad_offsets_are_an_error(H):
    c = Case(H, [(40, 0), (20, 0)], 4, 2, seed=12)
    for qs, ks in (([0, 40, 70], [0, 40, 60]), ([0, 40, 60], [0, 40, 1 << 29]), ([0, 50, 40], [0, 40, 60]), ([-3, 40, 60], [0, 40, 60])):
        c.qs, c.ks = ints(qs), ints(ks)
        with pytest.raises(H.HillError) as e:
            c.attend(0, ALL)
        assert e.value.status == H.HILL_ERR_DEVICE
    c.qs, c.ks = ints(c.q_start), ints(c.k_start)
    c.verify(0, ALL)


def test_another_stream_and_a_graph(H):
    c = Case(H, [(200, 50), (31, 0)], 8, 2, seed=13)
    want, wl = c.attend(0, ALL)
    accum = torch.zeros(2, 300, device="cuda")
    ws = H.alloc_prompt_workspace(c.desc)
    H.hill_prompt_importance(c.desc, c.q, c.k, c.lse, c.qs, c.ks, 0, ALL, ALL, accum, ws=ws)
    H.hill_sync_status()
    once = accum.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.out.fill_(0)
        out, lse = c.attend(0, ALL)
        assert np.array_equal(out, want) and np.array_equal(lse, wl)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            H.hill_prompt_attn(c.desc, c.q, c.k, c.v, c.qs, c.ks, 0, ALL, c.out, lse=c.lse)
            H.hill_prompt_importance(c.desc, c.q, c.k, c.lse, c.qs, c.ks, 0, ALL, ALL, accum, ws=ws)
        c.out.fill_(0)
        c.lse.fill_(0)
        accum.zero_()
        graph.replay()
        side.synchronize()
        assert np.array_equal(f64(c.out), want) and torch.equal(accum, once)
        c.q.copy_(c.q.flip(0))    # new contents, the same graph
        graph.replay()
        side.synchronize()
        got = f64(c.out)
        assert np.array_equal(got, c.attend(0, ALL)[0]) and not np.array_equal(got, want)
        c.qs.copy_(ints([0, 17, 231]))       # other lengths of the same rows
        c.ks.copy_(ints([0, 100, 281]))
        accum.zero_()
        graph.replay()
        side.synchronize()
        ref, rl, bound, lbound = prompt(f64(c.q), f64(c.k), f64(c.v), [0, 17, 231], [0, 100, 281], 0, ALL, HALF[c.dt])
        check(f64(c.out), ref, bound)
        seen = [17, 231 - 17 - max(0, 231 - 17 - 181)]     # queries that see a key give 1 per head
        np.testing.assert_allclose(f64(accum).sum(1), [8 * n for n in seen], rtol=1e-4)


# ---------------------------------------------------------------- importance
def run_importance(H, c, sinks, window, newest, kvh, cap, lse=None):
    B, Hkv = len(c.seqs), c.k.shape[1]
    start = torch.rand(B, *([Hkv] if kvh else []), cap, device="cuda", generator=gen(3))
    accum = start.clone()
    lse = c.lse if lse is None else lse
    H.hill_prompt_importance(c.desc, c.q, c.k, lse, c.qs, c.ks, sinks, window, newest, accum, kvh=kvh,
                             ws=H.alloc_prompt_workspace(c.desc))
    return start, accum, lse


def verify_importance(H, c, sinks, window, newest, kvh):
    cap = max(max(0, n + past) for n, past in c.seqs) + 3
    c.attend(sinks, window)
    start, accum, lse = run_importance(H, c, sinks, window, newest, kvh, cap)
    H.hill_sync_status()
    w, wb = importance(f64(c.q), f64(c.k), f64(lse), c.q_start, c.k_start, sinks, window, newest, cap, kvh)
    old = f64(start)
    check(f64(accum), old + w, wb + 2.0 ** -23 * (old + w))
    assert torch.equal(accum.cpu()[torch.from_numpy(w == 0)], start.cpu()[torch.from_numpy(w == 0)])
    again = start.clone()
    H.hill_prompt_importance(c.desc, c.q, c.k, lse, c.qs, c.ks, sinks, window, newest, again, kvh=kvh,
                             ws=H.alloc_prompt_workspace(c.desc))
    assert torch.equal(again, accum)   # the same order every time


@pytest.mark.parametrize("kvh", [False, True], ids=["seq", "kvh"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}x{h[1]}")
def test_importance(H, heads, dtype, kvh):
    c = Case(H, SEQS, *heads, dtype, seed=20 + heads[0], spare=3)
    for sinks, window in RULES:
        for newest in (ALL, 16, 1, 0):
            verify_importance(H, c, sinks, window, newest, kvh)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 64, 127, 128, 129, 257, 600])
def test_importance_lengths(H, n):
    for past in (0, 1, 127, 700):
        for heads in ((1, 1), (4, 1), (7, 1)):
            verify_importance(H, Case(H, [(n, past)], *heads, seed=n), 0, ALL, ALL, False)


def test_importance_long(H):
    verify_importance(H, Case(H, [(1500, 0), (700, 1500), (1, 2000)], 8, 2, seed=1), 0, ALL, ALL, True)
    verify_importance(H, Case(H, [(1600, 0)], 2, 2, "fp16", seed=2), 4, 500, 900, False)
    verify_importance(H, Case(H, [(3, 20), (130, 0)], 130, 1, seed=4), 0, ALL, ALL, False)
    for layout in ("head", "wide"):
        verify_importance(H, Case(H, [(200, 30), (77, 0)], 8, 2, seed=6, layout=layout), 0, ALL, ALL, True)


def test_importance_hidden_places(H):
    """What a counted query does not see, and queries that do not count, may hold anything."""
    for bad in (float("nan"), float("inf")):
        c = Case(H, [(150, 30), (90, 0)], 4, 2, seed=21, spare=5)
        c.attend(0, ALL)
        start, want, lse = run_importance(H, c, 0, ALL, 20, False, 200)
        lse = lse.clone()
        first = c.q_start[0], c.q_start[2]
        c.q[:first[0]] = bad
        c.q[first[1]:] = bad
        c.k[:5] = bad
        c.k[c.k_start[2]:] = bad
        c.q[c.q_start[0] + 10], c.q[c.q_start[1] + 3] = bad, bad     # not among the newest 20
        lse[c.q_start[0] + 10], lse[c.q_start[1] + 3] = bad, bad
        lse[:first[0]], lse[first[1]:] = bad, bad
        _, got, _ = run_importance(H, c, 0, ALL, 20, False, 200, lse)
        H.hill_sync_status()
        assert torch.equal(got, want)
        c.k[c.k_start[1] + 89] = bad      # seen by the last query of the second sequence alone
        _, got, _ = run_importance(H, c, 0, ALL, 20, False, 200, lse)
        hit = got != want
        assert hit[1, 89] and hit.sum() == 1


def test_importance_bad_offsets_are_an_error(H):
    """Offsets that descend name more keys than there are: recorded, and nothing outside accum is written."""
    B = 40
    c = Case(H, [(8, 100)] * B, 4, 2, seed=23)
    n = 108 * B
    c.attend(0, ALL)
    ws = H.alloc_prompt_workspace(c.desc)
    guarded = torch.full((3, B, n + 50), 5.0, device="cuda")
    for ks in ([0, n] * (B // 2) + [0], list(range(B, -1, -1)), [0] * B + [1 << 30], [-7] + [108 * b for b in range(1, B + 1)]):
        H.hill_prompt_importance(c.desc, c.q, c.k, c.lse, c.qs, ints(ks), 0, ALL, ALL, guarded[1], ws=ws)
        with pytest.raises(H.HillError) as e:
            H.hill_sync_status()
        assert e.value.status == H.HILL_ERR_DEVICE
        assert torch.all(guarded[0] == 5) and torch.all(guarded[2] == 5)
    verify_importance(H, c, 0, ALL, ALL, False)


def test_importance_past_the_capacity(H):
    c = Case(H, [(100, 0), (40, 0)], 4, 2, seed=22)
    c.attend(0, ALL)
    _, want, _ = run_importance(H, c, 0, ALL, ALL, False, 100)
    start, got, _ = run_importance(H, c, 0, ALL, ALL, False, 60)
    with pytest.raises(H.HillError) as e:
        H.hill_sync_status()
    assert e.value.status == H.HILL_ERR_DEVICE
    base = torch.rand(2, 100, device="cuda", generator=gen(3))
    torch.testing.assert_close(got - start, (want - base)[:, :60], rtol=0, atol=2.0 ** -15)   # sums up to 2^8, steps of 2^-16


def test_importance_behind_a_long_history(H):
    """128 query heads on one KV head at a position of 2^24 + 1200: the block of the last sinks is 2^31 rows of (query, head)
    before the query, and its keys from there on are hidden by the window.

    Logits of 0, so that a visible key has 128 / 1100.  A weight is off by 2^-21 of itself for lse (7.003 as a float32, times
    log2 e: 10.1 x 2^-23 in all, and 2^-22 of ex2), its sum by 128 additions of 2^-24: below 2^-16."""
    m, heads, sinks, window = (1 << 24) + 1200, 128, 100, 1000
    q, k = torch.zeros(1, heads, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(m, 1, 128, dtype=torch.bfloat16, device="cuda")
    desc = H.make_packed(q, k, k, 1)
    lse, accum = torch.full((1, heads), float(np.log(sinks + window)), device="cuda"), torch.zeros(1, m, device="cuda")
    H.hill_prompt_importance(desc, q, k, lse, ints([0, 1]), ints([0, m]), sinks, window, ALL, accum, ws=H.alloc_prompt_workspace(desc))
    H.hill_sync_status()
    want = heads / (sinks + window)
    for seen in (accum[0, :sinks], accum[0, m - window:]):
        assert ((seen - want).abs() <= want * 2.0 ** -16).all()
    assert not accum[0, sinks:m - window].any()


@pytest.mark.parametrize("dtype,low", [("bf16", -1e30), ("fp16", -60000.0)])
@pytest.mark.parametrize("heads", [(4, 1), (7, 1), (12, 1), (10, 2), (3, 3)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_importance_of_a_key_at_minus_infinity(H, heads, dtype, low):
    """A seen key whose logits are all -infinity has the weight 0, whatever the size of the group: as one whose
    logits are below -500, which changes no bit of the others (2^-720 is 0 in float32)."""
    c = Case(H, [(300, 0)], *heads, dtype, seed=40 + heads[0])
    c.q[:, :, 5] = c.q[:, :, 5].abs() + 0.125      # 60000 x 0.125 / sqrt(128) = 663
    c.k[40, :, 5] = low
    c.attend(0, ALL)
    start, want, lse = run_importance(H, c, 0, ALL, ALL, True, 300)
    assert torch.equal(want[:, :, 40], start[:, :, 40]) and torch.isfinite(lse).all()
    c.k[40, :, 5] = -float("inf")
    _, got, _ = run_importance(H, c, 0, ALL, ALL, True, 300, lse)
    H.hill_sync_status()
    assert torch.equal(got, want)


@pytest.mark.parametrize("kvh", [False, True], ids=["seq", "kvh"])
def test_importance_as_the_first_weights_of_an_insert(H, kvh):
    """Prompts go into bounded caches with the weights that their tokens received, as they lie; the next tokens take the
    slots of the smallest."""
    B, T, HQ, HKV, sinks, more = 2, 60, 8, 2, 4, 6
    c = Case(H, [(T, 0)] * B, HQ, HKV, seed=60)
    c.attend(0, ALL)
    rows = (B, HKV) if kvh else (B,)
    w = torch.zeros(*rows, T, device="cuda")
    H.hill_prompt_importance(c.desc, c.q, c.k, c.lse, c.qs, c.ks, 0, ALL, ALL, w, kvh=kvh, ws=H.alloc_prompt_workspace(c.desc))
    cache = H.BoundedCache(B, HQ, HKV, T + sinks, c.dt, sinks=sinks, kvh=kvh, max_new=T)
    new = [x.view(B, T, HKV, 128).transpose(1, 2) for x in (c.k, c.v)]
    cache.insert(*new, w_new=w)
    H.hill_sync_status()
    assert torch.equal(cache.accum[..., :T], w) and torch.all(cache.slots == torch.arange(T, device="cuda"))
    for x, held in zip(new, (cache.K, cache.V)):
        assert torch.equal(held[:, :, :T], x)
    assert (w.sum(-1) - T * HQ / (HKV if kvh else 1)).abs().max() < 1e-2      # every query gives 1 per head, to 2^-16
    # the free slots first, then the least weights behind the sinks; ties go to the later slot
    cache.insert(*(x[:, :, :sinks + more].contiguous() for x in new), w_new=torch.full((*rows, sinks + more), 1e6, device="cuda"))
    H.hill_sync_status()
    got = cache.slots.flatten()[:w[..., 0].numel() * (sinks + more)].view(*rows, sinks + more).cpu()
    for at in np.ndindex(rows):
        order = sorted(range(sinks, T), key=lambda j: (-float(w[at][j]), j))
        assert got[at].tolist() == list(range(T, T + sinks)) + sorted(order[-more:])
