"""Caches in pages against plain float64 forms (tests/paged_util.py, tests/bounded_util.py): attention of one token,
rows written (quantised) and read back, and a run of the calls together."""
import numpy as np
import pytest
import torch

from bounded_util import attn
from paged_util import ALL, HALF, paged_rows, prompt, quantise

pytestmark = pytest.mark.gpu

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
F8 = torch.float8_e4m3fn


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
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def f64(t):
    return t.double().cpu().numpy()


def check(got, ref, bound):
    assert not np.isnan(got).any()
    err = np.abs(got - ref)
    bad = np.argwhere(err > bound + 1e-30)
    assert not len(bad), (f"{len(bad)} of {err.size} out of bounds; first {bad[0]}: {got[tuple(bad[0])]} for "
                          f"{ref[tuple(bad[0])]}, bound {bound[tuple(bad[0])]}")


class Cache:
    """Pools of random rows under a shuffled table; entries that no length reaches are -1 or past the pool."""

    def __init__(self, H, held, Hq, Hkv, page, dtype="bf16", e4m3=False, seed=0, scale=1.0, spread=False):
        self.H, self.dt, self.e4m3, self.page = H, DT[dtype], e4m3, page
        g, B = gen(seed), len(held)
        cols = max(1, -(-max(held) // page))
        self.cap, used = cols * page, [-(-n // page) for n in held]
        pages = sum(used) + 3
        order = np.random.RandomState(seed).permutation(pages)
        table = np.random.RandomState(seed + 1).choice([-1, pages, 1 << 30], (B, cols))
        for b, n in enumerate(used):
            table[b, :n] = order[sum(used[:b]):sum(used[:b + 1])]
        self.table_np, self.table = table, ints(table)
        loud = 1 + 5 * (torch.rand(1, Hkv, 1, 128, generator=g, device="cuda") < 0.05)
        K, V = ((torch.randn(pages, Hkv, page, 128, generator=g, device="cuda") + 0.3) * loud * scale for _ in range(2))
        if e4m3:
            self.scales = torch.empty(pages, Hkv, page, 2, device="cuda")
            pools, vals = [], []
            for i, x in enumerate((K, V)):
                if spread and i == 1:      # V rows of very different sizes
                    x = x * torch.exp2(torch.randint(-20, 20, (pages, Hkv, page, 1), generator=g, device="cuda").float())
                amax = x.abs().amax(-1, keepdim=True)
                codes = (x * (448 / amax)).clamp(-448, 448).to(F8)
                self.scales[..., i] = (amax / 448)[..., 0]
                pools.append(codes)
                vals.append(f64(codes.float()) * f64(self.scales[..., i])[..., None])
            self.k, self.v = pools
        else:
            self.scales = None
            self.k, self.v = K.to(self.dt), V.to(self.dt)
            vals = [f64(self.k), f64(self.v)]
        self.K64, self.V64 = (paged_rows(x, table, self.cap) for x in vals)
        self.q = torch.randn(B, Hq, 128, generator=g, device="cuda").to(self.dt)
        self.out = torch.full((B, Hq, 128), float("nan"), device="cuda")
        self.handle()

    def handle(self):
        self.pages = self.H.make_pages(self.k, self.v, self.table, self.scales)
        self.desc = self.H.make_desc_paged(self.q, self.pages)

    def attend(self, lens, sinks, window, accum=None, kvh=False, ws=None, stream=None):
        H = self.H
        ws = ws if ws is not None else H.alloc_window_workspace(self.desc, accum is not None)
        H.hill_paged_attn(self.desc, self.q, self.pages, ints(lens), sinks, window, self.out, accum=accum, kvh=kvh, ws=ws,
                          stream=stream)
        H.hill_sync_status(stream)
        return f64(self.out)

    def verify(self, lens, sinks, window, kvh=False):
        ref, w, bound, wb = attn(f64(self.q), self.K64, self.V64, np.asarray(lens), sinks, window, kvh)
        start = torch.rand(*w.shape, device="cuda", generator=gen(3))
        accum = start.clone()
        check(self.attend(lens, sinks, window, accum, kvh), ref, bound)
        old = f64(start)
        check(f64(accum), old + w, wb + 2.0 ** -23 * (old + w))
        assert torch.equal(accum.cpu()[torch.from_numpy(w == 0)], start.cpu()[torch.from_numpy(w == 0)])
        again = self.out.clone()
        self.out.fill_(float("nan"))
        self.attend(lens, sinks, window, kvh=kvh)   # without an importance: the same output
        assert torch.equal(self.out, again)


FORMS = pytest.mark.parametrize("e4m3", [False, True], ids=["16bit", "e4m3"])
HEADS = [(4, 4), (8, 2), (14, 2), (16, 2), (12, 1), (32, 1), (5, 5), (20, 1)]
RULES = [(0, ALL), (4, 64), (0, 0), (3, 0), (61, 100), (200, 1), (0, 33), (32, 32)]


@FORMS
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}x{h[1]}")
def test_attention(H, heads, dtype, e4m3):
    lens = [0, 1, 31, 32, 33, 95, 300, 301]
    for page in (16, 64):
        c = Cache(H, lens, *heads, page, dtype, e4m3, seed=heads[0])
        for sinks, window in RULES:
            c.verify(lens, sinks, window)


@FORMS
@pytest.mark.parametrize("page", [16, 32, 48, 64, 112, 256])
def test_page_sizes(H, page, e4m3):
    lens = [5 * page + 7, 3 * page, 0, 1, page - 1, page + 1, 999]
    c = Cache(H, lens, 8, 2, page, "bf16", e4m3, seed=page)
    for sinks, window in [(0, ALL), (4, 300), (page + 1, page)]:
        c.verify(lens, sinks, window)


@FORMS
@pytest.mark.parametrize("heads", [(8, 4), (24, 2), (3, 3)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_rows_per_kv_head(H, heads, e4m3):
    B, Hkv = 3, heads[1]
    lens = np.random.RandomState(1).randint(0, 516, (B, Hkv))
    lens[0, 0], lens[1, 1] = 0, 515
    c = Cache(H, [515] * B, *heads, 16, "fp16", e4m3, seed=5)
    for sinks, window in [(0, ALL), (4, 100)]:
        c.verify(lens, sinks, window, kvh=True)


@FORMS
@pytest.mark.parametrize("heads,held", [((8, 2), [9000, 20000]), ((32, 32), [5000, 2, 1200]), ((32, 1), [7000] * 5),
                                        ((16, 1), [30000]), ((4, 4), [3000] * 40)])
def test_long_rows(H, heads, held, e4m3):
    """The list over all SMs and the clusters, runs of more than 32 boxes."""
    for page in (16, 112):
        c = Cache(H, held, *heads, page, "bf16", e4m3, seed=7)
        for sinks, window in [(0, ALL), (40, 1500)]:
            ref, w, bound, wb = attn(f64(c.q), c.K64, c.V64, np.asarray(held), sinks, window)
            accum = torch.zeros(len(held), c.cap, device="cuda")
            check(c.attend(held, sinks, window, accum), ref, bound)
            check(f64(accum), w, wb + 2.0 ** -23 * w)


@FORMS
def test_lengths_past_the_table_and_below_zero(H, e4m3):
    c = Cache(H, [200, 100], 8, 2, 16, "bf16", e4m3, seed=8)
    want = c.attend([c.cap, 0], 0, ALL)
    assert np.array_equal(c.attend([1 << 30, -5], 0, ALL), want)


@FORMS
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_hidden_slots_do_not_matter(H, e4m3, bad):
    """Slots behind a row's end, between sinks and window, and of other pages hold anything."""
    lens, sinks, window = [70, 301, 17], 5, 40
    c = Cache(H, lens, 8, 2, 16, "fp16", e4m3, seed=9)
    accum = torch.zeros(3, c.cap, device="cuda")
    want = c.attend(lens, sinks, window, accum)
    wa = accum.clone()
    seen = np.zeros(c.k.shape[:1] + (16,), bool)
    for b, n in enumerate(lens):
        for p in list(range(min(sinks, n))) + list(range(max(0, n - window), n)):
            seen[c.table_np[b, p // 16], p % 16] = True
    at = torch.from_numpy(~seen).cuda()[:, None].expand(-1, 2, -1)
    for x in (c.k, c.v):
        if e4m3:
            x.view(torch.uint8)[at] = 0x7f
        else:
            x[at] = float(bad)
    if e4m3:
        c.scales[at] = float(bad)
    accum.zero_()
    assert np.array_equal(c.attend(lens, sinks, window, accum), want) and torch.equal(accum, wa)


@FORMS
def test_seen_values_that_are_not_finite_show(H, e4m3):
    lens = [300, 50]
    c = Cache(H, lens, 8, 2, 16, "bf16", e4m3, seed=10)
    want = c.attend(lens, 0, ALL)
    page, slot = c.table_np[0, 77 // 16], 77 % 16
    if e4m3:
        c.v.view(torch.uint8)[page, 1, slot, 9] = 0x7f
    else:
        c.v[page, 1, slot, 9] = float("nan")
    out = c.attend(lens, 0, ALL)
    mask = np.ones_like(out, bool)
    mask[0, 4:, 9] = False
    assert np.isnan(out[~mask]).all() and np.array_equal(out[mask], want[mask])
    if e4m3:
        c.scales[page, 0, slot, 0] = float("nan")
    else:
        c.k[page, 0, slot, 3] = float("nan")
    out = c.attend(lens, 0, ALL)
    assert np.isnan(out[0, :4]).all() and np.array_equal(out[1], want[1])


def test_rows_of_very_different_size(H):
    """V rows of E4M3 whose scales span 2^40, and growing logits."""
    for dtype in DT:
        c = Cache(H, [700, 90], 8, 2, 16, dtype, True, seed=11, scale=1.5, spread=True)
        c.verify([700, 90], 0, ALL)


@FORMS
def test_pages_outside_the_pool(H, e4m3):
    """A page that is looked at and not there reads as zeros and is an error; one that is hidden is none."""
    lens = [100, 60]
    for page in (16, 32):
        c = Cache(H, lens, 8, 2, page, "bf16", e4m3, seed=12)
        for bad in (-1, c.k.shape[0], 1 << 30):
            c.table[0, 1] = bad
            with pytest.raises(H.HillError) as e:
                c.attend(lens, 0, ALL)
            assert e.value.status == H.HILL_ERR_DEVICE
            K, V = c.K64.copy(), c.V64.copy()
            K[0, :, page:2 * page] = V[0, :, page:2 * page] = 0
            ref, _, bound, _ = attn(f64(c.q), K, V, lens, 0, ALL)
            check(f64(c.out), ref, bound)
            c.attend(lens, 3, 20)     # hidden there
            if page == 16:
                want = attn(f64(c.q), K, V, lens, 3, 20)
                check(f64(c.out), want[0], want[2])


@FORMS
@pytest.mark.parametrize("page", [16, 32])
def test_a_window_of_nothing_looks_at_no_page(H, page, e4m3):
    """Sinks alone are visible: the pages behind them may be gone, the last token's among them."""
    lens, sinks = [100, 70], 3
    c = Cache(H, lens, 8, 2, page, "bf16", e4m3, seed=32)
    want = c.attend(lens, sinks, 0)
    c.table[:, 1:] = -1
    assert np.array_equal(c.attend(lens, sinks, 0), want)
    c.table[0, 0] = -1           # the sinks' own page
    with pytest.raises(H.HillError) as e:
        c.attend(lens, sinks, 0)
    assert e.value.status == H.HILL_ERR_DEVICE


@FORMS
def test_no_pages_at_all(H, e4m3):
    """A pool without a page: nothing is read or written; what is looked at counts as zeros, and is an error."""
    pool = torch.zeros(0, 2, 16, 128, device="cuda").to(F8 if e4m3 else torch.bfloat16)
    sc = torch.zeros(0, 2, 16, 2, device="cuda") if e4m3 else None
    table = ints([[0, -1, 5], [1 << 30, 0, 0]])
    pages = H.make_pages(pool, pool.clone(), table, sc)
    q = torch.randn(2, 8, 128, generator=gen(30), device="cuda").bfloat16()
    desc, out, accum = H.make_desc_paged(q, pages), torch.full((2, 8, 128), 7.0, device="cuda"), torch.zeros(2, 48, device="cuda")
    ws = H.alloc_window_workspace(desc, True)
    H.hill_paged_attn(desc, q, pages, ints([0, 0]), 0, ALL, out, accum=accum, ws=ws)
    H.hill_sync_status()
    assert torch.all(out == 0) and torch.all(accum == 0)
    H.hill_paged_attn(desc, q, pages, ints([40, 3]), 0, ALL, out, accum=accum, ws=ws)
    with pytest.raises(H.HillError):
        H.hill_sync_status()
    assert torch.all(out == 0)      # of values that are zeros
    np.testing.assert_allclose(f64(accum)[0, :40], 8 / 40, rtol=1e-5)
    k, v = new_rows(5, 2, torch.bfloat16, 31)
    H.hill_paged_write(desc, pages, k, v, ints([0, 3, 5]), ints([0, 1]))
    with pytest.raises(H.HillError):
        H.hill_sync_status()


@FORMS
def test_graph_stream_and_shared_pages(H, e4m3):
    """A captured call follows its table, lengths and pools; two sequences may share pages."""
    lens = [300, 300]
    c = Cache(H, lens, 8, 2, 16, "bf16", e4m3, seed=13)
    c.table[1] = c.table[0]
    c.q[1] = c.q[0]
    out = c.attend(lens, 0, ALL)
    assert np.array_equal(out[0], out[1])
    ws, ld = H.alloc_window_workspace(c.desc, True), ints(lens)
    accum = torch.zeros(2, c.cap, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call = lambda: H.hill_paged_attn(c.desc, c.q, c.pages, ld, 2, 250, c.out, accum=accum, ws=ws)
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        c.table.copy_(c.table.flip(0))
        ld.copy_(ints([123, 31]))
        c.q.copy_(c.q.flip(0) * 0.5)
        accum.zero_()
        graph.replay()
        side.synchronize()
        got, ga = f64(c.out), accum.clone()
        accum.zero_()
        call()
        H.hill_sync_status(side)
        assert np.array_equal(f64(c.out), got) and torch.equal(accum, ga)


# ---------------------------------------------------------------- rows in and out
def new_rows(T, Hkv, dt, seed, wide=False):
    g = gen(seed)
    rows = []
    for i in range(2):
        x = (torch.randn(T, Hkv, 128, generator=g, device="cuda") * torch.exp2(
            torch.randint(-8, 8, (T, Hkv, 1), generator=g, device="cuda").float())).to(dt)
        if wide:
            w = torch.zeros(T, 2 * Hkv + 1, 136, dtype=dt, device="cuda")
            w[:, 1::2, :128] = x
            x = w[:, 1::2, :128]
        rows.append(x)
    return rows


@FORMS
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,begin", [([1] * 16, [5 * i for i in range(16)]), ([0, 7, 0, 130, 1], [3, 0, 9, 14, 200]),
                                        ([700, 2000], [0, 50])], ids=["step", "ragged", "prompt"])
def test_write_and_read(H, lens, begin, dtype, e4m3):
    dt = DT[dtype]
    for Hkv, page, wide in ((2, 16, False), (5, 112, True), (1, 32, False)):
        c = Cache(H, [n + b for n, b in zip(lens, begin)], 2 * Hkv, Hkv, page, dtype, e4m3, seed=14)
        T, B = sum(lens), len(lens)
        k, v = new_rows(T + 4, Hkv, dt, 15, wide)     # two rows before the first sequence, two behind the last
        k[3 % T, 0] = 0                               # a row of zeros
        before = [x.clone() for x in (c.k, c.v)] + ([c.scales.clone()] if e4m3 else [])
        starts = [2 + sum(lens[:b]) for b in range(B + 1)]
        H.hill_paged_write(c.desc, c.pages, k, v, ints(starts), ints(begin))
        K, V = (torch.full((B, Hkv, c.cap + 5, 128), 3.0, dtype=dt, device="cuda") for _ in range(2))
        desc = H.make_desc(c.q, K, V)
        H.hill_paged_read(desc, c.pages, ints(begin), ints([b + n for b, n in zip(begin, lens)]), max(lens), K, V)
        H.hill_sync_status()
        touched = torch.zeros(c.k.shape[0], page, dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            rows = slice(starts[b], starts[b] + n)
            pos = np.arange(begin[b], begin[b] + n)
            touched[torch.from_numpy(c.table_np[b, pos // page]).long().cuda(), torch.from_numpy(pos % page).cuda()] = True
            for new, got in ((k, K), (v, V)):
                x = f64(new[rows]).transpose(1, 0, 2)
                if e4m3:
                    codes, scale = quantise(x)
                    x = f64(torch.from_numpy(codes.astype(np.float32) * scale[..., None]).to(dt))
                assert np.array_equal(f64(got[b, :, begin[b]:begin[b] + n]), x)
                assert torch.all(got[b, :, :begin[b]] == 3) and torch.all(got[b, :, begin[b] + n:] == 3)
        for was, now in zip(before, [c.k, c.v] + ([c.scales] if e4m3 else [])):   # other slots as they were
            rest = ~touched[:, None].expand(-1, Hkv, -1)
            bits = (lambda t: t.view(torch.uint8)) if e4m3 and now.dim() == 4 and now.shape[-1] == 128 else (lambda t: t)
            assert torch.equal(bits(was)[rest], bits(now)[rest])


def test_pages_written_before_they_are_scored(H):
    """A 16-bit pool with one page to a sequence is a contiguous cache: scoring it behind a write sees the new rows."""
    B, Hkv, cap, dt = 4, 8, 4096, torch.bfloat16
    k, v = (torch.zeros(B, Hkv, cap, 128, dtype=dt, device="cuda") for _ in range(2))
    q = torch.randn(B, 32, 128, generator=gen(41), device="cuda").to(dt)
    pages, desc = H.make_pages(k, v, ints([[b] for b in range(B)])), H.make_desc(q, k, v)
    new, lens = torch.zeros(B * cap, Hkv, 128, dtype=dt, device="cuda"), ints([cap] * B)
    starts, begin, ws = ints([b * cap for b in range(B + 1)]), ints([0] * B), H.alloc_workspace(desc, H.HILL_SCORE_ATTN, 0)
    got, want = (torch.zeros(B, cap, device="cuda") for _ in range(2))

    def chain():
        H.hill_paged_write(desc, pages, new, new, starts, begin)
        H.hill_score(desc, q, k, lens, H.HILL_SCORE_ATTN, got, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            chain()
        for i in range(20):
            new.copy_(torch.randn(new.shape, generator=gen(50 + i), device="cuda"))
            k.zero_()
            graph.replay() if i % 2 else chain()
            side.synchronize()
            H.hill_score(desc, q, k, lens, H.HILL_SCORE_ATTN, want, ws=ws)     # the rows are there by now
            H.hill_sync_status(side)
            assert torch.equal(got, want)
            assert torch.equal(k, new.view(B, cap, Hkv, 128).transpose(1, 2))


def test_codes_bit_for_bit(H):
    """Codes and scales of rows at the borders: halfway values, the largest, tiny ones, all of one sign."""
    for dtype in DT:
        dt = DT[dtype]
        c = Cache(H, [64], 2, 1, 16, dtype, True, seed=16)
        k, v = new_rows(64, 1, dt, 17)
        k[0] = 448
        k[1] = torch.arange(128, device="cuda")
        k[2] = torch.finfo(dt).max
        k[3] = torch.finfo(dt).tiny
        k[4], k[5] = 0, -0.0
        k[6, 0, 1:] = 0
        k[7, 0, ::2] *= 2.0 ** -9
        if dt == torch.bfloat16:
            k[8] = 2.0 ** -119
            k[9] = 2.0 ** -121
        H.hill_paged_write(c.desc, c.pages, k, v, ints([0, 64]), ints([0]))
        H.hill_sync_status()
        for i, (new, pool) in enumerate(((k, c.k), (v, c.v))):
            codes, scale = quantise(f64(new)[:, 0])
            got = paged_rows(f64(pool.float()), c.table_np, 64)[0, 0]
            assert np.array_equal(got, codes)
            assert np.array_equal(paged_rows(c.scales.cpu().numpy(), c.table_np, 64)[0, 0, :, i], scale)


def test_new_rows_that_are_not_finite(H):
    c = Cache(H, [32], 2, 1, 16, "bf16", True, seed=18)
    k, v = new_rows(32, 1, torch.bfloat16, 19)
    k[3, 0, 7], k[4] = float("nan"), float("nan")
    k[5, 0, 9] = float("inf")
    H.hill_paged_write(c.desc, c.pages, k, v, ints([0, 32]), ints([0]))
    K, V = (torch.zeros(1, 1, 32, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    H.hill_paged_read(H.make_desc(c.q, K, V), c.pages, ints([0]), ints([32]), 32, K, V)
    H.hill_sync_status()
    bad = ~torch.isfinite(K[0, 0])
    assert bad[3, 7] and bad[4].all() and bad[5].all() and not bad[[0, 1, 2] + list(range(6, 32))].any()
    assert torch.isfinite(V).all()


@FORMS
def test_places_that_are_not_there(H, e4m3):
    """Rows past the table, before its start, in pages outside the pool: dropped, and an error."""
    c = Cache(H, [100, 100], 4, 2, 16, "bf16", e4m3, seed=20)
    k, v = new_rows(20, 2, torch.bfloat16, 21)
    pools = [c.k.view(torch.uint8).clone(), c.v.view(torch.uint8).clone()]
    for begin, table in (([c.cap - 3, 0], None), ([0, -2], None), ([1 << 30, 0], None), ([0, 0], -1), ([0, 0], 1 << 29)):
        c.k.view(torch.uint8).copy_(pools[0])
        c.v.view(torch.uint8).copy_(pools[1])
        kept = c.table.clone()
        if table is not None:
            c.table[1, 0] = table
        H.hill_paged_write(c.desc, c.pages, k, v, ints([0, 10, 20]), ints(begin))
        with pytest.raises(H.HillError) as e:
            H.hill_sync_status()
        assert e.value.status == H.HILL_ERR_DEVICE
        c.table.copy_(kept)
        changed = (c.k.view(torch.uint8) != pools[0]).flatten(3).any(-1).any(1).sum().item()
        want = 0 if begin[0] == 1 << 30 else min(10, c.cap - begin[0])
        want += max(0, 10 + min(0, begin[1])) if table is None else 0
        assert changed == want
    K, V = (torch.full((2, 2, c.cap, 128), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.table[0, -1] = c.table[0, 0]     # (the table's last page belongs to no length here)
    c.table[1, 0] = -1
    H.hill_paged_read(H.make_desc(c.q, K, V), c.pages, ints([-5, 10]), ints([1 << 30, 20]), 1 << 20, K, V)
    with pytest.raises(H.HillError):
        H.hill_sync_status()
    assert torch.all(K[1, :, :16] == 3) and torch.all(K[1, :, 20:] == 3)
    assert (K[0, :, :100].flatten(2) != 3).any(-1).all()


def test_offsets_past_32_bits(H):
    """Pools of more than 2^32 bytes and elements: the last pages are written, read and attended."""
    page, Hkv = 256, 8
    pages = (1 << 32) // (page * Hkv * 128) + 40
    k, v = (torch.zeros(pages, Hkv, page, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = ints([[pages - 1, pages - 20, pages - 3]])
    handle = H.make_pages(k, v, table)
    q = torch.randn(1, 16, 128, generator=gen(22), device="cuda").bfloat16()
    desc = H.make_desc_paged(q, handle)
    kn, vn = new_rows(700, Hkv, torch.bfloat16, 23)
    H.hill_paged_write(desc, handle, kn * 0.01, vn, ints([0, 700]), ints([0]))
    out = torch.zeros(1, 16, 128, device="cuda")
    H.hill_paged_attn(desc, q, handle, ints([700]), 0, ALL, out, ws=H.alloc_window_workspace(desc, False))
    H.hill_sync_status()
    K64 = f64((kn * 0.01).transpose(0, 1))[None]
    ref, _, bound, _ = attn(f64(q), K64, f64(vn.transpose(0, 1))[None], [700], 0, ALL)
    check(f64(out), ref, bound)


# ---------------------------------------------------------------- together
@FORMS
def test_a_prompt_then_decode_steps(H, e4m3):
    """Prompts attended and written, their importance as the start of the running one, then steps over the pages."""
    lens, Hq, Hkv, page, steps, dt = [150, 37], 8, 2, 16, 5, torch.bfloat16
    c = Cache(H, [n + steps for n in lens], Hq, Hkv, page, "bf16", e4m3, seed=24)
    g, T, B = gen(25), sum(lens), 2
    q = torch.randn(T, Hq, 128, generator=g, device="cuda").to(dt)
    k, v = (torch.randn(T, Hkv, 128, generator=g, device="cuda").to(dt) for _ in range(2))
    starts, accum = ints([0, 150, 187]), torch.zeros(B, c.cap, device="cuda")
    desc = H.make_packed(q, k, v, B)
    out, lse = torch.zeros_like(q), torch.zeros(T, Hq, device="cuda")
    H.hill_prompt_attn(desc, q, k, v, starts, starts, 0, ALL, out, lse=lse)
    H.hill_prompt_importance(desc, q, k, lse, starts, starts, 0, ALL, ALL, accum, ws=H.alloc_prompt_workspace(desc))
    H.hill_paged_write(c.desc, c.pages, k, v, starts, ints([0, 0]))
    H.hill_sync_status()
    ref, _, bound, _ = prompt(f64(q), f64(k), f64(v), [0, 150, 187], [0, 150, 187], 0, ALL, HALF[dt])
    check(f64(out), ref, bound)
    total = f64(accum).sum(1)
    np.testing.assert_allclose(total, [n * Hq for n in lens], rtol=1e-4)   # every query gives 1 per head
    K64, V64 = np.zeros((B, Hkv, c.cap, 128)), np.zeros((B, Hkv, c.cap, 128))

    def held(x):
        if not e4m3:
            return f64(x)
        codes, scale = quantise(f64(x))
        return codes * scale.astype(np.float64)[..., None]

    for b in range(B):
        rows = slice([0, 150][b], [150, 187][b])
        K64[b, :, :lens[b]], V64[b, :, :lens[b]] = held(k[rows].transpose(0, 1)), held(v[rows].transpose(0, 1))
    ws = H.alloc_window_workspace(c.desc, True)
    for s in range(steps):
        kn, vn = (torch.randn(B, Hkv, 128, generator=g, device="cuda").to(dt) for _ in range(2))
        c.q.copy_(torch.randn(B, Hq, 128, generator=g, device="cuda"))
        at = [n + s for n in lens]
        H.hill_paged_write(c.desc, c.pages, kn, vn, ints([0, 1, 2]), ints(at))
        for b in range(B):
            K64[b, :, at[b]], V64[b, :, at[b]] = held(kn[b]), held(vn[b])
        before = f64(accum)
        got = c.attend([n + 1 for n in at], 4, 100, accum, ws=ws)
        ref, w, bound, wb = attn(f64(c.q), K64, V64, [n + 1 for n in at], 4, 100)
        check(got, ref, bound)
        check(f64(accum), before + w, wb + 2.0 ** -23 * (before + w))
