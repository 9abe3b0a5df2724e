"""The calls of a bounded cache against plain float64 forms (tests/bounded_util.py): attention over sinks and a window
from 16-bit and 4-bit caches with the weights accumulated, inserts that evict, 4-bit rows."""
import numpy as np
import pytest
import torch

from bounded_util import ALL, attn, encode, insert, pack, values

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


def to16(dtype):
    return lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dtype).double().numpy()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Case:
    """A cache of random rows with loud channels, in 16 or 4 bits, and its float64 values."""

    def __init__(self, H, B, Hq, Hkv, cap, dtype="fp16", q4=False, seed=0, layout="head", scale=1.0):
        self.H, self.q4, dt = H, q4, DT[dtype]
        g = gen(seed)
        self.q = torch.randn(B, Hq, 128, generator=g, device="cuda").to(dt)
        loud = 1 + 5 * (torch.rand(1, Hkv, 1, 128, generator=g, device="cuda") < 0.05)
        K, V = (((torch.randn(B, Hkv, cap, 128, generator=g, device="cuda") + 0.3) * loud * scale).to(dt) for _ in range(2))
        if layout == "token":
            K, V = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (K, V))
        self.K, self.V = K, V
        self.K64, self.V64 = K.double().cpu().numpy(), V.double().cpu().numpy()
        if q4:
            self.k4, self.v4, self.params = H.alloc_q4(B, Hkv, cap, dt)
            sides = []
            for i, (x, codes) in enumerate(((self.K64, self.k4), (self.V64, self.v4))):
                c, s, lo = encode(x, to16(dt))
                codes.copy_(torch.from_numpy(pack(c)))
                self.params[:, :, :cap, 2 * i] = torch.from_numpy(s).to(dt).cuda()
                self.params[:, :, :cap, 2 * i + 1] = torch.from_numpy(lo).to(dt).cuda()
                sides.append(values(pack(c), s, lo))
            self.K64, self.V64 = sides
            self.desc = H.make_desc_q4(self.q, self.k4)
        else:
            self.desc = H.make_desc(self.q, K, V)
        self.out = torch.full((B, Hq, 128), float("nan"), device="cuda")

    def attend(self, lens, sinks, window, accum=None, kvh=False, ws=None, stream=None):
        H = self.H
        lens = torch.as_tensor(np.asarray(lens), dtype=torch.int32, device="cuda")
        ws = ws if ws is not None else H.alloc_window_workspace(self.desc, accum is not None)
        if self.q4:
            H.hill_window_attn_q4(self.desc, self.q, self.k4, self.v4, self.params, lens, sinks, window, self.out,
                                  accum=accum, kvh=kvh, ws=ws, stream=stream)
        else:
            H.hill_window_attn(self.desc, self.q, self.K, self.V, lens, sinks, window, self.out, accum=accum, kvh=kvh,
                               ws=ws, stream=stream)
        H.hill_sync_status(stream)
        return self.out.cpu().numpy().astype(np.float64)

    def reference(self, lens, sinks, window, kvh=False):
        return attn(self.q.double().cpu().numpy(), self.K64, self.V64, np.asarray(lens), sinks, window, kvh)


def check(got, ref, bound):
    err = np.abs(got - ref)
    assert not np.isnan(got).any()
    bad = np.argwhere(err > bound + 1e-30)
    assert not len(bad), (f"{len(bad)} of {err.size} out of bounds; first {bad[0]}: {got[tuple(bad[0])]} for "
                          f"{ref[tuple(bad[0])]}, bound {bound[tuple(bad[0])]}")


HEADS = [(4, 4), (8, 2), (14, 2), (16, 2), (12, 1), (32, 1), (5, 5), (20, 1)]
RULES = [(0, ALL), (4, 64), (0, 0), (3, 0), (61, 100), (200, 1), (0, 33), (32, 32)]


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}x{h[1]}")
def test_attention(H, heads, dtype, q4):
    lens = [0, 1, 31, 32, 33, 95, 300, 301]
    c = Case(H, len(lens), *heads, 301, dtype, q4, seed=heads[0])
    for sinks, window in RULES:
        ref, w, bound, wb = c.reference(lens, sinks, window)
        start = torch.rand(len(lens), 301, device="cuda", generator=gen(3))
        accum = start.clone()
        check(c.attend(lens, sinks, window, accum), ref, bound)
        old = start.cpu().numpy().astype(np.float64)
        check(accum.cpu().numpy().astype(np.float64), old + w, wb + 2.0 ** -23 * (old + w))
        assert torch.equal(accum.cpu()[torch.from_numpy(w == 0)], start.cpu()[torch.from_numpy(w == 0)])
        again = c.out.clone()
        c.out.fill_(float("nan"))
        c.attend(lens, sinks, window)   # without an importance: the same output
        assert torch.equal(c.out, again)


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("heads", [(8, 4), (24, 2), (3, 3)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_rows_per_kv_head(H, heads, q4):
    B, Hkv, cap = 3, heads[1], 515
    lens = np.random.RandomState(1).randint(0, cap + 1, (B, Hkv))
    lens[0, 0], lens[1, 1] = 0, cap
    c = Case(H, B, *heads, cap, "fp16", q4, seed=5)
    for sinks, window in [(0, ALL), (4, 100)]:
        ref, w, bound, wb = c.reference(lens, sinks, window, kvh=True)
        accum = torch.zeros(B, Hkv, cap, device="cuda")
        check(c.attend(lens, sinks, window, accum, kvh=True), ref, bound)
        check(accum.cpu().numpy().astype(np.float64), w, wb + 2.0 ** -23 * w)


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("shape", [(1, 8, 1, 40000), (2, 32, 8, 9001), (300, 2, 2, 70), (1, 64, 8, 2049), (40, 40, 40, 33)])
def test_split_and_joined(H, shape, q4):
    """Long rows over many warps, many rows over few, lengths past the capacity and below zero."""
    B, Hq, Hkv, cap = shape
    lens = np.random.RandomState(2).randint(max(0, cap - 40), cap + 1, B)
    lens[-1] = cap + 7
    if B > 2:
        lens[1], lens[2] = -3, 0
    c = Case(H, B, Hq, Hkv, cap, "bf16", q4, seed=7)
    ref, w, bound, wb = c.reference(lens, 0, ALL)
    accum = torch.zeros(B, cap, device="cuda")
    check(c.attend(lens, 0, ALL, accum), ref, bound)
    check(accum.cpu().numpy().astype(np.float64), w, wb + 2.0 ** -23 * w)
    a, b = c.out.clone(), accum.clone()
    accum.zero_()
    c.attend(lens, 0, ALL, accum, ws=torch.full((H.hill_window_workspace_bytes(c.desc, True),), 0xff, dtype=torch.uint8, device="cuda"))
    assert torch.equal(a, c.out) and torch.equal(b, accum)   # bit for bit, whatever the workspace held


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (14, 2), (16, 2), (12, 1), (32, 1)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_both_forms(H, heads, dtype, q4):
    """Few short rows go to clusters, rows for which there are too few SMs to the list of tiles with its merge: the
    launches say so; long rows to either.  All are right, with and without the importance."""
    def run(c, lens, sinks, window, forms):
        n0 = H.hill_kernel_launches()
        got = c.attend(lens, sinks, window)
        assert H.hill_kernel_launches() - n0 in forms
        ref, w, bound, wb = c.reference(lens, sinks, window)
        check(got, ref, bound)
        accum = torch.zeros(w.shape, device="cuda")
        n0 = H.hill_kernel_launches()
        check(c.attend(lens, sinks, window, accum), ref, bound)
        assert H.hill_kernel_launches() - n0 - 1 in forms
        check(accum.cpu().numpy().astype(np.float64), w, wb + 2.0 ** -23 * w)

    c = Case(H, 3, *heads, 30000, dtype, q4, seed=43)
    run(c, [1000, 700, 64], 0, 900, (1,))
    run(c, [30000, 12345, 1], 0, ALL, (1, 2))
    run(c, [30000, 20000, 0], 100, 25000, (1, 2))
    c = Case(H, 160, *heads, 150, dtype, q4, seed=53)
    run(c, np.random.RandomState(5).randint(0, 151, 160), 3, 130, (2,))


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("shape", [(12, 32, 1, 9000), (6, 32, 1, 20000), (1, 20, 1, 40000), (5, 64, 2, 5000)])
def test_merges_of_many_partials(H, shape, q4):
    """Long rows of large groups: merging CTAs of every size, more outputs than SMs, rows without a partial among them."""
    B, heads, Hkv, n = shape
    c = Case(H, B, heads, Hkv, n, "bf16", q4, seed=59)
    for lens in ([n] * B, [n if b % 3 == 0 else (n // 7 if b % 3 == 1 else 0) for b in range(B)]):
        ref, w, bound, wb = c.reference(lens, 0, ALL)
        accum = torch.zeros(w.shape, device="cuda")
        check(c.attend(lens, 0, ALL, accum), ref, bound)
        check(accum.cpu().numpy().astype(np.float64), w, wb + 2.0 ** -23 * w)


def test_values_far_from_one(H):
    """4-bit rows of 2^100 under queries of 2^-100, and the reverse: the logits are ordinary, their factors are not."""
    for scale in (2.0 ** 100, 2.0 ** -100):
        c = Case(H, 1, 8, 2, 300, "bf16", True, seed=47, scale=scale)
        c.q = (c.q.float() / scale / 8).bfloat16()
        c.desc = H.make_desc_q4(c.q, c.k4)
        ref, w, bound, _ = c.reference([300], 0, ALL)
        check(c.attend([300], 0, ALL), ref, bound)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), "lowest"])
def test_hidden_slots_do_not_matter(H, bad, dtype):
    bad = torch.finfo(DT[dtype]).min if bad == "lowest" else bad
    lens, sinks, window = [250, 77, 0], 5, 70
    for q4 in (False, True):
        c = Case(H, 3, 8, 2, 290, dtype, q4, seed=11)
        ref, w, bound, _ = c.reference(lens, sinks, window)
        hidden = torch.from_numpy(w == 0).cuda()
        for b in range(3):
            for x in ((c.params,) if q4 else (c.K, c.V)):
                x[b, :, :290][:, hidden[b]] = bad
            if q4:
                c.params[b, :, 290:] = bad
                c.k4[b][:, hidden[b]] = 255
                c.v4[b][:, hidden[b]] = 255
        accum = torch.full((3, 290), 0.5, device="cuda")
        check(c.attend(lens, sinks, window, accum), ref, bound)
        assert torch.all(accum[hidden] == 0.5) and not torch.isnan(accum).any()


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
def test_a_heavy_token_leaves_the_small_weights_exact(H, q4):
    """One token holds nearly all the weight: the rest is 2^-20 of it and still counts in the output."""
    c = Case(H, 1, 4, 1, 3000, "fp16", q4, seed=13, scale=0.05)
    n = 3000
    if not q4:
        u = c.q[0, 0].float() / c.q[0, 0].float().norm()
        c.K[0, 0, 1234] = (u * 16).half()
        c.V[0, 0, 1234] = 0
        c.K64, c.V64 = c.K.double().cpu().numpy(), c.V.double().cpu().numpy()
    ref, w, bound, _ = c.reference([n], 0, ALL)
    check(c.attend([n], 0, ALL), ref, bound)


@pytest.mark.parametrize("scale", [2.0 ** -12, 2.0 ** 9])
@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
def test_small_and_large_values(H, scale, q4):
    """Rows far from 1, with queries that make up for it, and V scales that grow along the row."""
    c = Case(H, 2, 8, 2, 400, "bf16", q4, seed=17, scale=scale)
    c.q = (c.q.float() / scale / 8).bfloat16()
    ramp = torch.ones(400)
    ramp[200:] = 1024.0
    if q4:
        c.params[:, :, :400, 2:] *= ramp[:, None].cuda().bfloat16()
        c.V64 = c.V64 * ramp[:, None].numpy()
    lens = [400, 133]
    ref, w, bound, _ = c.reference(lens, 0, ALL)
    check(c.attend(lens, 0, ALL), ref, bound)


@pytest.mark.parametrize("layout", ["token", "mixed"])
def test_strides(H, layout):
    B, Hq, Hkv, cap = 2, 8, 2, 201
    c = Case(H, B, Hq, Hkv, cap, "fp16", seed=19, layout="token")
    if layout == "mixed":   # K token by token, V inside a wider buffer, q with a stride
        wide = torch.full((B, Hkv, cap + 3, 256), float("nan"), dtype=torch.float16, device="cuda")
        wide[:, :, 1:cap + 1, 64:192] = c.V
        c.V = wide[:, :, 1:cap + 1, 64:192]
    qq = torch.full((B, Hq, 3, 128), float("nan"), dtype=torch.float16, device="cuda")
    qq[:, :, 1] = c.q
    c.q = qq[:, :, 1]
    c.desc = H.make_desc(c.q, c.K, c.V)
    ref, w, bound, _ = c.reference([201, 64], 4, 50)
    check(c.attend([201, 64], 4, 50), ref, bound)


def test_offsets_past_32_bits(H):
    """The last KV head of a cache of more than 2^31 elements, in both formats."""
    Hkv, cap, win = 130, 131073, 40
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    dt = torch.float16
    q = torch.randn(1, Hkv, 128, device="cuda", generator=gen(23)).to(dt)
    K, V = (torch.zeros(1, Hkv, cap, 128, dtype=dt, device="cuda") for _ in range(2))
    new = torch.randn(2, 1, Hkv, win, 128, device="cuda", generator=gen(24)).to(dt)
    lens = torch.tensor([cap], dtype=torch.int32, device="cuda")
    desc = H.make_desc(q, K, V)
    seen = torch.tensor([cap - win], dtype=torch.int32, device="cuda")
    state = dict(pos=torch.zeros(1, cap, dtype=torch.int32, device="cuda"), accum=torch.zeros(1, cap, device="cuda"))
    slots = torch.zeros(1, win, dtype=torch.int32, device="cuda")
    H.hill_cache_insert(desc, new[0], new[1], K, V, seen, state["pos"], state["accum"], 0, 0, slots)
    assert torch.equal(slots[0].cpu(), torch.arange(cap - win, cap, dtype=torch.int32))
    assert torch.equal(K[:, :, cap - win:], new[0]) and torch.equal(V[:, :, cap - win:], new[1])
    out = torch.empty(1, Hkv, 128, device="cuda")
    H.hill_window_attn(desc, q, K, V, lens, 0, win, out, ws=H.alloc_window_workspace(desc, False))
    k64, v64 = new[0].double().cpu().numpy(), new[1].double().cpu().numpy()
    ref, _, bound, _ = attn(q.double().cpu().numpy(), k64, v64, [win], 0, ALL)
    check(out.cpu().numpy().astype(np.float64), ref, bound)
    del K, V
    k4, v4, params = H.alloc_q4(1, Hkv, cap, dt)
    seen.fill_(cap - win)
    desc = H.make_desc_q4(q, k4)
    H.hill_cache_insert_q4(desc, new[0], new[1], k4, v4, params, seen, state["pos"], state["accum"], 0, 0, slots)
    H.hill_window_attn_q4(desc, q, k4, v4, params, lens, 0, win, out, ws=H.alloc_window_workspace(desc, False))
    H.hill_sync_status()
    stands = [values(pack(c), s, lo) for c, s, lo in (encode(x, to16(dt)) for x in (k64, v64))]
    ref, _, bound, _ = attn(q.double().cpu().numpy(), *stands, [win], 0, ALL)
    check(out.cpu().numpy().astype(np.float64), ref, bound)


def test_another_stream_and_a_graph(H):
    c = Case(H, 2, 8, 2, 700, "bf16", True, seed=29)
    lens = [700, 650]
    ref, w, bound, _ = c.reference(lens, 0, ALL)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    check(c.attend(lens, 0, ALL, stream=st), ref, bound)
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws, accum = H.alloc_window_workspace(c.desc, True), torch.zeros(2, 700, device="cuda")
    graph = torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=st):
        H.hill_window_attn_q4(c.desc, c.q, c.k4, c.v4, c.params, dev, 0, ALL, c.out, accum=accum, ws=ws)
    for lens in ([3, 0], [700, 650], [0, 0]):
        dev.copy_(torch.tensor(lens))
        graph.replay()
        torch.cuda.synchronize()
        ref, w, bound, _ = c.reference(lens, 0, ALL)
        check(c.out.cpu().numpy().astype(np.float64), ref, bound)


# ---------------------------------------------------------------- inserts
class Store:
    """A cache under inserts beside its plain form."""

    def __init__(self, H, B, Hkv, cap, kvh=False, q4=False, dtype="fp16", layout="head", seed=0):
        self.H, self.B, self.Hkv, self.cap, self.kvh, self.q4, self.dt = H, B, Hkv, cap, kvh, q4, DT[dtype]
        self.rows = (B, Hkv) if kvh else (B,)
        self.g = gen(seed)
        q = torch.zeros(B, Hkv, 128, dtype=self.dt, device="cuda")
        self.K, self.V = (torch.zeros(B, Hkv, cap, 128, dtype=self.dt, device="cuda") for _ in range(2))
        if layout == "token":
            self.K, self.V = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (self.K, self.V))
        self.desc = H.make_desc(q, self.K, self.V)
        if q4:
            self.k4, self.v4, self.params = H.alloc_q4(B, Hkv, cap, self.dt)
            self.params.fill_(7)
        self.seen = torch.zeros(self.rows, dtype=torch.int32, device="cuda")
        self.pos = torch.zeros(*self.rows, cap, dtype=torch.int32, device="cuda")
        self.accum = torch.zeros(*self.rows, cap, device="cuda")
        self.Kp, self.Vp = self.K.clone(), self.V.clone()

    def insert(self, T, sinks, recent, n_new=None, weight=False, new=None):
        H, B, Hkv = self.H, self.B, self.Hkv
        k, v = new if new else (torch.randn(B, T, Hkv, 128, generator=self.g, device="cuda").to(self.dt).transpose(1, 2) for _ in range(2))
        w = torch.rand(*self.rows, T, generator=self.g, device="cuda") if weight else None
        n = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device="cuda")
        slots = torch.full((*self.rows, T), 99, dtype=torch.int32, device="cuda")
        pos, accum, seen = self.pos.cpu().numpy().copy(), self.accum.cpu().numpy().copy(), self.seen.cpu().numpy().copy()
        if self.q4:
            H.hill_cache_insert_q4(self.desc, k, v, self.k4, self.v4, self.params, self.seen, self.pos, self.accum, sinks,
                                   recent, slots, n, w, self.kvh)
        else:
            H.hill_cache_insert(self.desc, k, v, self.K, self.V, self.seen, self.pos, self.accum, sinks, recent, slots, n,
                                w, self.kvh)
        H.hill_sync_status()
        got = slots.cpu().numpy()
        for r in np.ndindex(*self.rows):
            want, after = insert(seen[r], pos[r], accum[r], None if n_new is None else n_new[r[0]], T, sinks, recent,
                                 None if w is None else w.cpu().numpy()[r])
            np.testing.assert_array_equal(got[r], want, err_msg=str(r))
            seen[r] = after
            heads = [r[1]] if self.kvh else range(Hkv)
            for g in heads:
                at = torch.from_numpy(want[want >= 0]).long().cuda()
                self.Kp[r[0], g, at] = k[r[0], g, :len(at)]
                self.Vp[r[0], g, at] = v[r[0], g, :len(at)]
        np.testing.assert_array_equal(self.seen.cpu().numpy(), seen)
        np.testing.assert_array_equal(self.pos.cpu().numpy(), pos)
        np.testing.assert_array_equal(self.accum.cpu().numpy(), accum)
        if not self.q4:
            assert torch.equal(self.K, self.Kp) and torch.equal(self.V, self.Vp)

    def weigh(self, ties=False):
        x = torch.rand(*self.rows, self.cap, generator=self.g, device="cuda")
        self.accum.copy_((x * 7).round() / 7 - 0.5 if ties else x)

    def codes_right(self):
        """Every slot written since the start, bit for bit."""
        for i, (p, codes) in enumerate(((self.Kp, self.k4), (self.Vp, self.v4))):
            c, s, lo = encode(p.double().cpu().numpy(), to16(self.dt))
            for b, g in np.ndindex(self.B, self.Hkv):
                n = int(min(self.seen[(b, g) if self.kvh else b], self.cap))
                np.testing.assert_array_equal(codes[b, g, :n].cpu().numpy(), pack(c)[b, g, :n])
                np.testing.assert_array_equal(self.params[b, g, :n, 2 * i].double().cpu().numpy(), s[b, g, :n])
                np.testing.assert_array_equal(self.params[b, g, :n, 2 * i + 1].double().cpu().numpy(), lo[b, g, :n])
                assert torch.all(codes[b, g, n:] == 0) and torch.all(self.params[b, g, n:] == 7)


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("kvh", [False, True], ids=["seq", "kvh"])
@pytest.mark.parametrize("Hkv", [1, 3])
def test_insert(H, Hkv, kvh, q4, ties):
    s = Store(H, 3, Hkv, 101, kvh, q4, "bf16" if ties else "fp16", "token" if not q4 and ties else "head", seed=Hkv)
    s.insert(40, 4, 8, weight=True)             # free slots
    s.insert(1, 4, 8)
    s.insert(50, 4, 8, n_new=[50, 0, 17])       # different lengths, none among them
    s.weigh(ties)
    s.insert(30, 4, 8, n_new=[30, 5, 30])       # the rest of the free slots, and evictions
    for T, sinks, recent in [(1, 4, 8), (1, 0, 0), (2, 4, 90), (7, 0, 50), (60, 4, 8), (97, 4, 97), (101, 0, 0), (1, 60, 41)]:
        s.weigh(ties)
        s.insert(T, sinks, recent, weight=ties)
    if q4:
        s.codes_right()


@pytest.mark.parametrize("cap", [1, 2, 33, 1024, 4097, 49152, 49153, 60001])
def test_insert_sizes(H, cap):
    """One CTA's keys in shared memory and past it, one slot, chunks."""
    s = Store(H, 2, 1, cap, seed=cap)
    s.insert(cap, 0, 0)
    for T in sorted({1, min(cap, 2), min(cap, 333)}):
        s.weigh(ties=T == 2)
        s.insert(T, 0, 0)
    s.accum[:, ::2] = -0.0   # equal to 0
    s.accum[:, 1::2] = 0.0
    s.insert(max(1, cap // 3), 0, 0)


def test_insert_drops_what_has_no_place(H):
    """Positions that no insert made: fewer slots may go than are needed."""
    for T in (1, 5):
        s = Store(H, 1, 2, 16, seed=31)
        s.insert(16, 0, 0)
        s.pos.zero_()   # all claim to be the first token
        before = s.K.clone()
        slots = torch.zeros(1, T, dtype=torch.int32, device="cuda")
        new = torch.ones(1, 2, T, 128, dtype=torch.float16, device="cuda")
        H.hill_cache_insert(s.desc, new, new, s.K, s.V, s.seen, s.pos, s.accum, 4, 0, slots)
        with pytest.raises(H.HillError) as e:
            H.hill_sync_status()
        assert e.value.status == H.HILL_ERR_DEVICE
        assert torch.all(slots == -1) and torch.equal(s.K, before) and int(s.seen[0]) == 16 + T


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_rows_of_four_bits(H, dtype):
    """Constant, zero, tiny, huge and half-way rows, bit for bit; and what they are read back as."""
    dt = DT[dtype]
    top = 60000.0 if dtype == "fp16" else 1e30
    base = torch.randn(12, 128, generator=gen(37), device="cuda")
    base[0] = 0
    base[1] = 3.25
    base[2] = -7
    base[3] *= top / 8
    base[4, ::2], base[4, 1::2] = top, -top
    base[5] *= 6e-8 if dtype == "fp16" else 1e-39
    base[6] = torch.arange(128, device="cuda") * 0.25   # codes half-way between two
    base[7] = torch.arange(128, device="cuda") % 31 * 0.5
    base[8] = 1000 + base[8] * 1e-3
    base[9, 1:] = 0
    x = base.to(dt).view(1, 1, 12, 128)
    s = Store(H, 1, 1, 12, q4=True, dtype=dtype)
    s.insert(12, 0, 0, new=(x, -x))
    s.codes_right()
    lo, hi = torch.tensor([2], dtype=torch.int32, device="cuda"), torch.tensor([99], dtype=torch.int32, device="cuda")
    K, V = (torch.full((1, 12, 1, 128), 5.0, dtype=dt, device="cuda").transpose(1, 2) for _ in range(2))
    desc = H.make_desc(torch.zeros(1, 1, 128, dtype=dt, device="cuda"), K, V)
    H.hill_cache_read_q4(desc, s.k4, s.v4, s.params, lo, hi, 12, K, V)
    H.hill_sync_status()
    for got, p in ((K, x), (V, -x)):
        assert torch.all(got[:, :, :2] == 5)
        c, sc, mn = encode(p.double().cpu().numpy(), to16(dt))
        want = values(pack(c), sc, mn)[:, :, 2:]
        # one float32 rounding of the sum and one to 16 bits
        bits = 10 if dtype == "fp16" else 7
        tiny = 2.0 ** -25 if dtype == "fp16" else 2.0 ** -134
        err = np.abs(got[:, :, 2:].double().cpu().numpy() - want)
        assert np.all(err <= np.abs(want) * (2.0 ** -(bits + 1) + 2.0 ** -23) + np.abs(mn[:, :, 2:, None]) * 2.0 ** -23 + tiny)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kvh", [False, True], ids=["seq", "kvh"])
def test_a_decode_loop(H, bits, kvh):
    """BoundedCache over chunks and steps: evictions, weights and outputs as the plain forms have them."""
    B, Hq, Hkv, cap, dt = 2, 8, 2, 96, torch.float16
    cache = H.BoundedCache(B, Hq, Hkv, cap, dt, bits, sinks=4, recent=16, kvh=kvh, max_new=32)
    s = Store(H, B, Hkv, cap, kvh)   # for its plain caches
    g = gen(41)
    for step in range(24):
        T = 32 if step < 4 else 1 + step % 3
        q = torch.randn(B, Hq, 128, generator=g, device="cuda").to(dt)
        k, v = (torch.randn(B, Hkv, T, 128, generator=g, device="cuda").to(dt) for _ in range(2))
        pos, accum, seen = (x.cpu().numpy().copy() for x in (cache.pos, cache.accum, cache.seen))
        slots = cache.insert(k, v).cpu().numpy()
        for r in np.ndindex(*s.rows):   # on the loop's own weights
            want, _ = insert(seen[r], pos[r], accum[r], None, T, 4, 16)
            np.testing.assert_array_equal(slots[r], want)
            for h in ([r[1]] if kvh else range(Hkv)):
                at = torch.from_numpy(want).long().cuda()
                s.Kp[r[0], h, at], s.Vp[r[0], h, at] = k[r[0], h], v[r[0], h]
        np.testing.assert_array_equal(cache.pos.cpu().numpy(), pos)
        out = cache.attend(q).cpu().numpy().astype(np.float64)
        K64, V64 = s.Kp.double().cpu().numpy(), s.Vp.double().cpu().numpy()
        if bits == 4:
            K64, V64 = (values(pack(c), sc, lo) for c, sc, lo in (encode(x, to16(dt)) for x in (K64, V64)))
        ref, w, bound, wb = attn(q.double().cpu().numpy(), K64, V64, cache.seen.cpu().numpy(), 0, ALL, kvh)
        check(out, ref, bound)
        check(cache.accum.cpu().numpy().astype(np.float64), accum + w, wb + 2.0 ** -23 * (accum + w))
    H.hill_sync_status()


def test_the_example(H):
    from paper_2602_18750_gb300 import bounded
    for bits in (16, 4):
        us, out, cache = bounded.run(bits, slots=256, prompt=700, steps=5, batch=2, heads=8, kv_heads=2, chunk=128)
        assert us > 0 and torch.isfinite(out).all()
        # the prompt, one step before the capture, three and five replays (capturing runs nothing)
        assert int(cache.seen[0]) == 700 + 1 + 3 + 5
        # each attention adds one unit of weight per query head; what was evicted took its weight along
        assert 0 < float(cache.accum[0].sum()) < 8 * 20
