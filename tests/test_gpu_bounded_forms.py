"""Rows per KV head in every form of the attention of a bounded cache, the importance kernel's forms, reading 4-bit rows
back."""
import numpy as np
import pytest
import torch

from bounded_util import ALL, encode, pack, values
from test_gpu_bounded import DT, H, Case, Store, check, gen, to16  # noqa: F401 (H: the fixture)

pytestmark = pytest.mark.gpu


def attend_kvh(H, c, lens, sinks, window, kernels):  # noqa: F811
    """Without and with the weights; kernels: how many launches the first takes."""
    n0 = H.hill_kernel_launches()
    got = c.attend(lens, sinks, window, kvh=True)
    assert H.hill_kernel_launches() - n0 == kernels
    ref, w, bound, wb = c.reference(lens, sinks, window, kvh=True)
    check(got, ref, bound)
    accum = torch.full(w.shape, 0.125, device="cuda")
    n0 = H.hill_kernel_launches()
    check(c.attend(lens, sinks, window, accum, kvh=True), ref, bound)
    assert H.hill_kernel_launches() - n0 == kernels + 1
    check(accum.cpu().numpy().astype(np.float64), 0.125 + w, wb + 2.0 ** -23 * (0.125 + w))
    assert torch.all(accum.cpu()[torch.from_numpy(w == 0)] == 0.125)


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("G", [1, 4, 12, 32])
def test_many_rows_per_kv_head(H, G, q4):  # noqa: F811
    """320 rows, more than are scanned at a time, empty ones among them, over the list of tiles."""
    B, Hkv, cap = 20, 16, 90
    r = np.random.RandomState(11)
    lens = r.randint(0, cap + 5, (B, Hkv))
    lens[r.rand(B, Hkv) < 0.3] = 0
    lens[0, :3] = lens[-1, -4:] = 0
    lens[7] = 0
    c = Case(H, B, G * Hkv, Hkv, cap, "bf16", q4, seed=89)
    for sinks, window in [(0, ALL), (3, 40)]:
        attend_kvh(H, c, lens, sinks, window, 2)
    attend_kvh(H, c, lens * 0, 0, ALL, 2)


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("G", [1, 4, 12])
def test_long_rows_per_kv_head(H, G, q4):  # noqa: F811
    """77 rows of different lengths, each split over many warps."""
    B, Hkv, cap = 7, 11, 5000
    lens = np.random.RandomState(12).randint(0, cap + 1, (B, Hkv))
    lens[0, 0], lens[3, 3:7], lens[6, 10] = cap + 9, 0, 1
    c = Case(H, B, G * Hkv, Hkv, cap, "fp16", q4, seed=97)
    attend_kvh(H, c, lens, 0, ALL, 2)


def test_the_importance_of_many_short_rows(H):  # noqa: F811
    """Enough tokens that a warp takes all heads of its own: the unsplit form, with one and several heads."""
    B, Hkv, cap = 103, 16, 272
    r = np.random.RandomState(13)
    lens = r.randint(0, 40, (B, Hkv))
    lens[::9] = r.randint(0, cap + 1, lens[::9].shape)
    for G in (1, 2):
        c = Case(H, B, G * Hkv, Hkv, cap, "bf16", seed=101)
        attend_kvh(H, c, lens, 0, ALL, 2)


def test_a_graph_adds_the_weights(H):  # noqa: F811
    """Lengths change between the replays of a captured call, whose weights add up."""
    for q4 in (False, True):
        c = Case(H, 2, 8, 2, 700, "fp16", q4, seed=103)
        dev, accum = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 700, device="cuda")
        ws, graph, st = H.alloc_window_workspace(c.desc, True), torch.cuda.CUDAGraph(), torch.cuda.Stream()
        call, cache = (H.hill_window_attn_q4, (c.k4, c.v4, c.params)) if q4 else (H.hill_window_attn, (c.K, c.V))
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            call(c.desc, c.q, *cache, dev, 0, ALL, c.out, accum=accum, ws=ws)   # (nothing is held yet)
            with torch.cuda.graph(graph, stream=st):
                call(c.desc, c.q, *cache, dev, 0, ALL, c.out, accum=accum, ws=ws)
        torch.cuda.synchronize()
        total = error = 0.0
        for lens in ([3, 0], [700, 650], [0, 0], [64, 700]):
            dev.copy_(torch.tensor(lens))
            graph.replay()
            torch.cuda.synchronize()
            ref, w, bound, wb = c.reference(lens, 0, ALL)
            check(c.out.cpu().numpy().astype(np.float64), ref, bound)
            total, error = total + w, error + wb + 2.0 ** -23 * (total + w)
            check(accum.cpu().numpy().astype(np.float64), total, error)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_reading_rows_back(H, layout, dtype):  # noqa: F811
    """Several sequences and KV heads, a range of slots of its own for each, into both layouts."""
    B, Hkv, cap, dt = 4, 3, 101, DT[dtype]
    s = Store(H, B, Hkv, cap, q4=True, dtype=dtype, layout=layout, seed=107)
    s.insert(cap, 0, 0)
    s.codes_right()
    begin, end = [0, -7, 40, 90], [101, 33, 500, 12]
    lo, hi = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (begin, end))
    K, V = (torch.full((B, Hkv, cap, 128), 5.0, dtype=dt, device="cuda") for _ in range(2))
    if layout == "token":
        K, V = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (K, V))
    H.hill_cache_read_q4(s.desc, s.k4, s.v4, s.params, lo, hi, cap, K, V)
    H.hill_sync_status()
    for got, rows in ((K, s.Kp), (V, s.Vp)):
        c, scale, mn = encode(rows.double().cpu().numpy(), to16(dt))
        want = values(pack(c), scale, mn)
        got = got.double().cpu().numpy()
        for b in range(B):
            read = np.zeros(cap, bool)
            read[max(begin[b], 0):max(min(end[b], cap), 0)] = True
            assert np.all(got[b][:, ~read] == 5)
            # one float32 rounding of the sum and one to 16 bits
            bits = 10 if dtype == "fp16" else 7
            err = np.abs(got[b][:, read] - want[b][:, read])
            assert np.all(err <= np.abs(want[b][:, read]) * (2.0 ** -(bits + 1) + 2.0 ** -23)
                          + np.abs(mn[b][:, read, None]) * 2.0 ** -23 + 2.0 ** -25)
