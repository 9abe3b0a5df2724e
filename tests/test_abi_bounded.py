"""What the calls of a bounded cache refuse on the host, without a GPU, and the plain forms that their GPU tests use."""
import ctypes

import numpy as np
import pytest

from bounded_util import ALL, attn, encode, insert, pack, values
from test_abi import FAKE, _desc


@pytest.fixture(scope="module")
def lib():
    from paper_2602_18750_gb300 import build, hill
    build.build()
    return hill.load()


def test_attention_refusals(lib):
    from paper_2602_18750_gb300.hill import HILL_ERR_CUDA as CUDA, HILL_ERR_INVALID_ARG as INV, HILL_ERR_UNSUPPORTED as UNS

    def call(desc=None, q4=False, **kw):
        a = dict(q=FAKE, k=FAKE, v=FAKE, params=FAKE, lens=FAKE, sinks=4, window=64, kvh=0, accum=None, out=FAKE,
                 ws=FAKE, n=1 << 40)
        a.update(kw)
        d = ctypes.byref(desc) if desc is not None else None
        mid = (a["q"], a["k"], a["v"]) + ((a["params"],) if q4 else ())
        f = lib.hill_window_attn_q4 if q4 else lib.hill_window_attn
        return f(d, *mid, a["lens"], a["sinks"], a["window"], a["kvh"], a["accum"], a["out"], a["ws"], a["n"], None)

    for q4 in (False, True):
        assert call(None, q4) == INV
        for bad in (dict(q=None), dict(k=None), dict(v=None), dict(lens=None), dict(out=None), dict(sinks=-1),
                    dict(window=-1), dict(q=FAKE + 2), dict(k=FAKE + 8), dict(v=FAKE + 8), dict(out=FAKE + 4)):
            assert call(_desc(), q4, **bad) == INV, bad
        assert call(_desc(head_dim=64), q4) == UNS
        assert call(_desc(batch=513), q4) == UNS
        assert call(_desc(batch=300, num_q_heads=8, num_kv_heads=8), q4, kvh=1) == UNS   # over 2048 rows
        # tiles are numbered in 32 bits
        assert call(_desc(batch=512, num_q_heads=4096, num_kv_heads=4096, capacity=131072), q4) == UNS
        import torch
        if not torch.cuda.is_available():   # what is fine goes as far as the device
            assert call(_desc(), q4) == CUDA
            assert call(_desc(batch=256, num_q_heads=8, num_kv_heads=8), q4, kvh=1) == CUDA
    assert call(_desc(), True, params=None) == INV
    assert call(_desc(), True, params=FAKE + 8) == INV
    assert lib.hill_window_workspace_bytes(ctypes.byref(_desc(head_dim=64)), 1) == 0


def test_insert_refusals(lib):
    from paper_2602_18750_gb300 import hill
    from paper_2602_18750_gb300.hill import HILL_ERR_CUDA as CUDA, HILL_ERR_INVALID_ARG as INV, HILL_OK as OK

    def rows(**kw):
        a = dict(k=FAKE, v=FAKE, k_sb=1024, k_sh=512, k_sn=128, v_sb=1024, v_sh=512, v_sn=128, max_new=4, count=None,
                 weight=None)
        a.update(kw)
        return hill.hill_new_rows(**a)

    def call(desc, n, q4=False, **kw):
        a = dict(k=FAKE, v=FAKE, params=FAKE, seen=FAKE, pos=FAKE, accum=FAKE, sinks=4, recent=8, kvh=0, slots=FAKE)
        a.update(kw)
        cache = (a["k"], a["v"]) + ((a["params"],) if q4 else ())
        f = lib.hill_cache_insert_q4 if q4 else lib.hill_cache_insert
        return f(ctypes.byref(desc) if desc is not None else None, ctypes.byref(n) if n is not None else None, *cache,
                 a["seen"], a["pos"], a["accum"], a["sinks"], a["recent"], a["kvh"], a["slots"], None)

    for q4 in (False, True):
        assert call(None, rows(), q4) == INV
        assert call(_desc(), None, q4) == INV
        for bad in (dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(seen=None), dict(pos=None), dict(accum=None),
                    dict(slots=None), dict(sinks=-1), dict(recent=-1), dict(sinks=57), dict(sinks=61, recent=0),
                    dict(sinks=0, recent=65), dict(sinks=1 << 30, recent=1 << 30)):
            assert call(_desc(), rows(), q4, **bad) == INV, bad
        for bad in (dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(k_sn=100), dict(v_sb=-8), dict(max_new=-1),
                    dict(max_new=61)):
            assert call(_desc(), rows(**bad), q4) == INV, bad
        assert call(_desc(), rows(max_new=0), q4) == OK   # nothing to do
        assert call(_desc(batch=0), rows(), q4) == OK
    assert call(_desc(), rows(), True, params=None) == INV
    d = _desc()
    read = lambda **kw: lib.hill_cache_read_q4(ctypes.byref(d), *{**dict(k4=FAKE, v4=FAKE, p=FAKE, b=FAKE, e=FAKE, n=1, k=FAKE, v=FAKE), **kw}.values(), None)
    for bad in (dict(k4=None), dict(v4=None), dict(p=None), dict(b=None), dict(e=None), dict(n=-1), dict(k=None),
                dict(v=None), dict(k=FAKE + 8), dict(p=FAKE + 4)):
        assert read(**bad) == INV, bad
    assert read(n=0) == OK
    import torch
    if not torch.cuda.is_available():
        assert call(_desc(), rows()) == CUDA and read() == CUDA


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    from paper_2602_18750_gb300 import hill
    q, k4 = torch.zeros(2, 8, 128, dtype=torch.float16), torch.zeros(2, 2, 10, 64, dtype=torch.uint8)
    d = hill.make_desc_q4(q, k4)
    assert (d.batch, d.num_q_heads, d.num_kv_heads, d.head_dim, d.capacity) == (2, 8, 2, 128, 10)
    with pytest.raises(ValueError):
        hill.make_desc_q4(q, k4[:1])
    with pytest.raises(ValueError):
        hill.make_desc_q4(q.float(), k4)
    with pytest.raises(ValueError):
        hill.make_desc_q4(q, torch.zeros(2, 2, 10, 128, dtype=torch.uint8))
    new = torch.zeros(2, 2, 3, 128, dtype=torch.float16)
    for bad in (new.bfloat16(), new[:, :1], new[..., :64], new.transpose(2, 3)):
        with pytest.raises(ValueError):
            hill.hill_cache_insert(d, new, bad, None, None, None, None, None, 0, 0, None)
    with pytest.raises(ValueError):
        hill.BoundedCache(1, 8, 2, 16, bits=8, device="cpu")


# ---------------------------------------------------------------- the plain forms themselves
def test_plain_attention_is_softmax_over_what_is_seen():
    torch = pytest.importorskip("torch")
    r = np.random.RandomState(0)
    q, K, V = r.randn(2, 4, 128), r.randn(2, 2, 50, 128), r.randn(2, 2, 50, 128)
    for sinks, window in [(0, ALL), (3, 10), (0, 0), (60, 1)]:
        out, w, _, _ = attn(q, K, V, [50, 7], sinks, window)
        for b, n in enumerate([50, 7]):
            seen = torch.zeros(50, dtype=torch.bool)
            seen[:n] = (torch.arange(n) < sinks) | (torch.arange(n) >= n - window)
            want = torch.nn.functional.scaled_dot_product_attention(
                torch.from_numpy(q[b])[:, None], torch.from_numpy(K[b]).repeat_interleave(2, 0),
                torch.from_numpy(V[b]).repeat_interleave(2, 0), attn_mask=seen[None, None])[:, 0]
            if not seen.any():
                want = torch.zeros(4, 128)
            np.testing.assert_allclose(out[b], want.numpy(), atol=1e-12)
            np.testing.assert_allclose(w[b].sum(), 4.0 if seen.any() else 0.0, atol=1e-12)
            assert np.all(w[b][~seen.numpy()] == 0)


def test_plain_insert_keeps_the_heaviest():
    r = np.random.RandomState(1)
    for _ in range(50):
        cap, t, sinks, recent = 20, r.randint(1, 9), r.randint(0, 4), r.randint(0, 8)
        seen = r.randint(0, 60)
        pos, accum = np.zeros(cap, np.int32), r.rand(cap).round(1)
        pos[:] = r.permutation(max(seen, cap))[:cap]
        old = accum.copy(), pos.copy()
        slots, after = insert(seen, pos, accum, None, t, sinks, recent)
        assert after == seen + t and len(set(slots)) == t and all(accum[s] == 0 for s in slots)
        gone = [s for s in slots if s < min(seen, cap)]
        for j in range(min(seen, cap)):
            if j not in gone and sinks <= old[1][j] < seen + t - recent:
                assert all((old[0][j], -j) > (old[0][s], -s) or old[0][j] > old[0][s] for s in gone)
        assert all(sinks <= old[1][s] < seen + t - recent for s in gone)


def test_plain_rows_of_four_bits():
    x = np.random.RandomState(2).randn(5, 128)
    f16 = lambda v: np.asarray(v).astype(np.float16).astype(np.float64)
    x = f16(x)
    c, s, lo = encode(x, f16)
    err = np.abs(values(pack(c), s, lo) - x)
    assert np.all(err <= 0.5 * s[:, None] * (1 + 2.0 ** -7)) and c.min() == 0 and c.max() == 15
