"""What the calls over prompts and caches in pages refuse on the host, without a GPU, and the plain forms that their GPU
tests use."""
import ctypes

import numpy as np
import pytest

from paged_util import ALL, e4m3, importance, paged_rows, prompt, quantise, sees
from test_abi import FAKE, _desc


@pytest.fixture(scope="module")
def lib():
    from paper_2602_18750_gb300 import build, hill
    build.build()
    return hill.load()


def packed(**kw):
    from paper_2602_18750_gb300 import hill
    d = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, dtype=0, q_rows=100, k_rows=120, q_st=1024, q_sh=128,
             k_st=256, k_sh=128, v_st=256, v_sh=128)
    d.update(kw)
    return hill.hill_packed(**d)


def on_gpu():
    import torch
    return torch.cuda.is_available()


BAD_PACKED = [dict(batch=-1), dict(num_q_heads=7), dict(num_kv_heads=0), dict(dtype=2), dict(q_rows=-1), dict(k_rows=-1),
              dict(q_st=100), dict(k_sh=-8), dict(v_st=4), dict(head_dim=0)]
UNBUILT_PACKED = [dict(head_dim=64), dict(batch=513), dict(q_rows=(1 << 30) + 1), dict(k_rows=(1 << 30) + 1),
                  dict(q_rows=1 << 30, num_q_heads=512, num_kv_heads=512), dict(k_rows=1 << 30, num_q_heads=64, num_kv_heads=64)]


def test_prompt_attention_refusals(lib):
    from paper_2602_18750_gb300.hill import HILL_ERR_CUDA as CUDA, HILL_ERR_INVALID_ARG as INV, HILL_ERR_UNSUPPORTED as UNS, HILL_OK as OK

    def call(desc, **kw):
        a = dict(q=FAKE, k=FAKE, v=FAKE, qs=FAKE, ks=FAKE, sinks=4, window=64, out=FAKE, lse=FAKE)
        a.update(kw)
        return lib.hill_prompt_attn(ctypes.byref(desc) if desc is not None else None, *a.values(), None)

    assert call(None) == INV
    for bad in BAD_PACKED:
        assert call(packed(**bad)) == INV, bad
        assert lib.hill_prompt_workspace_bytes(ctypes.byref(packed(**bad))) == 0
    for bad in UNBUILT_PACKED:
        assert call(packed(**bad)) == UNS, bad
        assert lib.hill_prompt_workspace_bytes(ctypes.byref(packed(**bad))) == 0
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(qs=None), dict(ks=None), dict(out=None), dict(sinks=-1),
                dict(window=-1), dict(q=FAKE + 2), dict(k=FAKE + 8), dict(v=FAKE + 4), dict(out=FAKE + 8)):
        assert call(packed(), **bad) == INV, bad
    assert call(packed(batch=0)) == OK and call(packed(q_rows=0), q=None, out=None) == OK
    if not on_gpu():   # what is fine goes as far as the device
        assert call(packed()) == CUDA and call(packed(), lse=None) == CUDA
        assert call(packed(k_rows=0), k=None, v=None) == CUDA


def test_prompt_importance_refusals(lib):
    from paper_2602_18750_gb300.hill import HILL_ERR_CUDA as CUDA, HILL_ERR_INVALID_ARG as INV, HILL_ERR_UNSUPPORTED as UNS, HILL_OK as OK

    def call(desc, **kw):
        a = dict(q=FAKE, k=FAKE, lse=FAKE, qs=FAKE, ks=FAKE, sinks=4, window=64, newest=5, kvh=0, accum=FAKE, cap=100, ws=FAKE,
                 n=1 << 40)
        a.update(kw)
        return lib.hill_prompt_importance(ctypes.byref(desc) if desc is not None else None, *a.values(), None)

    assert call(None) == INV
    for bad in BAD_PACKED:
        assert call(packed(**bad)) == INV, bad
    for bad in UNBUILT_PACKED:
        assert call(packed(**bad)) == UNS, bad
    for bad in (dict(q=None), dict(k=None), dict(lse=None), dict(qs=None), dict(ks=None), dict(accum=None), dict(sinks=-1),
                dict(window=-1), dict(newest=-1), dict(cap=-1), dict(q=FAKE + 8), dict(k=FAKE + 2)):
        assert call(packed(), **bad) == INV, bad
    for nothing in (dict(batch=0), dict(q_rows=0), dict(k_rows=0)):
        assert call(packed(**nothing)) == OK
    if not on_gpu():
        assert call(packed()) == CUDA


def pages(**kw):
    from paper_2602_18750_gb300 import hill
    p = dict(k=FAKE, v=FAKE, scales=None, table=FAKE, pages=9, page=16, cols=4)
    p.update(kw)
    return hill.hill_pages(**p)


BAD_PAGES = [dict(k=None), dict(v=None), dict(table=None), dict(pages=-1), dict(page=0), dict(page=-16), dict(cols=-1),
             dict(k=FAKE + 8), dict(v=FAKE + 2), dict(scales=FAKE + 8)]
UNBUILT_PAGES = [dict(page=24), dict(page=1), dict(pages=(1 << 29)), dict(cols=1 << 27)]


def test_paged_refusals(lib):
    from paper_2602_18750_gb300 import hill
    from paper_2602_18750_gb300.hill import HILL_ERR_CUDA as CUDA, HILL_ERR_INVALID_ARG as INV, HILL_ERR_UNSUPPORTED as UNS, HILL_OK as OK

    def attend(desc, p, **kw):
        a = dict(lens=FAKE, sinks=4, window=64, kvh=0, accum=None, out=FAKE, ws=FAKE, n=1 << 40)
        q = kw.pop("q", FAKE)
        a.update(kw)
        return lib.hill_paged_attn(ctypes.byref(desc) if desc is not None else None, q,
                                   ctypes.byref(p) if p is not None else None, *a.values(), None)

    def rows(**kw):
        return hill.hill_rows(**{**dict(k=FAKE, v=FAKE, k_st=256, k_sh=128, v_st=256, v_sh=128, rows=5), **kw})

    def write(desc, p, r, starts=FAKE, begin=FAKE):
        ref = lambda x: ctypes.byref(x) if x is not None else None
        return lib.hill_paged_write(ref(desc), ref(p), ref(r), starts, begin, None)

    def read(desc, p, **kw):
        a = dict(begin=FAKE, end=FAKE, n=5, k=FAKE, v=FAKE)
        a.update(kw)
        return lib.hill_paged_read(ctypes.byref(desc) if desc is not None else None,
                                   ctypes.byref(p) if p is not None else None, *a.values(), None)

    for call in (attend, read, lambda d, p: write(d, p, rows())):
        assert call(None, pages()) == INV and call(_desc(), None) == INV
        assert call(_desc(head_dim=64), pages()) == UNS
        for bad in BAD_PAGES:
            assert call(_desc(), pages(**bad)) == INV, bad
        for bad in UNBUILT_PAGES:
            assert call(_desc(), pages(**bad)) == UNS, bad
    for bad in (dict(q=None), dict(lens=None), dict(out=None), dict(sinks=-1), dict(window=-1), dict(q=FAKE + 8), dict(out=FAKE + 4)):
        assert attend(_desc(), pages(), **bad) == INV, bad
    assert attend(_desc(capacity=80), pages()) == INV     # not what the table covers
    assert attend(_desc(batch=300, num_q_heads=8, num_kv_heads=8), pages(), kvh=1) == UNS
    assert write(_desc(), pages(), None) == INV
    for bad in (dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(k_st=100), dict(v_sh=-8), dict(rows=-1)):
        assert write(_desc(), pages(), rows(**bad)) == INV, bad
    assert write(_desc(), pages(), rows(), starts=None) == INV and write(_desc(), pages(), rows(), begin=None) == INV
    assert write(_desc(), pages(), rows(rows=0)) == OK and write(_desc(batch=0), pages(), rows()) == OK
    for bad in (dict(begin=None), dict(end=None), dict(n=-1), dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2)):
        assert read(_desc(), pages(), **bad) == INV, bad
    assert read(_desc(), pages(), n=0) == OK and read(_desc(), pages(cols=0)) == OK
    if not on_gpu():
        assert attend(_desc(), pages()) == CUDA and attend(_desc(), pages(scales=FAKE)) == CUDA
        assert write(_desc(), pages(), rows()) == CUDA and read(_desc(), pages()) == CUDA
        assert write(_desc(), pages(pages=0, k=None, v=None), rows()) == CUDA   # (no page is there: every row is dropped)


@pytest.mark.parametrize("count", [(1 << 29) - 1, 1 << 29, (1 << 30) - 1, (1 << 31) - 2, (1 << 31) - 1])
def test_pools_of_more_pages_than_are_numbered(lib, count):
    """(pages + 1) x KV heads is at most 2^30, up to the largest count that the field holds."""
    from paper_2602_18750_gb300 import hill
    from paper_2602_18750_gb300.hill import HILL_ERR_UNSUPPORTED as UNS
    p = lambda: ctypes.byref(pages(pages=count))
    rows = hill.hill_rows(k=FAKE, v=FAKE, k_st=256, k_sh=128, v_st=256, v_sh=128, rows=0)   # (nothing to do where it is not refused)
    fits = (count + 1) * 2 <= 1 << 30
    assert lib.hill_paged_write(ctypes.byref(_desc()), p(), ctypes.byref(rows), FAKE, FAKE, None) == (0 if fits else UNS)
    assert lib.hill_paged_read(ctypes.byref(_desc()), p(), FAKE, FAKE, 0, FAKE, FAKE, None) == (0 if fits else UNS)
    if not fits:
        assert lib.hill_paged_attn(ctypes.byref(_desc()), FAKE, p(), FAKE, 0, 5, 0, None, FAKE, FAKE, 1 << 40, None) == UNS


def test_reading_pages_into_one_place_is_refused(lib):
    """A descriptor of the pages, or any without strides of a cache, does not say where rows go."""
    from paper_2602_18750_gb300.hill import HILL_ERR_INVALID_ARG as INV, HILL_OK as OK
    read = lambda **kw: lib.hill_paged_read(ctypes.byref(_desc(**kw)), ctypes.byref(pages()), FAKE, FAKE, 0, FAKE, FAKE, None)
    assert read() == OK
    for stride in ("k_sb", "k_sh", "k_sn", "v_sb", "v_sh", "v_sn"):
        assert read(**{stride: 0}) == INV, stride
    assert read(batch=1, k_sb=0, v_sb=0) == OK and read(num_kv_heads=1, k_sh=0, v_sh=0) == OK
    assert read(capacity=1, k_sn=0, v_sn=0) == OK


# ---------------------------------------------------------------- the binding
def refused(f):
    with pytest.raises(ValueError):
        f()


def reaches_the_library(monkeypatch, f):
    class Library:
        def __getattr__(self, name):
            return lambda *a: seen.append(name) or 0

    from paper_2602_18750_gb300 import hill
    seen = []
    with monkeypatch.context() as m:
        m.setattr(hill, "_lib", Library())
        f()
    assert seen


def others(t):
    """What may not stand in t's place: another type, a view with gaps, another shape."""
    import torch
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] * 2, dtype=t.dtype)
    yield t.double()
    yield t.long() if t.dtype == torch.int32 else t.to(torch.int16)
    yield wide[..., ::2]
    yield wide


def test_binding_of_prompts(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2602_18750_gb300 import hill
    B, T, S, HQ, HKV = 2, 7, 9, 8, 2
    good = dict(q=torch.zeros(T, HQ, 128, dtype=torch.bfloat16), k=torch.zeros(S, HKV, 128, dtype=torch.bfloat16),
                v=torch.zeros(S, HKV, 128, dtype=torch.bfloat16), qs=torch.zeros(B + 1, dtype=torch.int32),
                ks=torch.zeros(B + 1, dtype=torch.int32), out=torch.zeros(T, HQ, 128, dtype=torch.bfloat16),
                lse=torch.zeros(T, HQ), accum=torch.zeros(B, 11))
    d = hill.make_packed(good["q"], good["k"], good["v"], B)
    assert (d.batch, d.num_q_heads, d.num_kv_heads, d.head_dim, d.dtype, d.q_rows, d.k_rows) == (B, HQ, HKV, 128, 1, T, S)
    for q, k, v in ((good["q"].float(), good["k"], good["v"]), (good["q"], good["k"].half(), good["v"]),
                    (good["q"], good["k"], good["v"][:-1]), (good["q"][0], good["k"], good["v"]),
                    (good["q"][..., :64], good["k"], good["v"]), (good["q"].transpose(1, 2), good["k"], good["v"])):
        refused(lambda: hill.make_packed(q, k, v, B))

    def attend(**kw):
        a = {**good, **kw}
        return lambda: hill.hill_prompt_attn(d, a["q"], a["k"], a["v"], a["qs"], a["ks"], 0, 5, a["out"], lse=a["lse"], stream=1)

    def weigh(kvh=False, **kw):
        a = {**good, **kw}
        return lambda: hill.hill_prompt_importance(d, a["q"], a["k"], a["lse"], a["qs"], a["ks"], 0, 5, 4, a["accum"], kvh=kvh, stream=1)

    for f in (attend(), attend(lse=None), attend(q=good["q"].data_ptr()), weigh(), weigh(True, accum=torch.zeros(B, HKV, 11))):
        reaches_the_library(monkeypatch, f)
    for name in ("q", "k", "v", "qs", "ks", "out", "lse"):
        for bad in others(good[name]):
            refused(attend(**{name: bad}))
            if name not in ("v", "out"):
                refused(weigh(**{name: bad}))
    refused(weigh(True))
    for bad in list(others(good["accum"]))[:3] + [torch.zeros(B + 1, 11)]:
        refused(weigh(accum=bad))


def test_binding_of_pages(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2602_18750_gb300 import hill
    B, HQ, HKV, page, n = 2, 8, 2, 16, 5
    K = torch.zeros(n, HKV, page, 128, dtype=torch.float16)
    codes, scales = torch.zeros(n, HKV, page, 128, dtype=torch.float8_e4m3fn), torch.zeros(n, HKV, page, 2)
    table, lens = torch.zeros(B, 3, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    q, out, accum = torch.zeros(B, HQ, 128, dtype=torch.float16), torch.zeros(B, HQ, 128), torch.zeros(B, 48)
    for bad in ((K, K[:, :, :, :64], table, None), (K[0], K[0], table, None), (K, K.bfloat16(), table, None),
                (K.transpose(0, 1), K.transpose(0, 1), table, None), (K.float(), K.float(), table, None),
                (K, K, table.long(), None), (K, K, table[0], None), (K, K, table[:, ::2], None), (K, K, table, scales),
                (codes, codes, table, None), (codes, codes, table, scales[..., :1]), (codes, codes, table, scales.double())):
        refused(lambda: hill.make_pages(*bad))
    for pool, sc in ((K, None), (codes, scales), (codes.view(torch.uint8), scales)):
        p = hill.make_pages(pool, pool, table, sc)
        d = hill.make_desc_paged(q, p)
        assert (d.batch, d.num_q_heads, d.num_kv_heads, d.capacity) == (B, HQ, HKV, 48)
        refused(lambda: hill.make_desc_paged(q[:1], p))
        refused(lambda: hill.make_desc_paged(q.float(), p))
        if sc is None:
            refused(lambda: hill.make_desc_paged(q.bfloat16(), p))
        attend = lambda **kw: (lambda a=dict(dict(q=q, lens=lens, out=out, accum=accum), **kw): hill.hill_paged_attn(
            d, a["q"], p, a["lens"], 0, 5, a["out"], accum=a["accum"], stream=1))
        reaches_the_library(monkeypatch, attend())
        for name, t in (("lens", lens), ("out", out), ("accum", accum)):
            for bad in list(others(t))[:3]:
                refused(attend(**{name: bad}))
        refused(attend(q=q.bfloat16()))
        new, st, bg = torch.zeros(4, HKV, 128, dtype=torch.float16), torch.zeros(B + 1, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
        write = lambda k=new, v=new, s=st, b=bg: (lambda: hill.hill_paged_write(d, p, k, v, s, b, stream=1))
        reaches_the_library(monkeypatch, write())
        for bad in (new.bfloat16(), new[:, :1], new[..., :64], new.transpose(0, 2), new[0]):
            refused(write(k=bad, v=bad))
            refused(write(v=bad))
        for bad in others(st):
            refused(write(s=bad))
        for bad in others(bg):
            refused(write(b=bad))
        cache = torch.zeros(B, HKV, 48, 128, dtype=torch.float16)
        read = lambda lo, hi: (lambda: hill.hill_paged_read(d, p, lo, hi, 3, cache, cache, stream=1))
        reaches_the_library(monkeypatch, read(bg, bg))
        for bad in list(others(bg))[:3]:
            refused(read(bad, bg))
            refused(read(bg, bad))
    other = hill.make_desc(torch.zeros(3, HQ, 128, dtype=torch.float16), torch.zeros(3, HKV, 48, 128, dtype=torch.float16))
    refused(lambda: hill.hill_paged_read(other, p, bg, bg, 3, cache, cache, stream=1))


@pytest.mark.parametrize("e4m3", [False, True], ids=["16bit", "e4m3"])
def test_binding_of_pages_holds_shapes(monkeypatch, e4m3):
    """Every tensor of a call over pages has the shape that the pages, the descriptor and kvh give it."""
    torch = pytest.importorskip("torch")
    from paper_2602_18750_gb300 import hill
    B, HQ, HKV, page, n, cap, f16 = 2, 8, 4, 16, 5, 48, torch.float16
    pool = torch.zeros(n, HKV, page, 128, dtype=torch.uint8 if e4m3 else f16)
    p = hill.make_pages(pool, pool, torch.zeros(B, 3, dtype=torch.int32), torch.zeros(n, HKV, page, 2) if e4m3 else None)
    q, ints = torch.zeros(B, HQ, 128, dtype=f16), lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    d = hill.make_desc_paged(q, p)
    for kvh, rows in ((False, (B,)), (True, (B, HKV))):
        good = dict(lens=ints(*rows), out=torch.zeros(B, HQ, 128), accum=torch.zeros(*rows, cap))

        def attend(**kw):
            a = {**good, **kw}
            return lambda: hill.hill_paged_attn(d, q, p, a["lens"], 0, 5, a["out"], accum=a["accum"], kvh=kvh, stream=1)

        reaches_the_library(monkeypatch, attend())
        reaches_the_library(monkeypatch, attend(accum=None))
        reaches_the_library(monkeypatch, attend(lens=good["lens"].data_ptr(), accum=good["accum"].data_ptr()))
        for name, t in good.items():
            for bad in others(t):
                refused(attend(**{name: bad}))
        other = (B, HKV) if rows == (B,) else (B,)
        for bad in (dict(lens=ints(*other)), dict(lens=ints(B + 1)), dict(accum=torch.zeros(*other, cap)),
                    dict(accum=torch.zeros(*rows, cap - 1)), dict(out=torch.zeros(B, HKV, 128)), dict(out=torch.zeros(B, HQ * 128))):
            refused(attend(**bad))

    strided = torch.zeros(B, cap, HKV, 128, dtype=f16).transpose(1, 2)
    caches = (torch.zeros(B, HKV, cap, 128, dtype=f16), strided, torch.zeros(B, HKV, cap, 136, dtype=f16)[..., :128])
    read = lambda desc, K, V, lo=ints(B), hi=ints(B): (lambda: hill.hill_paged_read(desc, p, lo, hi, 3, K, V, stream=1))
    for K in caches:
        for V in caches:
            own = hill.make_desc(q, K, V)
            reaches_the_library(monkeypatch, read(own, K, V))
            reaches_the_library(monkeypatch, read(own, K.data_ptr(), V.data_ptr()))
            reaches_the_library(monkeypatch, read(d, K, V))    # the caches say how they lie
            for bad in caches:
                if bad is not V:
                    refused(read(own, K, bad))
                if bad is not K:
                    refused(read(own, bad, V))
    K, V = caches[:2]
    own = hill.make_desc(q, K, V)
    for bad in (K.bfloat16(), K.float(), K[:1], K[:, :2], K[:, :, :-1], K[..., :64], K[0], torch.zeros(B, HKV, cap + 16, 128, dtype=f16)):
        for desc in (own, d):
            refused(read(desc, bad, V))
            refused(read(desc, K, bad))
    for bad in others(ints(B)):
        refused(read(own, K, V, lo=bad))
        refused(read(own, K, V, hi=bad))
    refused(read(own, K, V, lo=ints(B + 1)))
    one = torch.zeros(1, 1, cap, 128, dtype=f16)      # dimensions of one element may have any stride
    p1 = hill.make_pages(pool[:, :1].contiguous(), pool[:, :1].contiguous(), ints(1, 3), p.tensors[3][:, :1].contiguous() if e4m3 else None)
    d1 = hill.make_desc(torch.zeros(1, HQ, 128, dtype=f16), one, one)
    reaches_the_library(monkeypatch, lambda: hill.hill_paged_read(d1, p1, ints(1), ints(1), 3, one.as_strided(one.shape, (8, 16, 128, 1)), one, stream=1))


def test_reading_pages_takes_the_caches_strides(monkeypatch):
    """With a descriptor of the pages the rows go where the caches have them; the descriptor itself stays as it is."""
    torch = pytest.importorskip("torch")
    from paper_2602_18750_gb300 import hill
    pool = torch.zeros(5, 2, 16, 128, dtype=torch.bfloat16)
    p = hill.make_pages(pool, pool, torch.zeros(3, 4, dtype=torch.int32))
    d = hill.make_desc_paged(torch.zeros(3, 8, 128, dtype=torch.bfloat16), p)
    K, V = torch.zeros(3, 2, 64, 128, dtype=torch.bfloat16), torch.zeros(3, 64, 2, 128, dtype=torch.bfloat16).transpose(1, 2)
    at, seen = torch.zeros(3, dtype=torch.int32), []

    class Library:
        def hill_paged_read(self, desc, *a):
            seen.append(((desc.k_sb, desc.k_sh, desc.k_sn), (desc.v_sb, desc.v_sh, desc.v_sn), desc.capacity))
            return 0

    monkeypatch.setattr(hill, "_lib", Library())
    hill.hill_paged_read(d, p, at, at, 3, K, V, stream=1)
    assert seen == [(K.stride()[:3], V.stride()[:3], 64)] and (d.k_sb, d.k_sn, d.v_sh) == (0, 0, 0)


# ---------------------------------------------------------------- the plain forms themselves
def test_plain_prompt_is_softmax_over_what_is_seen():
    torch = pytest.importorskip("torch")
    r = np.random.RandomState(0)
    seqs, Hq, Hkv = [(5, 9), (3, 3), (4, 0), (6, 4)], 4, 2
    qs = np.cumsum([0] + [n for n, _ in seqs])
    ks = np.cumsum([0] + [m for _, m in seqs])
    q, k, v = r.randn(qs[-1], Hq, 128), r.randn(ks[-1], Hkv, 128), r.randn(ks[-1], Hkv, 128)
    for sinks, window in [(0, ALL), (2, 3), (0, 0)]:
        out, lse, _, _ = prompt(q, k, v, qs, ks, sinks, window, 2.0 ** -8)
        w, _ = importance(q, k, lse, qs, ks, sinks, window, ALL, 10, True)
        for b, (n, m) in enumerate(seqs):
            for i in range(n):
                pos = i + m - n
                at = [j for j in range(m) if j <= pos and (j < sinks or j > pos - window)]
                t = qs[b] + i
                if not at:
                    assert np.all(out[t] == 0) and np.all(np.isneginf(lse[t]))
                    continue
                rows = ks[b] + np.array(at)
                want = torch.nn.functional.scaled_dot_product_attention(
                    torch.from_numpy(q[t])[:, None], torch.from_numpy(k[rows].transpose(1, 0, 2)).repeat_interleave(2, 0),
                    torch.from_numpy(v[rows].transpose(1, 0, 2)).repeat_interleave(2, 0))[:, 0]
                np.testing.assert_allclose(out[t], want.numpy(), atol=1e-12)
            rows = [i for i in range(n) if sees(n, m, sinks, window)[i].any()] if m else []
            np.testing.assert_allclose(w[b].sum(), Hq * len(rows), atol=1e-9)   # every query that sees something gives 1 per head


def test_plain_e4m3_is_torchs():
    torch = pytest.importorskip("torch")
    x = torch.randn(4000, generator=torch.Generator().manual_seed(1)) * torch.exp2(torch.randint(-12, 9, (4000,)).float())
    x = x.clamp(-448, 448)
    assert np.array_equal(e4m3(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())
    rows = torch.randn(50, 128, generator=torch.Generator().manual_seed(2)).bfloat16()
    codes, scale = quantise(rows.double().numpy())
    assert np.abs(codes).max(1).min() == 448
    assert np.all(np.abs(codes * scale[:, None] - rows.double().numpy()) <= 2.0 ** -4 * np.abs(rows.double().numpy()) + 2.0 ** -9 * scale[:, None])


def test_plain_pages():
    pool = np.arange(4 * 2 * 3).reshape(4, 2, 3).astype(float)
    rows = paged_rows(pool, np.array([[2, -1], [0, 3]]), 6)
    assert rows.shape == (2, 2, 6)
    assert np.array_equal(rows[0, 1], [15, 16, 17, 0, 0, 0]) and np.array_equal(rows[1, 0], [0, 1, 2, 18, 19, 20])
