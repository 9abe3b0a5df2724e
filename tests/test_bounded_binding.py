"""What the binding of a bounded cache refuses before a call: tensors that would be read as another type or layout."""
import pytest

torch = pytest.importorskip("torch")

from paper_2602_18750_gb300 import hill  # noqa: E402

B, HQ, HKV, CAP, T = 2, 8, 2, 10, 3


def refused(f):
    with pytest.raises(ValueError):
        f()


def reaches_the_library(monkeypatch, f):
    """The call gets as far as the library, here one that takes everything."""
    class Library:
        def __getattr__(self, name):
            return lambda *a: seen.append(name) or 0

    seen = []
    monkeypatch.setattr(hill, "_lib", Library())
    f()
    monkeypatch.undo()
    assert seen


def others(t):
    """What may not stand in t's place: other types, and a view with gaps."""
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] * 2, dtype=t.dtype)
    yield t.double()
    yield t.long() if t.dtype == torch.int32 else t.half()
    yield wide[..., ::2]


def test_attention(monkeypatch):
    q, out = torch.zeros(B, HQ, 128, dtype=torch.float16), torch.zeros(B, HQ, 128)
    K = torch.zeros(B, HKV, CAP, 128, dtype=torch.float16)
    k4, v4, params = hill.alloc_q4(B, HKV, CAP, device="cpu")
    lens, accum = torch.zeros(B, dtype=torch.int32), torch.zeros(B, CAP)
    d, d4 = hill.make_desc(q, K, K), hill.make_desc_q4(q, k4)

    def calls(lens=lens, out=out, accum=accum):
        yield lambda: hill.hill_window_attn(d, q, K, K, lens, 0, 5, out, accum=accum, stream=1)
        yield lambda: hill.hill_window_attn_q4(d4, q, k4, v4, params, lens, 0, 5, out, accum=accum, stream=1)

    for good in ({}, {"accum": None}, {"lens": lens.data_ptr()}):   # (pointers are taken as they are)
        for f in calls(**good):
            reaches_the_library(monkeypatch, f)
    for name, t in (("lens", lens), ("out", out), ("accum", accum)):
        for bad in others(t):
            for f in calls(**{name: bad}):
                refused(f)


def test_inserts(monkeypatch):
    new = torch.zeros(B, HKV, T, 128, dtype=torch.float16)
    q, K = torch.zeros(B, HQ, 128, dtype=torch.float16), torch.zeros(B, HKV, CAP, 128, dtype=torch.float16)
    k4, v4, params = hill.alloc_q4(B, HKV, CAP, device="cpu")
    desc = hill.make_desc(q, K, K)
    for kvh in (False, True):
        rows = (B, HKV) if kvh else (B,)
        good = dict(seen=torch.zeros(rows, dtype=torch.int32), pos=torch.zeros(*rows, CAP, dtype=torch.int32),
                    accum=torch.zeros(*rows, CAP), slots=torch.zeros(*rows, T, dtype=torch.int32),
                    n_new=torch.zeros(B, dtype=torch.int32), w_new=torch.zeros(*rows, T))

        def calls(**kw):
            a = {**good, **kw}
            s, opt = (a["seen"], a["pos"], a["accum"], 0, 0, a["slots"]), (a["n_new"], a["w_new"], kvh, 1)
            yield lambda: hill.hill_cache_insert(desc, new, new, K, K, *s, *opt)
            yield lambda: hill.hill_cache_insert_q4(desc, new, new, k4, v4, params, *s, *opt)

        for fine in ({}, {"n_new": None}, {"w_new": None}, {"seen": good["seen"].data_ptr()}):
            for f in calls(**fine):
                reaches_the_library(monkeypatch, f)
        for name, t in good.items():
            for bad in others(t):
                for f in calls(**{name: bad}):
                    refused(f)
        for name, bad in (("n_new", torch.zeros(B - 1, dtype=torch.int32)), ("w_new", torch.zeros(*rows, T + 1)),
                          ("w_new", torch.zeros(T))):
            for f in calls(**{name: bad}):
                refused(f)
    lo = torch.zeros(B, dtype=torch.int32)
    read = lambda lo, hi: lambda: hill.hill_cache_read_q4(desc, k4, v4, params, lo, hi, CAP, K, K, stream=1)
    reaches_the_library(monkeypatch, read(lo, lo))
    for bad in others(lo):
        refused(read(bad, lo))
        refused(read(lo, bad))


def test_codes_of_a_descriptor():
    q, k4 = torch.zeros(B, HQ, 128, dtype=torch.float16), torch.zeros(B, HKV, CAP, 64, dtype=torch.uint8)
    hill.make_desc_q4(q, k4)
    refused(lambda: hill.make_desc_q4(q, k4.short()))
    refused(lambda: hill.make_desc_q4(q, torch.zeros(B, HKV, CAP + 1, 64, dtype=torch.uint8)[:, :, 1:]))
    refused(lambda: hill.make_desc_q4(q, torch.zeros(B, CAP, HKV, 64, dtype=torch.uint8).transpose(1, 2)))


def test_queries_of_another_type(monkeypatch):
    monkeypatch.setattr(hill, "alloc_window_workspace", lambda *a: torch.zeros(1, dtype=torch.uint8))
    for bits in (16, 4):
        for dtype, bad in ((torch.float16, torch.bfloat16), (torch.bfloat16, torch.float16)):
            cache = hill.BoundedCache(B, HQ, HKV, CAP, dtype, bits, device="cpu")
            q = torch.zeros(B, HQ, 128, dtype=dtype)
            for x in (q.to(bad), q.float(), q[:, :4], q[:1]):
                refused(lambda: cache.attend(x))
            with monkeypatch.context() as m:
                reaches_the_library(m, lambda: cache.attend(q, stream=1))


def test_a_cache_without_room_for_what_is_to_stay(monkeypatch):
    """sinks + max(recent, max_new) slots are needed: said when the cache is made, not by its first insert."""
    monkeypatch.setattr(hill, "alloc_window_workspace", lambda *a: torch.zeros(1, dtype=torch.uint8))
    for bits in (16, 4):
        make = lambda **kw: hill.BoundedCache(B, HQ, HKV, 32, bits=bits, device="cpu", **kw)
        make(sinks=4, recent=28, max_new=28)
        for bad in (dict(max_new=29), dict(recent=29), dict(sinks=32), dict(sinks=-1), dict(recent=-1), dict(max_new=-1)):
            refused(lambda: make(**bad))
