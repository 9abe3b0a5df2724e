"""Values that are not finite where they are seen: the attention of a bounded cache answers with values that are not
finite either, whatever form the call takes, and leaves the other heads alone."""
import numpy as np
import pytest
import torch

from bounded_util import ALL
from test_gpu_bounded import H, Case, Store, check, gen  # noqa: F401 (H: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf")], ids=["nan", "inf"])
@pytest.mark.parametrize("form", ["clusters", "list"])
@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (12, 2), (32, 1)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_what_is_seen_shows(H, heads, q4, form, bad):  # noqa: F811
    """Sequence 0: a query head; 1: a key row; 2: a value row (one channel of it, in 16 bits)."""
    Hq, Hkv = heads
    G, g = Hq // Hkv, Hkv - 1
    B, cap, kernels = (4, 400, 1) if form == "clusters" else (160, 150, 2)
    c = Case(H, B, Hq, Hkv, cap, "fp16", q4, seed=61)
    lens = np.random.RandomState(8).randint(0, cap + 1, B)
    lens[:3] = cap
    lens[3] = 0
    c.q[1, :, 0] = c.q[1, :, 0].abs() + 1   # an infinite key channel is then +infinity in every head's logit
    ref, w, bound, wb = c.reference(lens, 0, ALL)
    hit, whole = np.zeros(ref.shape, bool), slice(g * G, (g + 1) * G)
    c.q[0, 1, 3] = bad
    hit[0, 1] = True
    hit[1, whole] = True
    if q4:
        c.params[1, g, 77, 0] = bad
        c.params[2, g, 77, 3] = bad
        hit[2, whole] = True
    else:
        c.K[1, g, 77, 0] = bad
        c.V[2, g, 77, 5] = bad
        hit[2, whole, 5] = True
    for weights in (False, True):
        accum = torch.full((B, cap), 0.5, device="cuda") if weights else None
        n0 = H.hill_kernel_launches()
        got = c.attend(lens, 0, ALL, accum)
        assert H.hill_kernel_launches() - n0 == kernels + weights
        assert not np.isfinite(got[hit]).any()
        check(got[~hit], ref[~hit], bound[~hit])
    accum = accum.cpu().numpy().astype(np.float64)
    assert np.isnan(accum[:2]).all()   # (every slot of these is seen)
    check(accum[2:], 0.5 + w[2:], wb[2:] + 2.0 ** -23 * (0.5 + w[2:]))


@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("B", [4, 160])
def test_rows_with_nothing_to_see_stay_zero(H, q4, B):  # noqa: F811
    """Zeros only where nothing is seen, even with a query that is not finite."""
    c = Case(H, B, 8, 2, 150, "bf16", q4, seed=67)
    c.q[:, 0] = float("nan")
    lens = [0, 150] * (B // 2)
    for sinks, window in [(0, ALL), (0, 0)]:
        accum = torch.full((B, 150), 0.25, device="cuda")
        got = c.attend(lens, sinks, window, accum)
        assert (got[::2] == 0).all() and torch.all(accum[::2] == 0.25)
        if window:
            assert np.isnan(got[1::2, 0]).all() and np.isfinite(got[1::2, 1:]).all() and torch.isnan(accum[1::2]).all()
        else:
            assert (got == 0).all() and torch.all(accum == 0.25)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), 3.3e38], ids=["nan", "inf", "-inf", "far"])
def test_new_rows_that_are_not_finite(H, bad, dtype):  # noqa: F811
    """In 4 bits such a row stands for no finite value, whichever channel was not; the others are as ever.  So does one
    whose max - min float32 does not hold."""
    T = 40
    for at in (0, 77, 127):
        s = Store(H, 1, 2, T, q4=True, dtype=dtype, seed=113)
        k, v = (torch.randn(1, 2, T, 128, device="cuda", generator=gen(114)).to(s.dt) for _ in range(2))
        s.insert(T, 0, 0, new=(k, v))
        clean = [x.clone() for x in (s.k4, s.v4, s.params)]
        k[0, 0, 3, at] = v[0, 1, 8, at] = bad
        if bad == 3.3e38:
            k[0, 0, 3, at ^ 1] = v[0, 1, 8, at ^ 1] = -bad
        s.seen.zero_()
        slots = torch.zeros(1, T, dtype=torch.int32, device="cuda")
        H.hill_cache_insert_q4(s.desc, k, v, s.k4, s.v4, s.params, s.seen, s.pos, s.accum, 0, 0, slots)
        H.hill_sync_status()
        K, V = torch.zeros_like(k), torch.zeros_like(v)
        lo, hi = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (0, T))
        desc = H.make_desc(torch.zeros(1, 2, 128, dtype=s.dt, device="cuda"), K, V)
        H.hill_cache_read_q4(desc, s.k4, s.v4, s.params, lo, hi, T, K, V)
        H.hill_sync_status()
        assert not torch.isfinite(K[0, 0, 3]).any() and not torch.isfinite(V[0, 1, 8]).any()
        rest = torch.ones(2, T, dtype=torch.bool, device="cuda")
        rest[0, 3] = rest[1, 8] = False
        assert all(torch.equal(a[0, :, :T][rest], b[0, :, :T][rest]) for a, b in zip((s.k4, s.v4, s.params), clean))
        assert torch.isfinite(K[0][rest]).all() and torch.isfinite(V[0][rest]).all()
