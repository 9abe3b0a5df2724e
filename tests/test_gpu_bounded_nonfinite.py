"""Values that are not finite where they are seen: the attention of a bounded cache answers with values that are not
finite either, whatever form the call takes, and leaves the other heads alone."""
import numpy as np
import pytest
import torch

from bounded_util import ALL
from test_gpu_bounded import H, Case, check  # noqa: F401 (H: the fixture)

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
