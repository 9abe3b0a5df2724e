"""The example loop where the cache is smaller than its usual chunk of a prompt."""
import pytest
import torch

from test_gpu_bounded import H  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("slots", [5, 100, 256])
def test_small_caches(H, slots):  # noqa: F811
    from paper_2602_18750_gb300 import bounded
    for bits in (16, 4):
        us, out, cache = bounded.run(bits, slots=slots, prompt=300, steps=4, batch=2, heads=8, kv_heads=2)
        assert us > 0 and torch.isfinite(out).all()
        # the prompt, one step before the capture, three and four replays
        assert cache.seen.tolist() == [300 + 1 + 3 + 4] * 2
        assert sorted(cache.pos[0].tolist())[:4] == [0, 1, 2, 3]   # the first tokens stay


@pytest.mark.parametrize("kvh", [False, True], ids=["seq", "kvh"])
def test_a_sliding_window(H, kvh):  # noqa: F811
    """recent = capacity - sinks: the oldest tokens after the sinks go, whatever their weights."""
    cap, sinks, T = 40, 4, 7
    cache = H.BoundedCache(2, 8, 2, cap, bits=4, sinks=sinks, recent=cap - sinks, kvh=kvh, max_new=T)
    for step in range(30):
        n = T if step < 12 else 1 + step % 3
        k, v = (torch.randn(2, 2, n, 128, device="cuda").half() for _ in range(2))
        cache.insert(k, v)
        cache.attend(torch.randn(2, 8, 128, device="cuda").half())
        seen = int(cache.seen.flatten()[0])
        want = list(range(sinks)) + list(range(seen - (cap - sinks), seen)) if seen > cap else list(range(seen))
        for row in cache.pos.view(-1, cap).tolist():
            assert sorted(row[:min(seen, cap)]) == want
    H.hill_sync_status()
