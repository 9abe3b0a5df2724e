"""Inserts for which too few slots of a bounded cache may go."""
import pytest
import torch

from test_gpu_bounded import H, Store  # noqa: F401 (H: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("held", [16, 14])
def test_too_few_slots_that_may_go(H, held):  # noqa: F811
    """Two slots may go where more are needed: none is given up, tokens without a free slot are dropped."""
    s = Store(H, 1, 2, 16, seed=109)
    s.insert(held, 0, 0)
    s.pos.zero_()
    s.pos[0, 3], s.pos[0, 9] = 7, 8
    before, pos, T = s.K.clone(), s.pos.clone(), 6
    slots = torch.zeros(1, T, dtype=torch.int32, device="cuda")
    new = torch.ones(1, 2, T, 128, dtype=torch.float16, device="cuda")
    H.hill_cache_insert(s.desc, new, new, s.K, s.V, s.seen, s.pos, s.accum, 4, 0, slots)
    with pytest.raises(H.HillError) as e:
        H.hill_sync_status()
    assert e.value.status == H.HILL_ERR_DEVICE and int(s.seen[0]) == held + T
    free = list(range(held, 16))
    assert slots[0].tolist() == free + [-1] * (T - len(free))
    assert torch.equal(s.K[:, :, :held], before[:, :, :held]) and torch.equal(s.pos[:, :held], pos[:, :held])
    assert torch.all(s.K[:, :, held:] == 1)
