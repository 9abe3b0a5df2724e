"""Weights and V scales of very different size in one row of a bounded cache: light tokens keep their share of the
output beside heavy ones, as float32 weights would have it."""
import numpy as np
import pytest
import torch

from bounded_util import ALL, encode, pack, values
from test_gpu_bounded import DT, H, Case, check, gen, to16  # noqa: F401 (H: the fixture)

pytestmark = pytest.mark.gpu


def plant_key(c, j, row):
    """Key row j of every sequence: row [B][Hkv][128], in the cache's type (or its 4-bit form)."""
    row = row.to(c.q.dtype)
    x = row.double().cpu().numpy()
    if c.q4:
        k, s, lo = encode(x, to16(c.q.dtype))
        c.k4[:, :, j] = torch.from_numpy(pack(k)).cuda()
        c.params[:, :, j, 0] = torch.from_numpy(s).to(c.q.dtype).cuda()
        c.params[:, :, j, 1] = torch.from_numpy(lo).to(c.q.dtype).cuda()
        c.K64[:, :, j] = values(pack(k), s, lo)
    else:
        c.K[:, :, j] = row
        c.K64[:, :, j] = x


def scale_value(c, j, by):
    """Value row j times a power of two (or 0)."""
    if c.q4:
        c.params[:, :, j, 2:] *= by
        if by == 0:
            c.v4[:, :, j] = 0
    else:
        c.V[:, :, j] *= by
    c.V64[:, :, j] *= by


def aligned_queries(c, seed):
    """The heads of a KV head look the same way; returns that direction [B][Hkv][128], of about unit entries."""
    B, Hkv = c.desc.batch, c.desc.num_kv_heads
    u = torch.randn(B, Hkv, 128, device="cuda", generator=gen(seed))
    u *= 128 ** 0.5 / u.norm(dim=-1, keepdim=True)
    c.q = (u.repeat_interleave(c.desc.num_q_heads // Hkv, 1) + 0.1 * c.q.float()).to(c.q.dtype)
    return u


# Kinds of rows: (type, size of all values, log2 of the large row's factor).
RATIOS = [("bf16", 1.0, 16), ("bf16", 1.0, 20), ("bf16", 1.0, 24), ("bf16", 1.0, 40), ("fp16", 2.0 ** -8, 18)]


@pytest.mark.parametrize("ratio", RATIOS, ids=lambda r: f"{r[0]}-2^{r[2]}")
@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (16, 2), (32, 1)], ids=lambda h: f"{h[0]}x{h[1]}")
@pytest.mark.parametrize("form", ["clusters", "list"])
def test_a_large_value_row_of_little_weight(H, form, heads, q4, ratio):  # noqa: F811
    """A row whose values are 2^16 to 2^40 times the others' but whose weight is 2^-60 of theirs."""
    dtype, size, log2 = ratio
    B, cap, kernels = (2, 300, 1) if form == "clusters" else (160, 150, 2)
    c = Case(H, B, *heads, cap, dtype, q4, seed=71, scale=size)
    u = aligned_queries(c, 72)
    for j in (5, 100):
        plant_key(c, j, -3.8 * u)   # a logit of -43, 2^-62
        scale_value(c, j, 2.0 ** log2)
    n0 = H.hill_kernel_launches()
    got = c.attend([cap] * B, 0, ALL)
    assert H.hill_kernel_launches() - n0 == kernels
    ref, w, bound, _ = c.reference([cap] * B, 0, ALL)
    assert w[0, [5, 100]].max() < 2.0 ** -50 * heads[0]
    check(got, ref, bound)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads", [(4, 1), (8, 1), (32, 1)], ids=lambda h: f"{h[0]}x{h[1]}")
@pytest.mark.parametrize("q4", [False, True], ids=["16bit", "q4"])
def test_a_heavy_token_without_a_value(H, q4, heads, dtype):  # noqa: F811
    """One token holds nearly all the weight and has the value zero: the output is what the others, each 2^-26 to
    2^-34 of it, add up to.

    Weights of 16-bit caches in fp16 carry an error of up to 2^-32 of the largest, which this output shows; the other
    forms keep a relative error."""
    n = 120001
    c = Case(H, 1, *heads, n, dtype, q4, seed=73)
    u = aligned_queries(c, 74)
    plant_key(c, 70003, 1.85 * u)
    scale_value(c, 70003, 0)
    ref, w, bound, _ = c.reference([n], 0, ALL)
    light = np.delete(w[0], 70003) / heads[0]
    assert 2.0 ** -32 < np.median(light) < 2.0 ** -27
    if dtype == "fp16" and not q4:
        bound = bound + 2.0 ** -32 * np.abs(c.V64[:, 0]).sum(1)[:, None, :]
    check(c.attend([n], 0, ALL), ref, bound)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (32, 1)], ids=lambda h: f"{h[0]}x{h[1]}")
@pytest.mark.parametrize("value", [0, 1])
def test_a_heavy_token_in_four_bits(H, value, heads, dtype):  # noqa: F811
    """The rest is 2^-20 of one token's weight, in 4 bits, with that token's value and without it."""
    c = Case(H, 1, *heads, 3000, dtype, True, seed=79, scale=0.05)
    u = aligned_queries(c, 80)
    plant_key(c, 1234, 2.0 * u)
    scale_value(c, 1234, value)
    ref, w, bound, wb = c.reference([3000], 0, ALL)
    assert np.delete(w[0], 1234).sum() < 2.0 ** -12 * heads[0]
    accum = torch.zeros(1, 3000, device="cuda")
    check(c.attend([3000], 0, ALL, accum), ref, bound)
    check(accum.cpu().numpy().astype(np.float64), w, wb + 2.0 ** -23 * w)


def test_scales_that_grow_and_weights_that_grow(H):  # noqa: F811
    """Every later token of a row is heavier, or its values larger, or the one while the other shrinks: what was summed
    is rescaled many times over."""
    n = 4000
    for seed, (kz, vz) in enumerate([(20, 0), (0, 30), (20, -30), (-20, 30), (20, 30)]):
        c = Case(H, 1, 4, 1, n, "bf16", True, seed=83 + seed)
        u = aligned_queries(c, 84)
        t = np.arange(n) / n
        x = torch.from_numpy(c.K64).cuda() * 0.1 + u[:, :, None].double() * torch.from_numpy(kz * t / 128 ** 0.5)[:, None].cuda()
        x = x.to(torch.bfloat16).double().cpu().numpy()
        k, s, lo = encode(x, to16(torch.bfloat16))
        c.k4.copy_(torch.from_numpy(pack(k)))
        c.params[:, :, :n, 0] = torch.from_numpy(s).bfloat16().cuda()
        c.params[:, :, :n, 1] = torch.from_numpy(lo).bfloat16().cuda()
        c.K64 = values(pack(k), s, lo)
        by = 2.0 ** np.round(vz * t)
        c.params[:, :, :n, 2:] *= torch.from_numpy(by)[:, None].cuda().bfloat16()
        c.V64 = c.V64 * by[:, None]
        ref, w, bound, _ = c.reference([n], 0, ALL)
        check(c.attend([n], 0, ALL), ref, bound)
