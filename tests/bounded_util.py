"""Plain float64 forms of the calls of a bounded cache, for the tests: the
attention over the visible part, inserts that evict by accumulated weight,
4-bit rows.  Written from the definitions in include/hill.h with numpy loops;
they share no code with the package."""
import numpy as np

ALL = 1 << 30
SQRT_D = np.sqrt(128.0)


def visible(n, sinks, window):
    j = np.arange(n)
    return j[(j < sinks) | (j >= n - window)]


def attn(q, K, V, lens, sinks, window, kvh=False):
    """(out [B][H][d], weights [rows][cap], bound [B][H][d], wbound [rows][cap]) of float64 arrays.

    bound: how far float32 sums may put the output (see the derivation in `error`)."""
    B, H, d = q.shape
    Hkv, cap = K.shape[1:3]
    G = H // Hkv
    out, bound = np.zeros((B, H, d)), np.zeros((B, H, d))
    w = np.zeros((B, Hkv, cap) if kvh else (B, cap))
    wb = np.zeros_like(w)
    for b in range(B):
        for g in range(Hkv):
            n = int(min(max(lens[b, g] if kvh else lens[b], 0), cap))
            at = visible(n, sinks, window)
            if not at.size:
                continue
            k, v = K[b, g, at], V[b, g, at]
            for h in range(g * G, (g + 1) * G):
                z = k @ q[b, h] / SQRT_D
                p = np.exp(z - z.max())
                p /= p.sum()
                out[b, h] = p @ v
                bound[b, h] = p @ np.abs(v)
                e = 2 * (np.abs(k) @ np.abs(q[b, h]) / SQRT_D).max()
                row = w[b, g] if kvh else w[b]
                row[at] += p
                (wb[b, g] if kvh else wb[b])[at] += p * error(e)
                bound[b, h] *= error(e)
    return out, w, bound, wb


def error(size, extra=0.0):
    """Relative error of a weight whose logit sums terms of total magnitude `size` / 2 in float32.

    A logit is summed in at most 16 float32 steps (eight products of 16 terms, the
    scale, the minimum and its product): its error is below 16 * 2^-23 * size, which is the weight's relative error
    (and once more for the sum that normalises).  The exponential adds 2^-21 (argument
    reduction and the function), the two 16-bit parts of a weight 2^-17 (bf16) and sums of up to
    2^17 weights in at most 2^10 sequential steps 2^-14 at the very worst, 2^-19 for random signs."""
    return 2 * 16 * 2.0 ** -23 * size + 2.0 ** -16 + extra


def encode(x, to16):
    """4-bit form of float64 rows [..][128]: (codes 0..15, scale, min); to16 rounds to the 16-bit type."""
    lo, hi = x.min(-1), x.max(-1)
    scale = to16((hi - lo) / 15)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(scale[..., None] > 0, (x - lo[..., None]) / scale[..., None], 0.0)
    return np.clip(np.rint(c), 0, 15).astype(np.uint8), scale, lo


def pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def values(packed, scale, lo):
    c = np.stack((packed & 15, packed >> 4), -1).reshape(*packed.shape[:-1], 128).astype(np.float64)
    return lo[..., None] + scale[..., None] * c


def insert(seen, pos, accum, n_new, max_new, sinks, recent, weight=None):
    """One row, in place on pos and accum: (slots [max_new], seen after)."""
    cap = pos.shape[0]
    t = max_new if n_new is None else min(max(int(n_new), 0), max_new)
    seen = max(int(seen), 0)
    held = min(seen, cap)
    slots = list(range(held, min(cap, held + t)))
    e = t - len(slots)
    if e:
        may = [j for j in range(held) if sinks <= pos[j] < seen + t - recent]
        order = sorted(may, key=lambda j: (-(accum[j] + 0.0), j))
        slots += sorted(order[len(order) - e:]) if len(order) >= e else [-1] * e
    for i, s in enumerate(slots):
        if s >= 0:
            pos[s] = seen + i
            accum[s] = 0 if weight is None else weight[i]
    return np.array(slots + [-1] * (max_new - t), dtype=np.int32), seen + t
