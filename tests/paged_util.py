"""Plain float64 forms of the calls over prompts and caches in pages, for the tests, written from the definitions in
include/hill.h; they share no code with the package."""
import numpy as np
import torch

from bounded_util import ALL, error

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a step, relative to the value


def sees(n, m, sinks, window):
    """[n][m]: what the last n of m positions look at."""
    pos, j = np.arange(n)[:, None] + m - n, np.arange(m)
    return (j <= pos) & ((j < sinks) | (j > pos - window))


def prompt(q, k, v, q_start, k_start, sinks, window, half):
    """(out, lse, bound of out, bound of lse) of packed float64 rows; rows of no sequence are NaN.

    A logit is off as in bounded_util.error; its weight meets v rounded (half), and so is the output."""
    T, H, d = q.shape
    G = H // k.shape[1]
    out, bound = np.full((T, H, d), np.nan), np.zeros((T, H, d))
    lse, lbound = np.full((T, H), np.nan), np.zeros((T, H))
    for b in range(len(q_start) - 1):
        qs, ks = slice(q_start[b], q_start[b + 1]), slice(k_start[b], k_start[b + 1])
        n, m = qs.stop - qs.start, ks.stop - ks.start
        if n == 0:
            continue
        see = sees(n, m, sinks, window)
        for h in range(H):
            kh, vh, qh = k[ks, h // G], v[ks, h // G], q[qs, h]
            z = np.where(see, qh @ kh.T / np.sqrt(d), -np.inf)
            size = np.where(see, np.abs(qh) @ np.abs(kh).T / np.sqrt(d), 0).max(1, initial=0)
            top = z.max(1, initial=-np.inf)
            p = np.where(see, np.exp(z - np.where(np.isfinite(top), top, 0)[:, None]), 0)
            total = p.sum(1)
            with np.errstate(divide="ignore"):
                lse[qs, h] = top + np.log(total)
            p = p / np.where(total > 0, total, 1)[:, None]
            out[qs, h] = p @ vh
            e = error(2 * size)
            bound[qs, h] = (p @ np.abs(vh)) * (e + half)[:, None] + half * np.abs(out[qs, h])
            lbound[qs, h] = e + 2.0 ** -22 * np.abs(np.where(total > 0, lse[qs, h], 0))
    return out, lse, bound, lbound


def importance(q, k, lse, q_start, k_start, sinks, window, newest, cap, kvh):
    """(sums [B][cap] or [B][Hkv][cap], bound): lse as given.

    Beside the logits' error a weight has that of lse * log2 e and of the argument (2^-23 of their size each); the sums
    are float32, a weight passing through at most 64 sequential additions per tile of 128 rows."""
    H, d = q.shape[1:]
    Hkv, B = k.shape[1], len(q_start) - 1
    G = H // Hkv
    w, wb = np.zeros((B, Hkv, cap)), np.zeros((B, Hkv, cap))
    for b in range(B):
        qs, ks = slice(q_start[b], q_start[b + 1]), slice(k_start[b], k_start[b + 1])
        n, m = qs.stop - qs.start, ks.stop - ks.start
        if n == 0 or m == 0:
            continue
        see = sees(n, m, sinks, window) & (np.arange(n) >= n - newest)[:, None]
        c = min(m, cap)
        for h in range(H):
            kh, qh = k[ks, h // G], q[qs, h]
            z = qh @ kh.T / np.sqrt(d)
            with np.errstate(invalid="ignore"):
                p = np.where(see, np.exp(np.where(see, z - lse[qs, h][:, None], 0)), 0)
            size = np.where(see, np.abs(qh) @ np.abs(kh).T / np.sqrt(d), 0).max()
            big = np.abs(lse[qs, h][see.any(1)]).max(initial=0) + size
            e = error(2 * size) + 2 * 2.0 ** -23 * big + (64 + n * G / 2) * 2.0 ** -24
            w[b, h // G, :c] += p.sum(0)[:c]
            wb[b, h // G, :c] += p.sum(0)[:c] * e
    return (w, wb) if kvh else (w.sum(1), wb.sum(1))


def e4m3(y):
    """The E4M3 value nearest to y (ties to even), float64."""
    step = 2.0 ** (np.clip(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -30))), -6, 8) - 3)
    return np.clip(np.rint(y / step) * step, -448, 448)


def quantise(x):
    """(codes' values, scales) of float64 rows of 16-bit numbers, in the float32 steps that the header states."""
    x = x.astype(np.float32)
    amax = np.abs(x).max(-1, keepdims=True)
    keep = amax >= 2.0 ** -119
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        r = np.where(keep, np.float32(448) * (np.float32(1) / np.where(keep, amax, 1)), np.float32(0)).astype(np.float32)
        scale = amax * (np.float32(1) / np.float32(448))
        return e4m3((x * r).astype(np.float64)), np.where(keep, scale, 0).astype(np.float32)[..., 0]


def paged_rows(pool, table, cap):
    """[B][Hkv][cap][...] of a pool [pages][Hkv][page][...], pages outside it as zeros."""
    pages, Hkv, page = pool.shape[:3]
    out = np.zeros((table.shape[0], Hkv, cap) + pool.shape[3:], pool.dtype)
    for b in range(table.shape[0]):
        for p in range(cap):
            pg = table[b, p // page]
            if 0 <= pg < pages:
                out[b, :, p] = pool[pg, :, p % page]
    return out
