"""A decode loop over a cache of bounded size, in 16 and in 4 bits.

    python -m paper_2602_18750_gb300.bounded [--slots 4096] [--prompt 16384] [--steps 256] [--batch 4]

A prompt goes in by chunks, with attention after each chunk's last token, then
the decode steps follow: every step inserts the new token (evicting by
accumulated attention weight once the slots are full) and attends over what is
held.  Synthetic rows stand in for a model's; the step is captured in a CUDA
graph, whose state (positions, weights, counts) lives on the device.
"""
from __future__ import annotations

import argparse

import torch

from . import hill


def rows(g, batch, kv_heads, n, dtype):
    return [torch.randn(batch, kv_heads, n, 128, generator=g, device="cuda").to(dtype) for _ in range(2)]


def run(bits: int, slots: int, prompt: int, steps: int, batch: int, heads: int = 32, kv_heads: int = 8,
        dtype=torch.float16, chunk: int = 512, seed: int = 0):
    """Returns (microseconds of a decode step, the last output, the cache)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    sinks = 4
    chunk = max(1, min(chunk, slots - sinks))   # a full cache has to have room for a chunk
    cache = hill.BoundedCache(batch, heads, kv_heads, slots, dtype, bits, sinks, recent=slots // 8, max_new=chunk)
    q = torch.randn(batch, heads, 128, generator=g, device="cuda").to(dtype)
    for start in range(0, prompt, chunk):
        cache.insert(*rows(g, batch, kv_heads, min(chunk, prompt - start), dtype))
        cache.attend(q)
    k, v = rows(g, batch, kv_heads, 1, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.step(q, k, v)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            cache.step(q, k, v)
    torch.cuda.current_stream().wait_stream(side)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(3):
        graph.replay()
    begin.record()
    for _ in range(steps):
        q.normal_(generator=g)
        k.normal_(generator=g)
        v.normal_(generator=g)
        graph.replay()
    end.record()
    hill.hill_sync_status()
    return begin.elapsed_time(end) * 1e3 / max(1, steps), cache.out, cache


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--slots", type=int, default=4096)
    ap.add_argument("--prompt", type=int, default=16384)
    ap.add_argument("--steps", type=int, default=256)
    ap.add_argument("--batch", type=int, default=4)
    a = ap.parse_args()
    hill.load()
    for bits in (16, 4):
        us, out, cache = run(bits, a.slots, a.prompt, a.steps, a.batch)
        print(f"{bits:2d} bits: {a.slots} slots of {int(cache.seen[0])} tokens, {us:.1f} us a step (new inputs drawn "
              f"each step included), |out| {out.norm().item():.4g}")


if __name__ == "__main__":
    main()
