"""A streaming session over the memory-capped cache, then an answer from it.

Frames arrive a few at a time. In every layer their queries attend over the
layer's cached rows and their own (the live half of the ping-pong cache, as it
stands), the cache is compressed whenever it reaches its cap, and at the end a
question and then one token at a time are answered twice: from the live half
in bf16, and from 4-bit or 8-bit pages into which the kept rows are moved. The
model is left out: its queries, keys and values are random tensors of its
shapes, and the two answers' distance is printed.

    python examples/stream_answer.py            # LLaVA-OV-7B shapes, 2 layers
    python examples/stream_answer.py --fmt u8 --frames 96
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2506_15745_gb300 import ipv  # noqa: E402
from paper_2506_15745_gb300.cache import PingPongCache  # noqa: E402
from paper_2506_15745_gb300.paged import PagedBatch, PagedCache  # noqa: E402


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def run(*, fmt: str = "u4", layers: int = 2, heads: int = 4, share: int = 7, dim: int = 128, grid: int = 14, cap: int = 48,
        keep: int = 32, step: int = 16, frames: int = 96, question: int = 23, answer: int = 8, page: int = 64, seed: int = 0):
    """Runs the session; returns passes, cached rows, and the answers' relative distance."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    p, slabs = grid * grid, layers * heads
    rows = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()  # noqa: E731
    reserve = question + answer  # room for the answer behind the cap
    capacity = cap * p + reserve
    ipv.init(dtype="bf16", max_head_dim=dim, max_frame_tokens=p, max_slabs=slabs, token_capacity=capacity)
    try:
        cache = PingPongCache(slabs, capacity, dim, "bf16", patch_ids=True, frame_ids=True)
        kept = torch.empty((slabs, keep * p), dtype=torch.int32, device="cuda")
        passes, fresh = 0, True
        for _ in range(0, frames, step):
            new = step * p
            k_new, v_new = rows(slabs, new, dim), rows(slabs, new, dim)
            k, v = cache.structs()
            ipv.append_frames(k, v, k_new, v_new, layers, heads, dim, cache.n_tokens, step, grid, grid)
            cache.n_tokens += new
            chunk = PagedBatch(None, ints(0, new), ints(cache.n_tokens), total_rows=new, max_rows=new, max_kv=capacity)
            for layer in range(layers):  # the frames' own attention
                PagedCache.of_layer(cache, layer, layers, heads).attend(rows(new, heads * share, dim), chunk)
            if cache.n_tokens >= cap * p:
                cache.compress(layers, heads, grid, grid, keep * p, 0.5, kept, pid_valid=not fresh)
                fresh, passes = False, passes + 1

        # The kept rows of every layer, quantised into pages of a pool of their own.
        n = cache.n_tokens
        per_layer = -(-(n + reserve) // page)
        pools, tables = [], ints(*range(per_layer)).view(1, -1)
        whole = PagedBatch(tables, ints(0, n), ints(n), total_rows=n, max_rows=n, max_kv=n)
        for layer in range(layers):
            pool = PagedCache(per_layer, page, heads, dim, fmt)
            live = slice(layer * heads, (layer + 1) * heads)
            pool.write(cache.k_live[live, :n].transpose(0, 1), cache.v_live[live, :n].transpose(0, 1), whole)
            pools.append(pool)

        off, size = 0.0, 0.0
        for new in [question] + [1] * answer:
            n += new
            live_batch = PagedBatch(None, ints(0, new), ints(n), total_rows=new, max_rows=new, max_kv=capacity)
            pool_batch = PagedBatch(tables, ints(0, new), ints(n), total_rows=new, max_rows=new, max_kv=per_layer * page)
            for layer in range(layers):
                q, k_new, v_new = rows(new, heads * share, dim), rows(new, heads, dim), rows(new, heads, dim)
                pages = PagedCache.of_layer(cache, layer, layers, heads)
                outs = []
                for held, batch in ((pages, live_batch), (pools[layer], pool_batch)):
                    held.write(k_new, v_new, batch)
                    outs.append(held.attend(q, batch).float())
                off += float((outs[0] - outs[1]).square().sum())
                size += float(outs[0].square().sum())
        return {"passes": passes, "rows": n, "distance": (off / size) ** 0.5, "finite": bool(torch.isfinite(outs[1]).all()),
                "bytes_bf16": 4 * dim * heads * layers * n,
                "bytes_pages": sum(t.numel() * t.element_size() for x in pools for t in (x.k, x.v, x.k_par, x.v_par))}
    finally:
        ipv.shutdown()


def main() -> None:
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--fmt", choices=("u4", "u8"), default="u4")
    a.add_argument("--layers", type=int, default=2)
    a.add_argument("--frames", type=int, default=96)
    a = a.parse_args()
    r = run(fmt=a.fmt, layers=a.layers, frames=a.frames)
    print(f"{r['passes']} compression passes, {r['rows']} rows cached; {a.fmt} pages {r['bytes_pages'] / 2**20:.1f} MiB "
          f"against {r['bytes_bf16'] / 2**20:.1f} MiB; the answers differ by {100 * r['distance']:.2f}%")


if __name__ == "__main__":
    main()
