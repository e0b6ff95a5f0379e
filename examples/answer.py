"""A video goes through the continual-compression loop, and questions are answered from what it keeps.

  1. frames enter a cache of pre-rotation keys and are compressed at its cap (ipv_ckv_stream);
  2. the kept rows go into pages of a pool that several conversations share: keys
     rotated to their new positions, rows quantised as they are written (ipv_page_write);
  3. a question's tokens are written behind them and attend over the pages, causally among
     themselves; then single tokens do, one at a time (ipv_page_write, ipv_attend);
  4. the pages' rows come back, keys rotated back, for more frames (ipv_page_read).

The model's projections are stand-ins (random rows); the shapes are a 7B-class video
model's. Run on an MI355X:  python examples/answer.py [--format fp8] [--layers 28]
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_15745_amd import ipv  # noqa: E402

FORMATS = {"bf16": ipv.PAGES_BF16, "fp8": ipv.PAGES_FP8, "fp4": ipv.PAGES_FP4}


def angles(positions, D, device):
    """Cosine and sine of every position and pair, fp32 [positions, D / 2, 2]."""
    a = torch.arange(positions)[:, None] * torch.exp(-math.log(1e6) * torch.arange(D // 2) / (D // 2))
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous().to(device)


def rotated(q, table, first):
    """Queries [B, heads, rows, D] turned to positions first, first + 1, ... (a model's own step)."""
    c, s = table[first:first + q.shape[2]].unbind(-1)
    lo, hi = q.float().chunk(2, -1)
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1).to(q.dtype)


class Answers:
    """What a serving program holds for one model: a pool of pages, its tables, the workspaces."""

    def __init__(self, streams, layers, kv_heads, q_heads, D, rows, page_rows, fmt, chunk, device):
        cols = -(-rows // page_rows)
        self.pool = ipv.PagePool.empty(streams * cols, layers, kv_heads, page_rows, D, fmt, device)
        # pages in no particular order, as an allocator hands them out
        self.table = torch.randperm(streams * cols).view(streams, cols).int().to(device)
        self.rotary = angles(rows, D, device)
        self.write_ws = ipv.alloc_page_workspace(device)
        self.attend_ws = ipv.alloc_attend_workspace(self.pool, streams, q_heads, chunk)

    def fill(self, K, V, rows):
        """The first `rows` rows of a compressed cache [B, L, H, S, D] into the pages."""
        ipv.ipv_page_write(self.pool, self.table, 0, K, V, self.write_ws, rows=rows, rotary=self.rotary)

    def layer(self, layer, q, k, v, at, out, window=0, sinks=0):
        """One layer's step for new tokens at positions at, ...: their rows are written, then they attend."""
        M = q.shape[2]
        ipv.ipv_page_write(self.pool, self.table, at, k[:, None], v[:, None], self.write_ws, first_layer=layer, rotary=self.rotary)
        ipv.ipv_attend(self.pool, self.table, at + M, at, layer, rotated(q, self.rotary, at), out, self.attend_ws, window=window,
                       sinks=sinks)
        return out

    def errors(self):
        return ipv.ipv_read_device_errors(self.write_ws) | ipv.ipv_read_device_errors(self.attend_ws)


def run(fmt="fp8", layers=28, kv_heads=4, q_heads=28, D=128, grid=(14, 14), cap=6272, budget=3136, recent=4, frames=48, question=35,
        tokens=16, page_rows=64, seed=0, device="cuda", say=print):
    """Returns (outputs [tokens + 1] of the last layer, the rows read back and those kept, rows in the cache)."""
    p = grid[0] * grid[1]
    g = torch.Generator(device=device).manual_seed(seed)

    def rows(*shape):
        return torch.randn(shape, generator=g, device=device).bfloat16()

    # 1. the video
    cache = [torch.zeros((1, layers, kv_heads, cap + p, D), dtype=torch.bfloat16, device=device) for _ in range(2)]
    meta = [torch.zeros((1, layers, kv_heads, cap + p), dtype=torch.int32, device=device) for _ in range(2)]
    comp = ipv.Compressor(cache[0], *grid, budget)
    n, passes = 0, 0
    for f in range(0, frames, 16):  # sixteen frames at a time, as the vision tower delivers them
        new = [rows(min(16, frames - f), 1, layers, kv_heads, p, D) for _ in range(2)]
        n, more = ipv.ipv_ckv_stream(*cache, *meta, n, *new, f, cap, budget, 0.5, recent, None, comp.tar, comp.van, comp.keep_idx,
                                     comp.ws, *grid)
        passes += more
    # 2. into pages
    a = Answers(1, layers, kv_heads, q_heads, D, n + question + tokens, page_rows, FORMATS[fmt], question, device)
    a.fill(*cache, n)
    # 3. the question, then one token at a time
    outputs, at = [], n
    torch.cuda.synchronize()
    begun = time.perf_counter()
    for M in [question] + [1] * tokens:
        out = torch.empty((1, q_heads, M, D), dtype=torch.bfloat16, device=device)
        for layer in range(layers):
            a.layer(layer, rows(1, q_heads, M, D), rows(1, kv_heads, M, D), rows(1, kv_heads, M, D), at, out)
        outputs.append(out)
        at += M
    torch.cuda.synchronize()
    took = time.perf_counter() - begun
    # 4. and back
    back = [torch.empty((1, layers, kv_heads, n, D), dtype=torch.bfloat16, device=device) for _ in range(2)]
    ipv.ipv_page_read(a.pool, a.table, 0, *back, a.write_ws, rotary=a.rotary)
    assert a.errors() == 0 and comp.device_errors() == 0
    say("%d frames in %d passes -> %d rows in %s pages; a question of %d tokens and %d more through %d layers in %.1f ms" % (
        frames, passes, n, fmt, question, tokens, layers, took * 1e3))
    return outputs, back, [c[..., :n, :] for c in cache]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--format", default="fp8", choices=sorted(FORMATS))
    ap.add_argument("--layers", type=int, default=28)
    ap.add_argument("--frames", type=int, default=48)
    o = ap.parse_args()
    outputs, back, kept = run(o.format, layers=o.layers, frames=o.frames)
    for name, x, y in zip("KV", back, kept):
        print("%s read back: relative error %.2g" % (name, float((x.float() - y.float()).norm() / y.float().norm())))
