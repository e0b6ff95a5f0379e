"""ipv_attend where the page table names pages that no query sees: entries of rows before the window, between the
first rows and the window, and after the newest position may hold anything."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R

pytestmark = pytest.mark.gpu


def needed(n, first, m, window, sinks):
    """The rows that some query sees."""
    out = set()
    for p in range(first, first + m):
        for j in range(min(p + 1, n)):
            if not window or j > p - window or j < sinks:
                out.add(j)
    return out


def attend(pool, table, n, first, q, window, sinks):
    ws = ipv.alloc_attend_workspace(pool, *q.shape[:3])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    ipv.ipv_attend(pool, table, n, first, 0, q, out, ws, window=window, sinks=sinks, lse=lse)
    return out, lse, ipv.ipv_read_device_errors(ws)


# windows whose oldest row lies inside a tile, first rows that end inside one, positions that end before the rows do
CASES = [(1, 0, 300, 0), (50, 0, 300, 0), (50, 3, 300, 0), (77, 21, 300, 0), (0, 0, 300, 130), (40, 5, 300, 130), (97, 0, 300, -40)]


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 7, 16, 36, 64])
@pytest.mark.parametrize("m", [1, 5, 30])
def test_entries_of_rows_that_nobody_sees(fmt, D, T, m):
    G, cols = 4, -(-300 // T)
    pool = R.filled_pool(fmt, cols + 2, 1, 2, T, D, T)
    pages = torch.arange(1, cols + 1, dtype=torch.int32).flip(0)[None]  # page 0, which stands in for others, is none of them
    for t in (pool.K, pool.V) if fmt in ("bf16", "f32") else (pool.K_scales, pool.V_scales):
        t[0] = float("nan") if fmt in ("bf16", "f32") else 255
    kind = torch.float32 if fmt == "f32" else torch.bfloat16
    q = torch.randn((1, 2 * G, m, D), generator=torch.Generator("cuda").manual_seed(m), device="cuda").to(kind)
    for window, sinks, n, back in CASES:
        first = n - m - back
        rows = needed(n, first, m, window, sinks)
        keep = torch.zeros(cols, dtype=torch.bool)
        keep[torch.tensor([j // T for j in rows])] = True
        print("entries", fmt, D, T, m, window, sinks, n, first, int(keep.sum()), "of", cols, flush=True)
        want = attend(pool, pages.cuda(), n, first, q, window, sinks)
        assert want[2] == 0
        for other in (-1, cols + 2, 2**31 - 1, -2**31):
            got = attend(pool, torch.where(keep, pages, torch.tensor(other, dtype=torch.int32)).cuda(), n, first, q, window, sinks)
            assert got[2] == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        for j in (min(rows), max(rows)):  # and one that is seen is reported
            table = pages.clone()
            table[0, j // T] = -1
            assert attend(pool, table.cuda(), n, first, q, window, sinks)[2] == ipv.DEV_BAD_PAGE
