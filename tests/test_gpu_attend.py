"""ipv_attend against plain attention in 64 bits: formats, head layouts,
lengths, pages that end inside a tile, windows, ragged streams, rows that see
nothing, infinities and NaN where they are not seen."""
import math

import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R

pytestmark = pytest.mark.gpu


def check(fmt, pool, table, n, first, layer, q, window=0, sinks=0, rows=None, scale=None, out=None):
    B, A, M, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    ws = ipv.alloc_attend_workspace(pool, B, A, M)
    out = torch.full_like(q, 777.0) if out is None else out
    lse = torch.full((B, A, M), 777.0, device=q.device)
    print("attend", fmt, tuple(q.shape), n, first, window, sinks, flush=True)
    ipv.ipv_attend(pool, table, n, first, layer, q, out, ws, q_rows=rows, scale=scale, window=window, sinks=sinks, lse=lse)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0
    want, wlse, spread, size = R.attend(pool, fmt, table, n, first, layer, q, scale, window, sinks, rows)
    tol = R.tolerance(fmt, D, spread, size)
    for b in range(B):
        m = M if rows is None else rows[b]
        o, w = out[b, :, :m].double(), want[b, :, :m]
        fine = torch.isfinite(w)
        assert torch.equal(torch.isfinite(o), fine) and torch.equal(torch.isnan(o), torch.isnan(w))
        assert torch.equal(o[~fine & ~torch.isnan(w)], w[~fine & ~torch.isnan(w)])
        off = (o - w)[fine].abs() - tol[b, :, :m][fine]
        assert off.numel() == 0 or float(off.max()) <= 0, float(off.max())
        # a row not asked for is left alone
        assert bool((out[b, :, m:] == 777.0).all()) and bool((lse[b, :, m:] == 777.0).all())
        ls, wl = lse[b, :, :m].double(), wlse[b, :, :m]
        assert torch.equal(ls == -math.inf, wl == -math.inf)
        ok = torch.isfinite(wl)
        lim = 2 * (D + 4) * 2.0**-24 * max(size, 1.0) + 1e-5 + 1e-6 * wl[ok].abs()
        assert bool(((ls[ok] - wl[ok]).abs() <= lim).all())
    return out, lse


def queries(fmt, B, A, M, D, seed, token_major=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = torch.float32 if fmt == "f32" else torch.bfloat16
    q = torch.randn((B, M, A, D) if token_major else (B, A, M, D), generator=g, device="cuda").to(kind)
    return q.transpose(1, 2) if token_major else q


FORMATS = ("bf16", "f32", "fp8", "fp4")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("G,m", [(1, 1), (7, 1), (2, 9), (3, 11), (8, 40), (1, 133)])
def test_formats_and_head_layouts(fmt, D, G, m):
    B, L, H, T, n = 2, 2, 2, 48, [301, 170]
    pool = R.filled_pool(fmt, 20, L, H, T, D, D + G)
    table = R.shuffled_table(B, 7, 20, m)
    check(fmt, pool, table, n, [x - m for x in n], 1, queries(fmt, B, H * G, m, D, 3, token_major=G == 3))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("T", [1, 7, 16, 31, 64, 100, 300])
@pytest.mark.parametrize("m", [1, 20])
def test_pages_that_end_inside_a_tile(fmt, T, m):
    n = 261
    cols = -(-n // T)
    pool = R.filled_pool(fmt, cols + 3, 1, 2, T, 64, T)
    check(fmt, pool, R.shuffled_table(1, cols, cols + 3, T), [n], [n - m], 0, queries(fmt, 1, 8, m, 64, T))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
def test_lengths(fmt, n):
    pool = R.filled_pool(fmt, 40, 1, 1, 32, 128, n)
    table = R.shuffled_table(1, 32, 40, n)
    for m in {1, min(n, 5), n if n <= 129 else 200}:
        check(fmt, pool, table, [n], [n - m], 0, queries(fmt, 1, 3, m, 128, n))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (31, 0), (32, 1), (33, 64), (64, 5), (100, 40), (299, 7), (300, 0), (5000, 9)])
@pytest.mark.parametrize("m", [1, 6, 90])
def test_windows_and_first_rows(fmt, window, sinks, m):
    B, n = 3, [300, 221, 90]
    pool = R.filled_pool(fmt, 40, 1, 2, 40, 64, window)
    table = R.shuffled_table(B, 8, 40, m)
    check(fmt, pool, table, n, [x - m for x in n], 0, queries(fmt, B, 6, m, 64, sinks), window, sinks)


@pytest.mark.parametrize("fmt", FORMATS)
def test_queries_anywhere(fmt):
    """Queries past the rows, before the last rows, and in gaps that leave them nothing to see; streams of
    no rows and of no queries."""
    B, m = 6, 12
    n = [100, 100, 0, 77, 50, 64]
    first = [500, 20, 3, 0, 0, 200]
    rows = [12, 12, 5, 0, 12, 7]
    pool = R.filled_pool(fmt, 30, 1, 2, 32, 64, 5)
    table = R.shuffled_table(B, 4, 30, 6)
    q = queries(fmt, B, 4, m, 64, 7)
    check(fmt, pool, table, n, first, 0, q, rows=rows)
    check(fmt, pool, table, n, first, 0, q, window=90, sinks=0, rows=rows)   # the first and last streams see nothing
    check(fmt, pool, table, n, first, 0, q, window=90, sinks=2, rows=rows)


@pytest.mark.parametrize("fmt", FORMATS)
def test_no_row_sees_anything(fmt):
    pool = R.filled_pool(fmt, 4, 1, 1, 32, 128, 5)
    for m in (1, 50):
        out, lse = check(fmt, pool, R.shuffled_table(1, 2, 4, 6), [60], [1000], 0, queries(fmt, 1, 2, m, 128, 7), window=3)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m", [1, 3, 30])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_what_is_not_seen_stays_out(fmt, m, window, sinks):
    """NaN and infinities in rows past the last, in rows between the first ones and the window, and in the new
    tokens' own rows, which only later queries see."""
    n, T, D = 150, 16, 64
    pool = R.filled_pool(fmt, 14, 1, 1, T, D, 8)
    table = R.shuffled_table(1, 12, 14, 9)
    q = queries(fmt, 1, 2, m, D, 10)

    def put(row, values):
        page, slot = int(table[0, row // T]), row % T
        for name, v in zip(("K", "V"), values):
            if fmt in ("bf16", "f32"):
                getattr(pool, name)[page, 0, 0, slot] = v
            else:
                getattr(pool, name + "_scales")[page, 0, 0, slot] = 255

    for row in range(n, 12 * T):
        put(row, (math.nan, math.nan))
    if window:
        for row in range(sinks, n - m - window):
            put(row, (math.inf, -math.inf if row % 2 else math.nan))
    if m > 1:  # seen by the last query alone, and by those from there on
        put(n - 1, (0.5 if fmt in ("bf16", "f32") else math.nan, math.inf))
        put(n - m // 2 - 1, (0.25, math.nan))
    check(fmt, pool, table, [n], [n - m], 0, q, window, sinks)


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 70])
def test_large_scores(fmt, m):
    """Scores far apart: one row takes all the weight, and the running maximum moves by hundreds."""
    n, D = 700, 64
    pool = R.filled_pool(fmt, 12, 1, 1, 64, D, 8)
    pool.K.mul_((torch.arange(12, device="cuda").view(-1, 1, 1, 1, 1) * 3 + 1).to(pool.K.dtype))
    table = R.shuffled_table(1, 11, 12, 9)
    check(fmt, pool, table, [n], [n - m], 0, queries(fmt, 1, 4, m, D, 10) * 4)


@pytest.mark.parametrize("fmt", FORMATS)
def test_long_rows_are_split_and_joined(fmt):
    n, D = [9000, 4111], 128
    pool = R.filled_pool(fmt, 160, 1, 2, 96, D, 8)
    table = R.shuffled_table(2, 94, 200, 9) % 160
    for m, G in ((1, 4), (5, 4), (33, 2)):
        check(fmt, pool, table, n, [x - m for x in n], 0, queries(fmt, 2, 2 * G, m, D, 10))


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_many_streams(fmt):
    """More streams than one launch takes, with lengths of their own."""
    B, D, T = 230, 32, 16
    n = [(7 * b) % 61 for b in range(B)]
    m = [min(x, 1 + b % 3) for b, x in enumerate(n)]
    pool = R.filled_pool(fmt, 300, 1, 1, T, D, 8)
    table = (torch.arange(B * 4, device="cuda").view(B, 4) % 300).int()
    check(fmt, pool, table, n, [x - y for x, y in zip(n, m)], 0, queries(fmt, B, 2, 3, D, 10), rows=m)


def test_the_cache_itself():
    """A cache [B, L, H, S, D] as a pool of B pages, no table: a pass, then attention over what it kept."""
    B, L, H, S, D = 2, 3, 2, 200, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn((B, L, H, S, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    fr = (torch.arange(S, device="cuda") // 20).int().expand(B, L, H, S).contiguous()
    pa = (torch.arange(S, device="cuda") % 20).int().expand(B, L, H, S).contiguous()
    comp = ipv.Compressor(K, 4, 5, 80)
    comp.compress(K, V, fr, pa, S, 0.5, 2)
    pool = ipv.PagePool(K, V)
    for m in (1, 37):
        check("bf16", pool, None, [80, 80], [80 - m, 80 - m], 2, queries("bf16", B, 6, m, D, 4))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m", [1, 100])
def test_same_bits_every_time_and_in_a_graph(fmt, m):
    n, D, B = [2000, 1500], 128, 2
    pool = R.filled_pool(fmt, 70, 1, 2, 64, D, 8)
    table = R.shuffled_table(B, 32, 70, 9)
    q = queries(fmt, B, 8, m, D, 10)
    ws = ipv.alloc_attend_workspace(pool, B, 8, m)
    out, lse = torch.empty_like(q), torch.empty(B, 8, m, device="cuda")
    args = (pool, table, n, [x - m for x in n], 0, q, out, ws)
    ipv.ipv_attend(*args, lse=lse)
    torch.cuda.synchronize()
    want, wlse = out.clone(), lse.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(5):
            ipv.ipv_attend(*args, lse=lse)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ipv.ipv_attend(*args, lse=lse)
    for k in range(4):
        out.zero_(), lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wlse)
        q.mul_(1.0)


def test_strides_beyond_32_bits():
    """Pages whose offsets pass 2^32 bytes."""
    T, D, H = 1 << 14, 256, 4
    pages = 160  # 160 * 4 * 16384 * 512 bytes = 5 GiB each of K and V
    K = torch.zeros((pages, 1, H, T, D), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    pool = ipv.PagePool(K, V)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    n = 2 * T + 100
    for page in (pages - 1, 0, pages - 2):
        K[page].normal_()
        V[page].normal_()
    q = queries("bf16", 1, H, 2, D, 1)
    check("bf16", pool, table, [n], [n - 2], 0, q)


def test_a_table_entry_outside_the_pool_is_reported():
    for fmt in FORMATS:
        for m in (1, 60):
            pool = R.filled_pool(fmt, 4, 1, 1, 32, 64, 1)
            table = torch.tensor([[1, 4, 2]], dtype=torch.int32, device="cuda")
            q = queries(fmt, 1, 1, m, 64, 2)
            ws = ipv.alloc_attend_workspace(pool, 1, 1, m)
            out = torch.empty_like(q)
            ipv.ipv_attend(pool, table, 90, 90 - m, 0, q, out, ws)
            assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE
            table[0, 1] = -1
            ipv.ipv_clear_device_errors(ws)
            ipv.ipv_attend(pool, table, 90, 90 - m, 0, q, out, ws)
            assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE
            table[0, 1] = 3
            ipv.ipv_clear_device_errors(ws)
            ipv.ipv_attend(pool, table, 90, 90 - m, 0, q, out, ws)
            assert ipv.ipv_read_device_errors(ws) == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("T", [64, 192])
@pytest.mark.parametrize("G,m,window,sinks", [(1, 1, 0, 0), (5, 1, 90, 3), (2, 9, 0, 0), (3, 11, 70, 33), (8, 40, 0, 0), (1, 133, 100, 1)])
def test_pages_of_whole_tiles(fmt, D, T, G, m, window, sinks):
    """A tile's rows follow each other in a page, whose rows past the last are not zeros."""
    B, L, H, n = 2, 2, 2, [413, 192]
    pool = R.filled_pool(fmt, 20, L, H, T, D, D + G)
    table = R.shuffled_table(B, 7, 20, m)
    check(fmt, pool, table, n, [x - m for x in n], 1, queries(fmt, B, H * G, m, D, 3, token_major=G == 3), window, sinks)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T", [100, 128])
@pytest.mark.parametrize("G,m", [(1, 1), (2, 13), (1, 40), (2, 300)])
def test_key_range_in_many_parts(fmt, T, G, m):
    """One KV head: more parts than are joined in one go."""
    n = 9000
    pool = R.filled_pool(fmt, 95, 1, 1, T, 128, 2)
    table = R.shuffled_table(1, 92, 95, m)
    check(fmt, pool, table, [n], [n - m], 0, queries(fmt, 1, G, m, 128, 3))


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("B,m", [(1, 300), (5, 140), (12, 40)])
def test_parts_beyond_one_round(fmt, B, m):
    """Row tiles that fill a part of the card: key ranges in parts that take it more than once."""
    H, G, D, n = 8, 8, 128, [700 + 100 * b for b in range(B)]
    pool = R.filled_pool(fmt, 30 * B, 1, H, 64, D, 2)
    table = R.shuffled_table(B, 30, 30 * B, m)
    check(fmt, pool, table, n, [x - m for x in n], 0, queries(fmt, B, H * G, m, D, 3))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("m", [1, 6, 40])
def test_what_is_not_seen_stays_out_of_whole_tiles(fmt, D, m):
    """The same in pages that hold whole tiles, which are read to their last row; and an entry outside the pool."""
    n, T, G, window, sinks = 300, 64, 4, 50, 3
    pool = R.filled_pool(fmt, 8, 1, 1, T, D, 8)
    table = R.shuffled_table(1, 6, 8, 9)
    dirty = [(r, 0) for r in range(n, 6 * T)] + [(r, r) for r in range(sinks, n - m - window)]
    dirty += [(n - 1, 1)] * (m > 1)  # the last query alone sees this one
    for row, kind in dirty:
        at = (int(table[0, row // T]), 0, 0, row % T)
        if fmt in ("bf16", "f32"):
            pool.K[at], pool.V[at] = (0.5 if row == n - 1 else math.nan), (math.nan, math.inf, -math.inf)[kind % 3]
        else:
            pool.K_scales[at] = pool.V_scales[at] = 255
    q = queries(fmt, 1, G, m, D, 10)
    check(fmt, pool, table, [n], [n - m], 0, q, window, sinks)
    ws = ipv.alloc_attend_workspace(pool, 1, G, m)
    for entry in (8, -1, 1 << 30):
        table[0, 4] = entry
        ipv.ipv_attend(pool, table, n, n - m, 0, q, torch.empty_like(q), ws)
        assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE
        ipv.ipv_clear_device_errors(ws)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m", [1, 70])
@pytest.mark.parametrize("window,sinks", [(2**31 - 1, 0), (2**31 - 1, 2**31 - 1), (20, 2**31 - 1), (2**30, 5)])
def test_windows_beyond_any_position(fmt, m, window, sinks):
    """The widest window is none, and all rows may be first rows."""
    n = 200
    pool = R.filled_pool(fmt, 5, 1, 2, 64, 64, 3)
    table = R.shuffled_table(1, 4, 5, 4)
    q = queries(fmt, 1, 4, m, 64, 5)
    out, lse = check(fmt, pool, table, [n], [n - m], 0, q, window, sinks)
    full, flse = check(fmt, pool, table, [n], [n - m], 0, q)
    if window > n:
        assert torch.equal(out, full) and torch.equal(lse, flse)
