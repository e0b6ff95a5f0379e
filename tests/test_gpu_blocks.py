"""ipv_block_select and ipv_attend_blocks against plain forms in 64 bits: lists equal to the last entry, attention within the
roundings that it makes."""
import math

import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import blocks as X
from tests import paged as R

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "f32", "fp8", "fp4")


def queries(fmt, B, A, M, D, seed, token_major=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = torch.float32 if fmt == "f32" else torch.bfloat16
    q = torch.randn((B, M, A, D) if token_major else (B, A, M, D), generator=g, device="cuda").to(kind)
    return q.transpose(1, 2) if token_major else q


def made_bounds(pool, fmt, table, n, R_):
    """Bounds of the first n[b] rows of every stream."""
    bounds, ws = ipv.BlockBounds(pool, R_), ipv.alloc_page_workspace("cuda")
    ipv.ipv_block_bounds(pool, table, [0] * len(n), n, bounds, ws)
    assert ipv.ipv_read_device_errors(ws) == 0
    return bounds


def check_attend(fmt, pool, table, n, first, layer, q, blocks, R_, out, lse, rows=None, scale=None):
    B, A, M, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    want, wlse, spread, size = X.attend_lists(pool, fmt, table, n, first, layer, q, blocks.cpu(), R_, scale, rows)
    tol = R.tolerance(fmt, D, spread, size)
    for b in range(B):
        m = M if rows is None else rows[b]
        off = (out[b, :, :m].double() - want[b, :, :m]).abs() - tol[b, :, :m]
        assert off.numel() == 0 or float(off.max()) <= 0, float(off.max())
        assert bool((out[b, :, m:] == 777.0).all()) and bool((lse[b, :, m:] == 777.0).all())
        ls, wl = lse[b, :, :m].double(), wlse[b, :, :m]
        assert torch.equal(ls == -math.inf, wl == -math.inf)
        ok = torch.isfinite(wl)
        assert bool(((ls[ok] - wl[ok]).abs() <= 2 * (D + 4) * 2.0**-24 * max(size, 1.0) + 1e-5 + 1e-6 * wl[ok].abs()).all())


def check(fmt, pool, table, n, first, layer, q, bounds, top, first_blocks=0, last_blocks=1, rows=None):
    B, A, M, D = q.shape
    H, R_ = pool.shape.kv_heads, bounds.block_rows
    print("blocks", fmt, tuple(q.shape), n, first, R_, top, first_blocks, last_blocks, flush=True)
    ws = ipv.alloc_blocks_workspace(bounds, B, A, M, top, max(n))
    ws[4352:] = 0xff  # whatever it holds
    got = torch.full((B, H, M, top), 777, dtype=torch.int32, device="cuda")
    ipv.ipv_block_select(pool, table, bounds, n, first, layer, q, got, ws, q_rows=rows, first_blocks=first_blocks, last_blocks=last_blocks)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), X.select(bounds, table, n, first, layer, q, top, first_blocks, last_blocks, rows))
    both = torch.full_like(got, 777)
    out, lse = torch.full_like(q, 777.0), torch.full((B, A, M), 777.0, device="cuda")
    ipv.ipv_attend_blocks(pool, table, n, first, layer, q, both, out, ws, bounds=bounds, q_rows=rows, first_blocks=first_blocks,
                          last_blocks=last_blocks, lse=lse)
    torch.cuda.synchronize()
    assert torch.equal(both, got) and ipv.ipv_read_device_errors(ws) == 0
    check_attend(fmt, pool, table, n, first, layer, q, got, R_, out, lse, rows)
    # the lists as they were left, read: the same sums in the same or other parts
    again, lse2 = torch.full_like(q, 777.0), torch.full_like(lse, 777.0)
    ipv.ipv_attend_blocks(pool, table, n, first, layer, q, got, again, ws, block_rows=R_, q_rows=rows, lse=lse2)
    torch.cuda.synchronize()
    check_attend(fmt, pool, table, n, first, layer, q, got, R_, again, lse2, rows)
    return got, out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("G,m", [(1, 1), (7, 1), (16, 2), (17, 1), (40, 2), (2, 21)])
def test_formats_and_head_layouts(fmt, D, G, m):
    B, L, H, T, n = 2, 2, 2, 48, [301, 170]
    pool = R.filled_pool(fmt, 20, L, H, T, D, D + G)
    table = R.shuffled_table(B, 7, 20, m)
    bounds = made_bounds(pool, fmt, table, n, 16)
    check(fmt, pool, table, n, [x - m for x in n], 1, queries(fmt, B, H * G, m, D, 3, token_major=G == 2), bounds, 5)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,R_", [(16, 16), (32, 32), (96, 48), (64, 64), (160, 80), (128, 16), (256, 128)])
@pytest.mark.parametrize("top,first,last", [(1, 0, 0), (1, 0, 1), (4, 1, 2), (9, 0, 0), (40, 3, 1)])
def test_blocks_and_pages(fmt, T, R_, top, first, last):
    n = [517, 40]
    cols = -(-n[0] // T)
    pool = R.filled_pool(fmt, 2 * cols + 3, 1, 2, T, 64, T)
    table = R.shuffled_table(2, cols, 2 * cols + 3, T)
    check(fmt, pool, table, n, [512, 35], 0, queries(fmt, 2, 6, 5, 64, T), made_bounds(pool, fmt, table, n, R_), top, first, last)


@pytest.mark.parametrize("fmt", ("bf16", "fp8"))
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 255, 256, 257])
def test_lengths(fmt, n):
    pool = R.filled_pool(fmt, 20, 1, 1, 32, 128, n)
    table = R.shuffled_table(1, 16, 20, n)
    bounds = made_bounds(pool, fmt, table, [n], 16)
    for m in {1, min(n, 5), min(n, 40)}:
        check(fmt, pool, table, [n], [n - m], 0, queries(fmt, 1, 3, m, 128, n), bounds, 3)


@pytest.mark.parametrize("fmt", FORMATS)
def test_queries_anywhere(fmt):
    """Queries past the rows and before the last ones; streams of no rows and of no queries."""
    B, m = 6, 12
    n, first, rows = [100, 100, 0, 77, 50, 64], [500, 20, 3, 0, 0, 200], [12, 12, 5, 0, 12, 7]
    pool = R.filled_pool(fmt, 30, 1, 2, 32, 64, 5)
    table = R.shuffled_table(B, 4, 30, 6)
    bounds = made_bounds(pool, fmt, table, n, 16)
    got, out = check(fmt, pool, table, n, first, 0, queries(fmt, B, 4, m, 64, 7), bounds, 4, 1, 1, rows=rows)
    assert bool((got[2, :, :5] == -1).all()) and bool((out[2, :, :5] == 0).all())


@pytest.mark.parametrize("top,first,last", [(5, 0, 0), (64, 1, 1), (700, 5, 5)])
@pytest.mark.parametrize("n", [8000, 8192, 16400, 40000])
def test_many_blocks(top, first, last, n):
    """More blocks than the lanes' registers take, and lists that waves look up in turns; a few queries."""
    T, D = 64, 32
    cols = -(-n // T)
    pool = R.filled_pool("bf16", cols, 1, 1, T, D, 3)
    table = R.shuffled_table(1, cols, cols, 4)
    check("bf16", pool, table, [n], [n - 3], 0, queries("bf16", 1, 2, 3, D, n), made_bounds(pool, "bf16", table, [n], 16), top, first, last)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,G", [(64, 3), (128, 20)])
def test_a_wave_a_query(fmt, D, G):
    """So many queries that each is one wave's, over lists of ten key tiles, the last ones cut by the query's position."""
    B, H, M, n = 2, 8, 100, [700, 395]
    pool, table = R.filled_pool(fmt, 24, 1, H, 64, D, 2), R.shuffled_table(B, 11, 24, 3)
    check(fmt, pool, table, n, [x - M for x in n], 0, queries(fmt, B, H * G, M, D, 8, token_major=True), made_bounds(pool, fmt, table, n, 16), 20,
          1, 3)


@pytest.mark.parametrize("fmt,D", [("bf16", 32), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 256)])
@pytest.mark.parametrize("blocks", [100, 600, 1100, 2100])
@pytest.mark.parametrize("crowd", [False, True])
def test_many_queries(fmt, D, blocks, crowd):
    """Tiles of queries without workgroups that share their blocks; scores all over their range, or one far above the others,
    which are then next to each other in it. (Random scores: none are equal, and 64 bits in any order rank them alike.)"""
    B, H, G, m, top = 1, 8, 2, 512, 9
    n = blocks * 16 - 5
    pool, table = R.filled_pool(fmt, -(-n // 64), 1, H, 64, D, 3), R.shuffled_table(1, -(-n // 64), -(-n // 64), 4)
    bounds, g = ipv.BlockBounds(pool, 16), torch.Generator(device="cuda").manual_seed(blocks)
    bounds.values.copy_(torch.randn(bounds.values.shape, generator=g, device="cuda"))
    if crowd:
        for h in range(H):
            X.bounds_at(bounds, table, 0, 0, h, 7).mul_(2.0**60)
    q = queries(fmt, B, H * G, m, D, 9)
    print("many queries", fmt, D, blocks, crowd, flush=True)
    ws = ipv.alloc_blocks_workspace(bounds, B, H * G, m, top, n)
    got = torch.full((B, H, m, top), 777, dtype=torch.int32, device="cuda")
    ipv.ipv_block_select(pool, table, bounds, n, n - m, 0, q, got, ws, first_blocks=1, last_blocks=2)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0
    count = (torch.arange(n - m, n, device="cuda") + 16) // 16
    j = torch.arange(blocks, device="cuda")
    for h in range(H):
        at = torch.stack([X.bounds_at(bounds, table, 0, 0, h, x) for x in range(blocks)]).double()  # [blocks, 2, D]
        qs = q[0, h * G:(h + 1) * G].double()
        score = qs.clamp_min(0).sum(0) @ at[:, 1].T + qs.clamp_max(0).sum(0) @ at[:, 0].T
        forced = (j < 1) | (j >= count[:, None] - 2)
        score = torch.where(j >= count[:, None], -math.inf, torch.where(forced, math.inf, score))
        assert torch.equal(got[0, h].long(), score.topk(top, -1).indices.sort(-1).values)


@pytest.mark.parametrize("fmt", ("bf16", "f32"))
def test_equal_scores_go_to_the_lower_block(fmt):
    """Blocks that are copies of a few: ties everywhere, also at the end of what is picked."""
    n, T, D = 1600, 16, 64
    pool = R.filled_pool(fmt, 100, 1, 1, T, D, 3)
    g = torch.Generator().manual_seed(1)
    for t in (pool.K, pool.V):
        t.copy_(t[torch.randint(0, 4, (100,), generator=g).cuda()])
    table = R.shuffled_table(1, 100, 100, 4)
    bounds = made_bounds(pool, fmt, table, [n], 16)
    for top in (1, 7, 30, 77):
        check(fmt, pool, table, [n], [n - 2], 0, queries(fmt, 1, 3, 2, D, top), bounds, top, 0, 0)
    # all scores zero
    check(fmt, pool, table, [n], [n - 2], 0, torch.zeros_like(queries(fmt, 1, 3, 2, D, 1)), bounds, 5, 0, 1)


def test_scores_that_differ_in_the_last_bits():
    """Blocks whose scores differ by less than fp32 sees are still told apart."""
    T, D, N = 16, 128, 60
    pool = R.filled_pool("f32", N, 1, 1, T, D, 3)
    pool.K.fill_(1.0)
    for j in range(N):
        pool.K[j, 0, 0, :, j] = 1 + 2.0**-23 * ((j * 37) % N)
    table = R.shuffled_table(1, N, N, 4)
    q = torch.ones((1, 2, 1, D), device="cuda")
    bounds = made_bounds(pool, "f32", table, [N * T], 16)
    for top in (1, 10, 59):
        check("f32", pool, table, [N * T], [N * T - 1], 0, q, bounds, top, 0, 0)


def test_nan_and_infinite_scores():
    """A block with a NaN bound ranks above all but those that are always picked, one with an infinity above finite ones."""
    T, D, N = 16, 64, 30
    pool = R.filled_pool("bf16", N, 1, 1, T, D, 3)
    table = torch.arange(N, dtype=torch.int32, device="cuda")[None]
    bounds = made_bounds(pool, "bf16", table, [N * T], 16)
    q = queries("bf16", 1, 2, 1, D, 3)
    bounds.values[7, 0, 0, 0, 1, 5] = math.nan
    bounds.values[9, 0, 0, 0, 0, 5] = -math.nan
    bounds.values[20, 0, 0, 0, 1] = math.inf
    bounds.values[21, 0, 0, 0, 0] = -math.inf  # with infinities of both signs in the sum or not: as the formula has it
    ws = ipv.alloc_blocks_workspace(bounds, 1, 2, 1, 6, N * T)
    for top in (1, 2, 3, 5, 6):
        got = torch.full((1, 1, 1, top), 777, dtype=torch.int32, device="cuda")
        ipv.ipv_block_select(pool, table, bounds, N * T, N * T - 1, 0, q, got, ws, last_blocks=0)
        assert torch.equal(got.cpu(), X.select(bounds, table, [N * T], [N * T - 1], 0, q, top, 0, 0))
        assert 7 in got.tolist()[0][0][0] and (top < 2 or 9 in got.tolist()[0][0][0])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R_", [16, 48])
def test_lists_of_ones_own(fmt, R_):
    """In any order, with gaps, entries past the rows or the query, blocks listed twice, and empty ones."""
    B, H, G, M, T, D, n = 2, 2, 3, 4, 96, 64, [290, 100]
    pool = R.filled_pool(fmt, 8, 1, H, T, D, 3)
    table = R.shuffled_table(B, 4, 8, 4)
    first, top = [250, 96], 70
    g = torch.Generator().manual_seed(R_)
    blocks = torch.randint(-3, -(-290 // R_) + 2, (B, H, M, top), generator=g, dtype=torch.int32)
    blocks[0, 0, 0] = -1
    blocks[0, 1, 1, :] = 2
    blocks[1, 0, 2] = 2**31 - 1
    blocks[1, 1, 3] = -2**31
    blocks[1, 1, 0, :-1] = -1
    q, R_blocks = queries(fmt, B, H * G, M, D, 5), blocks.cuda()
    bounds = ipv.BlockBounds(pool, R_)
    ws = ipv.alloc_blocks_workspace(bounds, B, H * G, M, top, 290)
    out, lse = torch.full_like(q, 777.0), torch.full((B, H * G, M), 777.0, device="cuda")
    ipv.ipv_attend_blocks(pool, table, n, first, 0, q, R_blocks, out, ws, block_rows=R_, lse=lse)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0 and torch.equal(R_blocks.cpu(), blocks)
    check_attend(fmt, pool, table, n, first, 0, q, blocks, R_, out, lse)
    assert bool((out[0, :G, 0] == 0).all()) and bool((lse[1, :G, 2] == -math.inf).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_what_is_not_listed_or_not_seen_stays_out(fmt):
    """NaN in every row that a query does not see, in listed blocks and others."""
    T, D, n, first = 32, 64, 100, 80
    pool = R.filled_pool(fmt, 4, 1, 1, T, D, 8)
    table = R.shuffled_table(1, 4, 4, 9)
    q = queries(fmt, 1, 2, 1, D, 10)
    for row in list(range(first + 1, 128)) + list(range(16, 48)):
        page, slot = int(table[0, row // T]), row % T
        for name in "KV":
            if fmt in ("bf16", "f32"):
                getattr(pool, name)[page, 0, 0, slot] = math.nan
            else:
                getattr(pool, name + "_scales")[page, 0, 0, slot] = 255
    blocks = torch.tensor([0, 5, 3, 6, -1], dtype=torch.int32, device="cuda").view(1, 1, 1, 5)
    ws = ipv.alloc_blocks_workspace(ipv.BlockBounds(pool, 16), 1, 2, 1, 5, n)
    out, lse = torch.full_like(q, 777.0), torch.full((1, 2, 1), 777.0, device="cuda")
    ipv.ipv_attend_blocks(pool, table, n, first, 0, q, blocks, out, ws, block_rows=16, lse=lse)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out).all())
    blocks[..., 3] = -1  # (block 6 has no row up to the query)
    check_attend(fmt, pool, table, [n], [first], 0, q, blocks, 16, out, lse)


def test_all_blocks_are_plain_attention():
    """With every block picked the results are ipv_attend's, to the roundings of both."""
    B, H, G, m, T, D, n = 2, 2, 7, 3, 64, 128, [900, 333]
    pool = R.filled_pool("bf16", 40, 1, H, T, D, 3)
    table = R.shuffled_table(B, 15, 40, 4)
    first = [x - m for x in n]
    q = queries("bf16", B, H * G, m, D, 5)
    bounds = made_bounds(pool, "bf16", table, n, 64)
    ws, full = ipv.alloc_blocks_workspace(bounds, B, H * G, m, 15, 900), ipv.alloc_attend_workspace(pool, B, H * G, m)
    out, plain = torch.empty_like(q), torch.empty_like(q)
    blocks = torch.empty((B, H, m, 15), dtype=torch.int32, device="cuda")
    ipv.ipv_attend_blocks(pool, table, n, first, 0, q, blocks, out, ws, bounds=bounds)
    ipv.ipv_attend(pool, table, n, first, 0, q, plain, full)
    want, _, spread, size = R.attend(pool, "bf16", table, n, first, 0, q, D ** -0.5)
    tol = R.tolerance("bf16", D, spread, size)
    for x in (out, plain):
        assert bool(((x.double() - want).abs() <= tol).all())


def test_the_bits_are_the_same_every_time():
    B, H, G, m, T, D, n = 3, 2, 7, 5, 64, 128, [4000, 2000, 77]
    pool = R.filled_pool("fp8", 200, 1, H, T, D, 3)
    table = R.shuffled_table(B, 63, 200, 4)
    bounds = made_bounds(pool, "fp8", table, n, 32)
    q = queries("fp8", B, H * G, m, D, 5)
    ws = ipv.alloc_blocks_workspace(bounds, B, H * G, m, 40, 4000)
    got = []
    for _ in range(5):
        out, blocks = torch.empty_like(q), torch.empty((B, H, m, 40), dtype=torch.int32, device="cuda")
        ipv.ipv_attend_blocks(pool, table, n, [x - m for x in n], 0, q, blocks, out, ws, bounds=bounds)
        got.append((out, blocks))
    assert all(torch.equal(o, got[0][0]) and torch.equal(b, got[0][1]) for o, b in got)
    assert bool((ws[256:4352] == 0).all())  # the counters


def test_bad_pages_are_reported():
    """Entries of blocks that a query can pick or picked; others may hold anything."""
    pool = R.filled_pool("bf16", 8, 1, 1, 32, 64, 3)
    table = torch.tensor([[0, 1, 99, 3, -7]], dtype=torch.int32, device="cuda")
    bounds = ipv.BlockBounds(pool, 32)
    q = queries("bf16", 1, 2, 1, 64, 5)
    ws = ipv.alloc_blocks_workspace(bounds, 1, 2, 1, 2, 160)
    out, blocks = torch.empty_like(q), torch.empty((1, 1, 1, 2), dtype=torch.int32, device="cuda")
    for first, listed, bits in ((63, None, 0), (64, None, ipv.DEV_BAD_PAGE), (100, [0, 3], 0), (100, [0, 2], ipv.DEV_BAD_PAGE), (100, [4, 1], 0)):
        if listed is None:
            ipv.ipv_attend_blocks(pool, table, 128, first, 0, q, blocks, out, ws, bounds=bounds)
        else:
            ipv.ipv_attend_blocks(pool, table, 128, first, 0, q, torch.tensor(listed, dtype=torch.int32, device="cuda").view(1, 1, 1, 2), out,
                                  ws, block_rows=32)
        assert ipv.ipv_read_device_errors(ws) == bits, (first, listed)
        ipv.ipv_clear_device_errors(ws)


def test_more_streams_than_a_launch_takes():
    B, H, D, T = 70, 1, 64, 32
    pool = R.filled_pool("bf16", B * 2, 1, H, T, D, 1)
    table = R.shuffled_table(B, 2, B * 2, 1)
    n = [1 + (b * 7) % 64 for b in range(B)]
    bounds = made_bounds(pool, "bf16", table, n, 16)
    check("bf16", pool, table, n, [max(0, x - 2) for x in n], 0, queries("bf16", B, 2, 2, D, 3), bounds, 2, rows=[min(2, x) for x in n])


def test_scores_that_do_not_fit_at_once():
    """A workspace of the least size: queries sixteen at a time."""
    n, m, T, D = 700, 100, 64, 64
    pool = R.filled_pool("bf16", 11, 1, 2, T, D, 1)
    table = R.shuffled_table(1, 11, 11, 1)
    bounds = made_bounds(pool, "bf16", table, [n], 16)
    q = queries("bf16", 1, 4, m, D, 3)
    least = ipv.blocks_workspace_bytes(pool, 16, 1, 4, 16, 6, n)
    least = max(least, 4352 + 1024 * 16 * (D + 2) * 4)
    ws = torch.zeros(least, dtype=torch.uint8, device="cuda")
    got = torch.empty((1, 2, m, 6), dtype=torch.int32, device="cuda")
    small = torch.zeros(4352 + 2 * 48 * 8 * 20, dtype=torch.uint8, device="cuda")  # scores of 20 queries: 16 at a time
    ipv.ipv_block_select(pool, table, bounds, n, n - m, 0, q, got, small)
    assert torch.equal(got.cpu(), X.select(bounds, table, [n], [n - m], 0, q, 6, 0, 1))
    out = torch.empty_like(q)
    ipv.ipv_attend_blocks(pool, table, n, n - m, 0, q, got, out, ws, bounds=bounds)
    assert torch.equal(got.cpu(), X.select(bounds, table, [n], [n - m], 0, q, 6, 0, 1))
    with pytest.raises(ipv.IpvError) as e:
        ipv.ipv_block_select(pool, table, bounds, n, n - m, 0, q, got, small[:4352 + 2 * 48 * 8 * 15])
    assert e.value.status == ipv.ERR_WORKSPACE
