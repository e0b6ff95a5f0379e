"""ipv_page_compact and ipv_page_copy: rows bit for bit where they are copied, turned keys step by step, bounds."""
import math

import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import blocks as X
from tests import paged as R
from tests.test_gpu_qkv import check_bounds

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "f32", "fp8", "fp4")


def kept(B, L, H, n, C, seed):
    """Ascending rows, other ones in every slice."""
    g = torch.Generator().manual_seed(seed)
    out = torch.zeros((B, L, H, C), dtype=torch.int32)
    for b in range(B):
        for l in range(L):
            for h in range(H):
                c = min(C, n[b])
                out[b, l, h, :c] = torch.randperm(n[b], generator=g)[:c].sort().values
    return out.cuda()


def check(fmt, pool, table, new_table, n, keep, rows=None, rotary=True, R_=0):
    B, L, H, C = keep.shape
    T, D = pool.shape.page_rows, pool.head_dim
    before, ws = X.like(pool), ipv.alloc_page_workspace("cuda")
    angles = R.angles(max(max(n), C), D, "cuda") if rotary else None
    bounds = ipv.BlockBounds(pool, R_) if R_ else None
    if R_:
        bounds.values.fill_(777)
    counts = [C] * B if rows is None else rows
    print("compact", fmt, tuple(keep.shape), n, counts, rotary, R_, flush=True)
    ipv.ipv_page_compact(pool, table, new_table, n, keep, ws, rows=rows, rotary=angles, bounds=bounds)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0
    want = [t.clone() for t in X.raw(before)]
    got = X.raw(pool)
    for b in range(B):
        j = torch.arange(counts[b], device="cuda")
        to, slot = new_table[b].long()[j // T], j % T
        for l in range(L):
            for h in range(H):
                at = keep[b, l, h, :counts[b]].long()
                page, old = (table[b].long()[at // T] if table is not None else torch.full_like(at, b)), at % T
                for i, t in enumerate(X.raw(before)):
                    want[i][to, l, h, slot] = t[page, l, h, old]
                if not rotary:
                    continue
                # turned rows by value; then taken over from the result, so that the rest is compared bit for bit
                scales = None if before.K_scales is None else before.K_scales[page, l, h, old]
                x = R.stored_values(before.K[page, l, h, old], scales, fmt).float()[None, None]
                y = X.turned(X.turned(x, angles, at[None], back=True), angles, j[None])[0, 0]
                moved = at != j
                scales = None if pool.K_scales is None else pool.K_scales[to, l, h, slot]
                stored = R.stored_values(pool.K[to, l, h, slot], scales, fmt)
                assert torch.equal(stored[moved], X.coded_again(y[moved], fmt))
                for i in (0, 2) if len(got) > 2 else (0,):
                    want[i][to[moved], l, h, slot[moved]] = got[i][to[moved], l, h, slot[moved]]
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    if R_:
        check_bounds(fmt, pool, new_table, bounds, [0] * B, counts, range(L))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("rotary,R_", [(True, 16), (True, 0), (False, 48)])
def test_formats_and_sizes(fmt, D, rotary, R_):
    B, L, H, T, n, C = 2, 2, 3, 48, [200, 131], 77
    pool = R.filled_pool(fmt, 20, L, H, T, D, D)
    tables = R.shuffled_table(1, 14, 20, 3)[0]
    check(fmt, pool, tables[:10].view(2, 5).contiguous(), tables[10:].view(2, 2).contiguous(), n, kept(B, L, H, n, C, D), rotary=rotary, R_=R_)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,R_", [(16, 16), (64, 16), (64, 64), (7, 0), (100, 0), (320, 160)])
@pytest.mark.parametrize("n,C,rows", [([1, 300], 1, None), ([300, 65], 65, [65, 0]), ([64, 300], 300, [3, 299])])
def test_lengths_and_pages(fmt, T, R_, n, C, rows):
    B, L, H, D = 2, 1, 2, 64
    cols, new_cols = -(-300 // T), -(-C // T)
    pool = R.filled_pool(fmt, 2 * (cols + new_cols), L, H, T, D, T)
    order = R.shuffled_table(1, 2 * (cols + new_cols), 2 * (cols + new_cols), 3)[0]
    check(fmt, pool, order[:2 * cols].view(2, cols).contiguous(), order[2 * cols:].view(2, new_cols).contiguous(), n,
          kept(B, L, H, n, C, T), rows=rows, R_=R_)


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_in_any_order_and_twice(fmt):
    pool = R.filled_pool(fmt, 8, 1, 2, 32, 64, 1)
    order = R.shuffled_table(1, 8, 8, 3)
    g = torch.Generator().manual_seed(1)
    keep = torch.randint(0, 120, (1, 1, 2, 100), generator=g, dtype=torch.int32).cuda()
    check(fmt, pool, order[:, :4].contiguous(), order[:, 4:].contiguous(), [120], keep, R_=32)


@pytest.mark.parametrize("fmt", FORMATS)
def test_out_of_a_contiguous_cache(fmt):
    """Without a table stream b's rows are page b; the new pages are others of the pool."""
    pool = R.filled_pool(fmt, 5, 2, 2, 128, 64, 1)
    new = torch.tensor([[3], [2]], dtype=torch.int32, device="cuda")
    check(fmt, pool, None, new, [128, 90], kept(2, 2, 2, [128, 90], 60, 1), R_=16)


@pytest.mark.parametrize("fmt", FORMATS)
def test_bad_rows_and_pages_are_left_out(fmt):
    pool = R.filled_pool(fmt, 8, 1, 1, 32, 64, 1)
    before, ws = X.like(pool), ipv.alloc_page_workspace("cuda")
    keep = torch.arange(0, 80, dtype=torch.int32).view(1, 1, 1, 80).cuda()
    keep[..., 5], keep[..., 6], keep[..., 7] = -1, 100, 2**31 - 1
    table = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device="cuda")
    new = torch.tensor([[4, 5, 6]], dtype=torch.int32, device="cuda")
    angles = R.angles(128, 64, "cuda")
    ipv.ipv_page_compact(pool, table, new, 100, keep, ws, rotary=angles)
    assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_KEEP
    for a, b in zip(X.raw(pool), X.raw(before)):
        assert torch.equal(a[4, 0, 0, 5:8], b[4, 0, 0, 5:8]) and torch.equal(a[4, 0, 0, 8:], b[0, 0, 0, 8:]) and torch.equal(a[:4], b[:4])
    ipv.ipv_clear_device_errors(ws)
    # a new page and an old one that are none: their rows stay out, and nothing else is written
    keep = torch.arange(0, 80, dtype=torch.int32).view(1, 1, 1, 80).cuda()
    pool = X.like(before)
    bounds = ipv.BlockBounds(pool, 16)
    bounds.values.fill_(777)
    ipv.ipv_page_compact(pool, torch.tensor([[0, -5, 2, 3]], dtype=torch.int32, device="cuda"),
                         torch.tensor([[4, 5, 99]], dtype=torch.int32, device="cuda"), 100, keep, ws, rotary=angles, bounds=bounds)
    assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE
    for a, b in zip(X.raw(pool), X.raw(before)):
        assert torch.equal(a[4], b[0]) and torch.equal(a[:4], b[:4]) and torch.equal(a[5:], b[5:])
    assert bool((bounds.values[6:] == 777).all())


@pytest.mark.parametrize("fmt", ("fp8", "fp4"))
def test_a_turn_of_next_to_nothing_keeps_the_scale(fmt):
    """Blocks whose largest value is the type's largest, turned by angles near zero: no bit is lost to a larger scale."""
    D, n = 64, 64
    pool = R.filled_pool(fmt, 2, 1, 1, 64, D, 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    if fmt == "fp8":
        pool.K[0] = torch.where(torch.rand(pool.K[0].shape, generator=g, device="cuda") < 0.3, 0x7e, 0).to(torch.uint8)
    else:
        pool.K[0] = torch.where(torch.rand(pool.K[0].shape, generator=g, device="cuda") < 0.3, 0x77, 0).to(torch.uint8)
    a = torch.rand((n, D // 2), generator=g, device="cuda") * 1e-6
    angles = torch.stack((a.cos(), a.sin()), -1).contiguous()
    keep = torch.arange(n - 1, -1, -1, dtype=torch.int32).view(1, 1, 1, n).cuda()
    new, ws = torch.tensor([[1]], dtype=torch.int32, device="cuda"), ipv.alloc_page_workspace("cuda")
    ipv.ipv_page_compact(pool, torch.zeros_like(new), new, n, keep, ws, rotary=angles)
    torch.cuda.synchronize()
    old, got = (R.stored_values(pool.K[p], pool.K_scales[p], fmt) for p in (0, 1))
    # An element x with the pair y becomes x + d, |d| <= 1e-6 |y| (the angles differ by no more) and four roundings. x is itself a
    # stored value, so the nearest one to x + d is no further than |d| from that: |got - x| <= 2 |d|. (A zero whose
    # pair lies in a block of a larger scale may become the type's least value.)
    pair = old.roll(D // 2, -1)
    d = 1e-6 * pair.abs() + 4 * 2.0**-24 * (old.abs() + pair.abs())
    assert bool(((got.flip(2) - old).abs() <= 2 * d).all())
    assert torch.equal(pool.K_scales[1].flip(2), pool.K_scales[0])


@pytest.mark.parametrize("fmt", ("fp8", "fp4"))
def test_blocks_that_are_nan_stay_nan(fmt):
    pool = R.filled_pool(fmt, 2, 1, 1, 32, 64, 1)
    pool.K_scales[0, 0, 0, 9, 0] = 255
    pool.V_scales[0, 0, 0, 9, 1] = 255
    keep = torch.arange(3, 20, dtype=torch.int32).view(1, 1, 1, 17).cuda()
    new, ws = torch.tensor([[1]], dtype=torch.int32, device="cuda"), ipv.alloc_page_workspace("cuda")
    ipv.ipv_page_compact(pool, torch.zeros_like(new), new, 32, keep, ws, rotary=R.angles(32, 64, "cuda"))
    assert ipv.ipv_read_device_errors(ws) == ipv.DEV_NAN  # as it turned the keys: the pair of each NaN is one too
    x = R.rows_of(pool, fmt, torch.ones_like(new), 0, 0, 0)[6]
    assert bool(x.isnan().all()) and bool((pool.V_scales[1, 0, 0, 6] == pool.V_scales[0, 0, 0, 9]).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("T,rows,R_", [(64, 64, 16), (64, 37, 32), (48, 1, 48), (5, 3, 0), (7, 7, 0), (31, 30, 0)])
def test_copies(fmt, D, T, rows, R_):
    L, H = 3, 2
    pool = R.filled_pool(fmt, 9, L, H, T, D, T)
    before, ws = X.like(pool), ipv.alloc_page_workspace("cuda")
    bounds = ipv.BlockBounds(pool, R_) if R_ else None
    if R_:
        bounds.values.copy_(torch.randn(bounds.values.shape, device="cuda"))
        kept_bounds = bounds.values.clone()
    src, dst = [0, 3, 3, 8, 6], [1, 2, 7, 5, 6]
    ipv.ipv_page_copy(pool, *(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (src, dst)), ws, rows=rows, bounds=bounds)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0
    for a, b in zip(X.raw(pool), X.raw(before)):
        want = b.clone()
        for s, d in zip(src, dst):
            want[d, :, :, :rows] = b[s, :, :, :rows]
        assert torch.equal(a.view(torch.uint8), want.view(torch.uint8))
    if R_:
        for s, d in zip(src, dst):
            kept_bounds[d, :, :, :-(-rows // R_)] = kept_bounds[s, :, :, :-(-rows // R_)]
        assert torch.equal(bounds.values, kept_bounds)


def test_copies_of_nothing_and_bad_pages():
    pool, ws = R.filled_pool("fp8", 4, 1, 1, 16, 64, 1), ipv.alloc_page_workspace("cuda")
    before = X.like(pool)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    ipv.ipv_page_copy(pool, none, none, ws)
    assert ipv.ipv_read_device_errors(ws) == 0
    src, dst = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 4, 1, 2**31 - 1], [2, 1, -1, 0]))
    ipv.ipv_page_copy(pool, src, dst, ws)
    assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE
    for a, b in zip(X.raw(pool), X.raw(before)):
        assert torch.equal(a[2], b[0]) and torch.equal(a[[0, 1, 3]], b[[0, 1, 3]])
    assert math.isfinite(float(pool.K.float().sum()))
