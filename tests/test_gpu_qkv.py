"""ipv_qkv_write and ipv_block_bounds: new tokens normed, turned and written as the header says, against
64 bits and, bit for bit, against ipv_page_write of rows normed step by step; bounds against the stored rows."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import blocks as X
from tests import paged as R

pytestmark = pytest.mark.gpu
EPS = 1e-6
FORMATS = ("bf16", "f32", "fp8", "fp4")


def tokens(B, A, H, M, D, kind, seed, token_major=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for h in (A, H, H):
        x = torch.randn((B, M, h, D) if token_major else (B, h, M, D), generator=g, device="cuda") * 3
        out.append((x.transpose(1, 2) if token_major else x).to(kind))
    return out


def check(fmt, pool, table, first, layer, q, k, v, rows=None, norm=True, rotary=True, R_=0, out=None):
    B, A, M, D = q.shape
    H = pool.shape.kv_heads
    g = torch.Generator(device="cuda").manual_seed(9)
    qw, kw = ((torch.rand(D, generator=g, device="cuda") + 0.5) if norm else None for _ in range(2))
    counts = [M] * B if rows is None else rows
    angles = R.angles(max(f + c for f, c in zip(first, counts)) or 1, D, "cuda") if rotary else None
    bounds = ipv.BlockBounds(pool, R_) if R_ else None
    if R_:
        bounds.values.fill_(777)
    other, ws = X.like(pool), ipv.alloc_page_workspace("cuda")
    out = torch.full(q.shape, 777.0, dtype=pool.dtype, device="cuda") if out is None else out
    q0 = q.clone()
    print("qkv", fmt, tuple(q.shape), first, rows, norm, rotary, R_, flush=True)
    ipv.ipv_qkv_write(pool, table, first, layer, q, k, v, out, ws, rows=rows, q_norm=qw, k_norm=kw, eps=EPS, rotary=angles, bounds=bounds)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0
    # keys and values: the bits that ipv_page_write makes of rows normed step by step
    k32 = X.normed32(k, kw, EPS) if norm else k.float()
    ipv.ipv_page_write(other, table, first, k32[:, None].contiguous(), v[:, None].float().contiguous(), ws, rows=rows, first_layer=layer,
                       rotary=angles)
    for a, b in zip(X.raw(pool), X.raw(other)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # queries: step by step, and in 64 bits
    q32 = X.normed32(q0, qw, EPS) if norm else q0.float()
    q64 = X.head_normed(q0.double(), qw, EPS) if norm else q0.double()
    pos = torch.tensor(first, device="cuda")[:, None] + torch.arange(M, device="cuda")
    if rotary:
        at = pos.clamp_max(angles.shape[0] - 1)
        lo, hi = q64.abs().chunk(2, -1)
        size = torch.cat((lo + hi, lo + hi), -1)
        q32, q64 = X.turned(q32, angles, at), X.turned(q64, angles, at)
    else:
        size = q64.abs()
    # rounding: s, two products, a product and a sum of the turn (fp32), then the result's
    tol = 6 * 2.0**-24 * size + (2.0**-8 if pool.dtype is torch.bfloat16 else 2.0**-24) * q64.abs()
    for b, m in enumerate(counts):
        assert torch.equal(out[b, :, :m], q32[b, :, :m].to(pool.dtype))
        assert bool(((out[b, :, :m].double() - q64[b, :, :m]).abs() <= tol[b, :, :m]).all())
        if out.data_ptr() != q.data_ptr():
            assert bool((out[b, :, m:] == 777.0).all())
    if R_:
        check_bounds(fmt, pool, table, bounds, first, counts, range(layer, layer + 1))
    return out


def check_bounds(fmt, pool, table, bounds, first, counts, layers):
    """Blocks with one of the positions have the bounds of their stored rows, all others are as they were (777)."""
    want = torch.full_like(bounds.values, 777)
    R_, T = bounds.block_rows, pool.shape.page_rows
    for b, m in enumerate(counts):
        for j in range(first[b] // R_, -(-(first[b] + m) // R_) if m else 0):
            for layer in layers:
                for h in range(pool.shape.kv_heads):
                    lo, hi = X.block_bounds(pool, fmt, table, b, layer, h, j, R_, first[b] + m)
                    page = int(table[b, j * R_ // T]) if table is not None else b
                    want[page, layer, h, j * R_ % T // R_] = torch.stack((lo, hi)).to(want.dtype)
    assert torch.equal(bounds.values, want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("G,M,kind", [(1, 1, "bf16"), (7, 1, "f32"), (3, 37, "bf16"), (8, 70, "f32")])
def test_formats_and_sizes(fmt, D, G, M, kind):
    B, L, H, T = 2, 2, 2, 48
    pool = R.filled_pool(fmt, 10, L, H, T, D, D + M)
    table = R.shuffled_table(B, 4, 10, G)
    q, k, v = tokens(B, H * G, H, M, D, R_TYPE[kind], 5, token_major=M > 1)
    check(fmt, pool, table, [61, 17], 1, q, k, v, R_=16)


R_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,R_", [(16, 16), (64, 16), (64, 64), (96, 48), (320, 160)])
@pytest.mark.parametrize("first,rows", [([0, 0, 0], [1, 64, 0]), ([15, 16, 47], [2, 1, 70]), ([63, 64, 200], [1, 1, 90]), ([5, 0, 31], [0, 0, 33])])
def test_positions_and_blocks(fmt, T, R_, first, rows):
    B, H, D = 3, 2, 64
    cols = -(-320 // T)
    pool = R.filled_pool(fmt, B * cols + 1, 1, H, T, D, T)
    table = R.shuffled_table(B, cols, B * cols + 1, R_)
    q, k, v = tokens(B, 4, H, 90, D, torch.bfloat16, 7)
    check(fmt, pool, table, first, 0, q, k, v, rows=rows, R_=R_)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("norm,rotary,R_", [(False, False, 0), (True, False, 0), (False, True, 32), (True, True, 0)])
def test_without_parts_of_it(fmt, norm, rotary, R_):
    pool = R.filled_pool(fmt, 4, 2, 3, 32, 128, 1)
    q, k, v = tokens(1, 15, 3, 19, 128, torch.bfloat16, 3)  # heads that do not fill a workgroup's four
    check(fmt, pool, R.shuffled_table(1, 4, 4, 1), [50], 0, q, k, v, norm=norm, rotary=rotary, R_=R_)


def test_only_one_norm():
    """q_norm without k_norm and the other way round: each norms what it names."""
    pool, ws = R.filled_pool("bf16", 2, 1, 1, 32, 64, 1), ipv.alloc_page_workspace("cuda")
    q, k, v = tokens(1, 2, 1, 5, 64, torch.bfloat16, 3)
    w = torch.rand(64, device="cuda") + 0.5
    table = R.shuffled_table(1, 2, 2, 1)
    out = torch.empty_like(q)
    for qw, kw in ((w, None), (None, w)):
        ipv.ipv_qkv_write(pool, table, 3, 0, q, k, v, out, ws, q_norm=qw, k_norm=kw, eps=EPS)
        back = [torch.empty_like(k)[:, None] for _ in range(2)]
        ipv.ipv_page_read(pool, table, 3, *back, ws)
        assert torch.equal(out, q if qw is None else X.normed32(q, w, EPS).bfloat16())
        assert torch.equal(back[0][:, 0], k if kw is None else X.normed32(k, w, EPS).bfloat16())
        assert torch.equal(back[1][:, 0], v)


@pytest.mark.parametrize("fmt,kind", [("bf16", torch.bfloat16), ("f32", torch.float32)])
def test_queries_in_place(fmt, kind):
    pool = R.filled_pool(fmt, 4, 1, 2, 32, 128, 1)
    q, k, v = tokens(2, 6, 2, 33, 128, kind, 3, token_major=True)
    check(fmt, pool, R.shuffled_table(2, 2, 4, 1), [3, 20], 0, q, k, v, out=q)


def test_strided_inputs_of_one_projection():
    """q, k and v as slices of one row of a projection, outputs into a wider tensor."""
    B, A, H, M, D = 2, 6, 2, 9, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    whole = torch.randn((B, M, (A + 2 * H) * D), generator=g, device="cuda").bfloat16()
    q, k, v = (x.unflatten(-1, (-1, D)).transpose(1, 2) for x in whole.split((A * D, H * D, H * D), -1))
    pool = R.filled_pool("fp8", 4, 1, H, 32, D, 1)
    wide = torch.full((B, A, M, 2 * D), 777.0, dtype=torch.bfloat16, device="cuda")
    check("fp8", pool, R.shuffled_table(B, 2, 4, 1), [3, 20], 0, q, k, v, out=wide[..., :D], R_=16)
    assert bool((wide[..., D:] == 777.0).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_no_table(fmt):
    """A contiguous cache is a pool of one page a stream."""
    pool = R.filled_pool(fmt, 3, 2, 2, 160, 64, 1)
    q, k, v = tokens(3, 4, 2, 40, 64, torch.bfloat16, 3)
    check(fmt, pool, None, [0, 100, 31], 1, q, k, v, R_=32)


def test_more_streams_than_a_launch_takes():
    B, H, D, T = 131, 1, 64, 16
    pool = R.filled_pool("bf16", B * 2, 1, H, T, D, 1)
    table = R.shuffled_table(B, 2, B * 2, 1)
    q, k, v = tokens(B, 2, H, 3, D, torch.bfloat16, 3)
    check("bf16", pool, table, [b % 29 for b in range(B)], 0, q, k, v, rows=[b % 4 for b in range(B)], R_=16)


def test_large_and_small_values():
    """Norms of rows whose squares leave fp32, and of rows of zeros."""
    pool = R.filled_pool("f32", 2, 1, 1, 32, 64, 1)
    q, k, v = tokens(1, 2, 1, 8, 64, torch.float32, 3)
    for x in (q, k):
        x[:, :, 0] *= 1e30
        x[:, :, 1] *= 1e-30
        x[:, :, 2] = 0
        x[:, :, 3] *= 1e-3
    check("f32", pool, R.shuffled_table(1, 2, 2, 1), [3], 0, q, k, v)


@pytest.mark.parametrize("fmt", FORMATS)
def test_bad_pages_are_left_out(fmt):
    pool = R.filled_pool(fmt, 6, 1, 1, 32, 64, 1)
    table = torch.tensor([[0, 99, 2], [3, -1, 5]], dtype=torch.int32, device="cuda")
    q, k, v = tokens(2, 2, 1, 70, 64, torch.bfloat16, 3)
    ws, bounds, before = ipv.alloc_page_workspace("cuda"), ipv.BlockBounds(pool, 16), X.like(pool)
    bounds.values.fill_(777)
    ipv.ipv_qkv_write(pool, table, [10, 20], 0, q, k, v, torch.empty(q.shape, dtype=pool.dtype, device="cuda"), ws, bounds=bounds)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE
    for a, b in zip(X.raw(pool), X.raw(before)):  # pages 1 and 4 are nobody's
        assert torch.equal(a[1], b[1]) and torch.equal(a[4], b[4]) and not torch.equal(a[0], b[0]) and not torch.equal(a[5], b[5])
    assert bool((bounds.values[1] == 777).all()) and bool((bounds.values[4] == 777).all())
    # (positions 10 .. 79 and 20 .. 89: the third page's rows end at 79 and 89)
    ipv.ipv_clear_device_errors(ws)
    ipv.ipv_block_bounds(pool, table, [10, 20], 70, bounds, ws)
    assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE


def test_nan_and_infinities_in_bounds():
    """Infinities are bounds like others; a channel with a NaN has a NaN bound, of either sign; quantised blocks with
    one are NaN whole and reported."""
    D = 64
    for fmt in FORMATS:
        pool, ws = R.filled_pool(fmt, 1, 1, 1, 64, D, 1), ipv.alloc_page_workspace("cuda")
        bounds = ipv.BlockBounds(pool, 16)
        q, k, v = tokens(1, 1, 1, 64, D, torch.float32, 3)
        k[0, 0, 3, 1] = float("inf")
        k[0, 0, 18, 2] = float("-inf")
        k[0, 0, 35, 3] = float("nan")
        k[0, 0, 50, 4] = -float("nan")
        ipv.ipv_qkv_write(pool, None, 0, 0, q, k, v, torch.empty(q.shape, dtype=pool.dtype, device="cuda"), ws, bounds=bounds)
        torch.cuda.synchronize()
        assert ipv.ipv_read_device_errors(ws) == (ipv.DEV_NAN if fmt in ("fp8", "fp4") else 0)
        got = bounds.values[0, 0, 0].double()
        nan = got.isnan().any(1)  # [4, D]
        if fmt in ("bf16", "f32"):
            assert nan.nonzero().tolist() == [[2, 3], [3, 4]]
            assert got[0, 1, 1] == float("inf") and got[1, 0, 2] == -float("inf")
        else:
            assert bool(nan[:, :32].all()) and not bool(nan[:, 32:].any())
        stored = R.rows_of(pool, fmt, None, 0, 0, 0).view(4, 16, D)
        fine = ~nan
        assert torch.equal(got[:, 0][fine], stored.amin(1)[fine]) and torch.equal(got[:, 1][fine], stored.amax(1)[fine])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [32, 64, 128, 256])
def test_bounds_of_rows_that_are_there(fmt, D):
    B, L, H, T, R_ = 3, 3, 2, 96, 48
    pool = R.filled_pool(fmt, 8, L, H, T, D, 3)
    table = R.shuffled_table(B, 2, 8, 4)
    bounds, ws = ipv.BlockBounds(pool, R_), ipv.alloc_page_workspace("cuda")
    bounds.values.fill_(777)
    first, rows = [0, 50, 95], [191, 1, 2]
    ipv.ipv_block_bounds(pool, table, first, rows, bounds, ws, first_layer=1, layers=2)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0
    check_bounds(fmt, pool, table, bounds, first, rows, range(1, 3))


def test_an_empty_call_does_nothing():
    pool, ws = R.filled_pool("bf16", 2, 1, 1, 32, 64, 1), ipv.alloc_page_workspace("cuda")
    before = X.like(pool)
    q, k, v = tokens(2, 2, 1, 0, 64, torch.bfloat16, 3)
    table = R.shuffled_table(2, 1, 2, 1)
    ipv.ipv_qkv_write(pool, table, [0, 5], 0, q, k, v, torch.empty_like(q), ws, rotary=R.angles(3, 64, "cuda"))
    ipv.ipv_block_bounds(pool, table, 0, 0, ipv.BlockBounds(pool, 16), ws)
    assert all(torch.equal(a, b) for a, b in zip(X.raw(pool), X.raw(before))) and ipv.ipv_read_device_errors(ws) == 0
