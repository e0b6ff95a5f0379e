"""ipv_page_write and ipv_page_read against the definitions in 64 bits: the
quantised formats bit for bit, rotation, layers, positions, strides."""
import math

import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R

pytestmark = pytest.mark.gpu
KIND = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows(src, B, L, H, N, D, seed, order="rows"):
    """K, V [B, L, H, N, D], contiguous, or strided as [B, L, N, H, D] or with other elements between the rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    got = []
    for _ in range(2):
        if order == "tokens":
            x = torch.randn((B, L, N, H, D), generator=g, device="cuda").to(KIND[src]).transpose(2, 3)
        elif order == "fused":
            x = torch.randn((B, L, N, H, 3, D), generator=g, device="cuda").to(KIND[src])[..., 1, :].transpose(2, 3)
        else:
            x = torch.randn((B, L, H, N, D), generator=g, device="cuda").to(KIND[src])
        got.append(x)
    return got


def pool_rows(pool, fmt, table, name, L0, L, first, m):
    """Positions first[b] .. first[b] + m of layers L0 .. L0 + L: float64 [B, L, H, m, D]."""
    T = pool.shape.page_rows
    B = len(first)
    at = torch.tensor(first, device="cuda")[:, None] + torch.arange(m, device="cuda")
    pages = table.long().gather(1, at // T) if table is not None else torch.arange(B, device="cuda")[:, None].expand(B, m)
    codes, scales = getattr(pool, name), getattr(pool, name + "_scales")
    v = R.stored_values(codes[pages, L0:L0 + L, :, at % T], None if scales is None else scales[pages, L0:L0 + L, :, at % T], fmt)
    return v.permute(0, 2, 3, 1, 4)


def f32_turned(K, rotary, pos, back=False):
    """The rotation as the header states it: fp32, each product and sum rounded once."""
    a = rotary[pos][:, None, None]
    c, s = a[..., 0], (-a[..., 1] if back else a[..., 1])
    lo, hi = K.float().chunk(2, -1)
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
@pytest.mark.parametrize("src", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("order", ["rows", "tokens", "fused"])
@pytest.mark.parametrize("rotate", [False, True])
def test_write(fmt, src, D, order, rotate):
    B, L, H, N, T = 2, 3, 3, 21, 16
    pool = ipv.PagePool.empty(12, 5, H, T, D, R.FORMATS[fmt])
    before = [t.clone() for t in (pool.K, pool.V)]
    table = R.shuffled_table(B, 5, 12, D)
    K, V = rows(src, B, L, H, N, D, D + N, order)
    first, ws = [0, 50], ipv.alloc_page_workspace("cuda")
    rotary = R.angles(80, D, "cuda") if rotate else None
    print("write", fmt, src, D, order, rotate, flush=True)
    ipv.ipv_page_write(pool, table, first, K, V, ws, first_layer=1, rotary=rotary)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0
    pos = torch.tensor(first, device="cuda")[:, None] + torch.arange(N, device="cuda")
    want_K = f32_turned(K, rotary, pos) if rotate else K.float()
    for name, want in (("K", want_K), ("V", V.float())):
        got = pool_rows(pool, fmt, table, name, 1, L, first, N)
        if fmt in KIND:
            assert torch.equal(got, want.to(KIND[fmt]).double())
        else:
            y, e = R.nearest_codes(want.double().reshape(-1, D), fmt)
            value = (y.reshape(-1, D // 32, 32) * torch.exp2(e)[..., None]).reshape(want.shape)
            assert torch.equal(got, value)
        if rotate and name == "K":  # and near the rotation in 64 bits: two roundings of products, one of the sum
            exact = R.turned(K.double(), rotary, pos)
            size = K.double().abs().max()
            assert float((want.double() - exact).abs().max()) <= 4 * 2.0**-24 * float(size) * 2
    # nothing else was written: other layers, other positions, other pages
    for t, b in zip((pool.K, pool.V), before):
        assert torch.equal(t[:, 0], b[:, 0]) and torch.equal(t[:, 4], b[:, 4])
        left = torch.ones(t.shape[0], T, dtype=torch.bool, device="cuda")
        for b_ in range(B):
            for p in range(first[b_], first[b_] + N):
                left[table[b_, p // T].long(), p % T] = False
        assert torch.equal(t.transpose(1, 3)[left], b.transpose(1, 3)[left])


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
@pytest.mark.parametrize("dst", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("order,rotate", [("rows", False), ("rows", True), ("fused", True)])
def test_read(fmt, dst, D, order, rotate):
    B, L, H, N, T = 2, 2, 5, 19, 12
    pool = R.filled_pool(fmt, 9, 3, H, T, D, D)
    table = R.shuffled_table(B, 4, 9, D)
    first, counts, ws = [0, 20], [19, 7], ipv.alloc_page_workspace("cuda")
    K, V = rows(dst, B, L, H, N, D, 5, order)
    keep = [K.clone(), V.clone()]
    rotary = R.angles(80, D, "cuda") if rotate else None
    print("read", fmt, dst, D, order, rotate, flush=True)
    ipv.ipv_page_read(pool, table, first, K, V, ws, rows=counts, first_layer=1, rotary=rotary)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0
    for b in range(B):
        pos = torch.arange(first[b], first[b] + counts[b], device="cuda")[None]
        for name, got, old in (("K", K, keep[0]), ("V", V, keep[1])):
            want = pool_rows(pool, fmt, table[b:b + 1], name, 1, L, [first[b]], counts[b]).float()
            if rotate and name == "K":
                want = f32_turned(want, rotary, pos, back=True)
            assert torch.equal(got[b, :, :, :counts[b]], want[0].to(KIND[dst]))
            assert torch.equal(got[b, :, :, counts[b]:], old[b, :, :, counts[b]:])


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_rounding_on_every_magnitude(fmt):
    """Blocks over the whole fp32 range: every tie, both sides of each, the type's largest value and one above, zeros, subnormals."""
    D = 32
    values = R.element_values(fmt)
    mags = values[values >= 0].unique()
    mids = (mags[1:] + mags[:-1]) / 2
    base = torch.cat((mags, mids, mids * (1 + 2.0**-20), mids * (1 - 2.0**-20))).float()
    base = torch.cat((base, -base))
    blocks = []
    for e in (-120, -100, -30, -3, 0, 1, 40, 110):
        for top in (R.TOP[fmt], R.TOP[fmt] * (1 - 2.0**-10), R.TOP[fmt] * 0.51):
            x = base[base.abs() <= top]
            x = torch.cat((x, torch.zeros(-len(x) % 31))).view(-1, 31)
            blocks.append(torch.cat((x, torch.full((len(x), 1), top)), 1) * 2.0**e)
    blocks.append(torch.full((1, 32), R.TOP[fmt] * (1 + 2.0**-22)))
    blocks.append(torch.zeros(1, 32))
    blocks.append(torch.full((1, 32), 1e-42))
    blocks.append(torch.full((1, 32), 3.0e38))
    x = torch.cat(blocks).float().cuda()
    N = len(x)
    pool = ipv.PagePool.empty(1, 1, 1, N, D, R.FORMATS[fmt])
    ws = ipv.alloc_page_workspace("cuda")
    K = x.view(1, 1, 1, N, D).contiguous()
    ipv.ipv_page_write(pool, None, 0, K, -K, ws)
    assert ipv.ipv_read_device_errors(ws) == 0
    y, e = R.nearest_codes(x.double(), fmt)
    want = (y.view(N, 1, 32) * torch.exp2(e)[..., None]).view(N, D)
    assert torch.equal(R.stored_values(pool.K, pool.K_scales, fmt).view(N, D), want)
    assert torch.equal(R.stored_values(pool.V, pool.V_scales, fmt).view(N, D), -want)
    assert torch.equal(pool.K_scales.view(N), (e[:, 0] + 127).to(torch.uint8))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("special", [math.inf, -math.inf, math.nan])
def test_blocks_of_infinities_and_nan(fmt, special):
    pool = ipv.PagePool.empty(2, 1, 2, 8, 128, R.FORMATS[fmt])
    ws = ipv.alloc_page_workspace("cuda")
    K, V = rows("bf16", 1, 1, 2, 8, 128, 3)
    want_K, want_V = K.clone(), V.clone()
    K[0, 0, 1, 3, 70] = special
    V[0, 0, 0, 5, 0] = special
    table = torch.tensor([[1]], dtype=torch.int32, device="cuda")
    ipv.ipv_page_write(pool, table, 0, K, V, ws)
    assert ipv.ipv_read_device_errors(ws) == ipv.DEV_NAN
    back = [torch.empty_like(K) for _ in range(2)]
    ipv.ipv_page_read(pool, table, 0, *back, ws)
    nan = torch.zeros(K.shape, dtype=torch.bool, device="cuda")
    nan[0, 0, 1, 3, 64:96] = True
    assert torch.equal(back[0].isnan(), nan)
    nan = torch.zeros(K.shape, dtype=torch.bool, device="cuda")
    nan[0, 0, 0, 5, :32] = True
    assert torch.equal(back[1].isnan(), nan)
    for got, want in zip(back, (want_K, want_V)):  # the other blocks: at most half a step off, and a step is at most 2^-2 (e2m1: 2^-1) of a value's size
        ok = ~got.isnan()
        limit = {"fp8": 2.0**-4, "fp4": 2.0**-1}[fmt]
        top = want.float().view(1, 1, 2, 8, 4, 32).abs().amax(-1, keepdim=True).expand(1, 1, 2, 8, 4, 32).reshape(want.shape)
        assert bool(((got.float() - want.float()).abs() <= limit * top)[ok].all())


def test_pages_outside_the_pool():
    for fmt in ("bf16", "fp8"):
        pool = R.filled_pool(fmt, 3, 1, 1, 8, 64, 1)
        old = pool.K.clone()
        table = torch.tensor([[0, 3, 2]], dtype=torch.int32, device="cuda")
        ws = ipv.alloc_page_workspace("cuda")
        K, V = rows("bf16", 1, 1, 1, 24, 64, 2)
        ipv.ipv_page_write(pool, table, 0, K, V, ws)
        assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE
        assert torch.equal(pool.K[1], old[1]) and not torch.equal(pool.K[0], old[0]) and not torch.equal(pool.K[2], old[2])
        ipv.ipv_clear_device_errors(ws)
        ipv.ipv_page_read(pool, table, 0, K, V, ws)
        assert ipv.ipv_read_device_errors(ws) == ipv.DEV_BAD_PAGE


def test_there_and_back():
    """Rows written rotated and read turned back: bf16 pages give each key back to its rounding, fp32 ones to the rotation's."""
    B, L, H, N, D = 2, 2, 2, 300, 128
    K, V = rows("f32", B, L, H, N, D, 9)
    rotary = R.angles(1000, D, "cuda")
    for fmt, limit in (("f32", 8 * 2.0**-24), ("bf16", 2.0**-8 + 2.0**-9), ("fp8", 2.0**-3)):
        pool = ipv.PagePool.empty(B * 8, L, H, 64, D, R.FORMATS[fmt])
        table = R.shuffled_table(B, 8, B * 8, 4)
        ws = ipv.alloc_page_workspace("cuda")
        ipv.ipv_page_write(pool, table, [0, 200], K, V, ws, rotary=rotary)
        k, v = torch.empty_like(K), torch.empty_like(V)
        ipv.ipv_page_read(pool, table, [0, 200], k, v, ws, rotary=rotary)
        pair = torch.hypot(*K.chunk(2, -1)).repeat(1, 1, 1, 1, 2)
        top = pair if fmt != "fp8" else pair.amax(-1, keepdim=True).expand_as(pair)
        assert bool(((k - K).abs() <= limit * top + 1e-30).all()), fmt
        if fmt == "f32":
            assert torch.equal(v, V)


def test_the_pass_reads_on_from_pages():
    """A cache goes to pages and back, and a compression pass on what comes back gives what it gives on the cache."""
    B, L, H, S, D = 1, 2, 2, 160, 64
    K, V = rows("bf16", B, L, H, S, D, 3)
    K, V = K.contiguous(), V.contiguous()
    fr = (torch.arange(S, device="cuda") // 16).int().expand(B, L, H, S).contiguous()
    pa = (torch.arange(S, device="cuda") % 16).int().expand(B, L, H, S).contiguous()
    pool = ipv.PagePool.empty(12, L, H, 16, D, ipv.PAGES_BF16)
    table, ws = R.shuffled_table(B, 10, 12, 1), ipv.alloc_page_workspace("cuda")
    ipv.ipv_page_write(pool, table, 0, K, V, ws)
    k, v = torch.zeros_like(K), torch.zeros_like(V)
    ipv.ipv_page_read(pool, table, 0, k, v, ws)
    assert torch.equal(k, K) and torch.equal(v, V)
    got = []
    for a, b in ((K, V), (k, v)):
        f, p = fr.clone(), pa.clone()
        ipv.Compressor(a, 4, 4, 80).compress(a, b, f, p, S, 0.5, 2)
        got.append((a[..., :80, :], b[..., :80, :], f[..., :80], p[..., :80]))
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_many_streams_and_counts():
    B, L, H, N, D, T = 300, 1, 2, 5, 32, 8
    K, V = rows("bf16", B, L, H, N, D, 3)
    counts, first = [b % 6 for b in range(B)], [b % 3 for b in range(B)]
    pool = ipv.PagePool.empty(B, L, H, T, D, ipv.PAGES_BF16)
    ws = ipv.alloc_page_workspace("cuda")
    ipv.ipv_page_write(pool, None, first, K, V, ws, rows=counts)
    k, v = torch.full_like(K, 5.0), torch.full_like(V, 5.0)
    ipv.ipv_page_read(pool, None, first, k, v, ws, rows=counts)
    inside = torch.arange(N, device="cuda") < torch.tensor(counts, device="cuda")[:, None]
    inside = inside[:, None, None, :, None]
    assert torch.equal(k, torch.where(inside, K, torch.full_like(K, 5.0)))
    assert torch.equal(v, torch.where(inside, V, torch.full_like(V, 5.0)))


def test_refused_calls_touch_nothing():
    pool = R.filled_pool("fp8", 6, 2, 2, 16, 64, 3)
    table, ws = R.shuffled_table(1, 3, 6, 1), ipv.alloc_page_workspace("cuda")
    K, V = rows("bf16", 1, 2, 2, 8, 64, 3)
    rotary = R.angles(10, 64, "cuda")
    q = torch.ones(1, 4, 3, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(q, 3.0), torch.full((1, 4, 3), 4.0, device="cuda")
    aws = ipv.alloc_attend_workspace(pool, 1, 4, 3)
    held = (pool.K, pool.V, pool.K_scales, pool.V_scales, K, V, ws, aws, out, lse)
    before = [t.clone() for t in held]
    W, Rd, A = ipv.ipv_page_write, ipv.ipv_page_read, ipv.ipv_attend
    for status, f, args, kw in (
            (ipv.ERR_SHAPE, W, (pool, table, 41, K, V, ws), {}),               # past the table's 48 rows
            (ipv.ERR_SHAPE, W, (pool, table, 0, K, V, ws), dict(rows=9)),
            (ipv.ERR_SHAPE, W, (pool, table, 0, K, V, ws), dict(first_layer=1)),
            (ipv.ERR_ARG, W, (pool, table, 5, K, V, ws), dict(rotary=rotary)),  # angles up to position 9
            (ipv.ERR_SHAPE, W, (pool, table, 0, K, V, ws), dict(rotary=rotary[:, :16])),
            (ipv.ERR_SHAPE, W, (pool, table, 0, K[:, :, :1], V[:, :, :1], ws), {}),
            (ipv.ERR_DTYPE, W, (pool, table, 0, K, V.float(), ws), {}),
            (ipv.ERR_DTYPE, W, (pool, table, 0, K.half(), V.half(), ws), {}),
            (ipv.ERR_SHAPE, W, (pool, table.repeat(2, 1), 0, K, V, ws), {}),
            (ipv.ERR_SHAPE, W, (pool, table.long(), 0, K, V, ws), {}),
            (ipv.ERR_ARG, W, (pool, table.cpu(), 0, K, V, ws), {}),
            (ipv.ERR_ARG, W, (pool, table, 0, K.cpu(), V, ws), {}),
            (ipv.ERR_SHAPE, W, (pool, table, [0, 0], K, V, ws), {}),
            (ipv.ERR_WORKSPACE, W, (pool, table, 0, K, V, None), {}),
            (ipv.ERR_WORKSPACE, Rd, (pool, table, 0, K, V, ws[:128]), {}),
            (ipv.ERR_SHAPE, Rd, (pool, table, 0, K.transpose(3, 4), V.transpose(3, 4), ws), {}),
            (ipv.ERR_SHAPE, Rd, (pool, table, 0, K, V.transpose(2, 3).contiguous().transpose(2, 3), ws), {}),
            (ipv.ERR_SHAPE, A, (pool, table, 49, 46, 0, q, out, aws), {}),
            (ipv.ERR_SHAPE, A, (pool, table, 40, 37, 2, q, out, aws), {}),
            (ipv.ERR_SHAPE, A, (pool, table, 40, 37, 0, q[:, :3], out[:, :3], aws), {}),
            (ipv.ERR_SHAPE, A, (pool, table, 40, 37, 0, q, out, aws), dict(q_rows=4)),
            (ipv.ERR_SHAPE, A, (pool, table, 40, 37, 0, q, out[:, :, :2], aws), {}),
            (ipv.ERR_DTYPE, A, (pool, table, 40, 37, 0, q.float(), out.float(), aws), {}),
            (ipv.ERR_DTYPE, A, (pool, table, 40, 37, 0, q, out, aws), dict(lse=lse.double())),
            (ipv.ERR_SHAPE, A, (pool, table, 40, 37, 0, q, out, aws), dict(lse=lse[:, :, :2])),
            (ipv.ERR_ARG, A, (pool, table, 40, 37, 0, q, out, aws), dict(scale=0.0)),
            (ipv.ERR_ARG, A, (pool, table, 40, 37, 0, q, out, aws), dict(window=-1)),
            (ipv.ERR_WORKSPACE, A, (pool, table, 40, 37, 0, q, out, ws), {}),
            (ipv.ERR_ARG, A, (pool, table, 40, 37, 0, q.cpu(), out, aws), {})):
        with pytest.raises(ipv.IpvError) as e:
            f(*args, **kw)
        assert e.value.status == status, (status, f.__name__, args[1:3], kw)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(held, before))
