"""ipv_attend row by row: queries that put all their weight on one row give that row of V, so that a row lost, doubled or
taken from its neighbour anywhere in a long range (at a tile's, page's or part's end) is seen as such."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R
from tests.test_gpu_attend import check, queries

pytestmark = pytest.mark.gpu


def sign_pool(fmt, pages, H, T, D, seed):
    """Keys of +-1 (scales of 1), so that 8 times a key gives a score of 8 sqrt(D) with itself and 8 N(0, 1) with
    others; random values."""
    pool = R.filled_pool(fmt, pages, 1, H, T, D, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    sign = torch.randint(0, 2, (pages, 1, H, T, D), generator=g, device="cuda")
    if fmt in ("bf16", "f32"):
        pool.K.copy_(1 - 2 * sign)
    else:
        code = (0x38 | sign << 7) if fmt == "fp8" else (2 | sign << 3)
        if fmt == "fp4":
            code = code[..., ::2] | code[..., 1::2] << 4
        pool.K.copy_(code.to(torch.uint8))
        pool.K_scales.fill_(127)
    return pool


def needle_limit(fmt, V):
    """The weights of all other rows sum to less than n e^-40. fp32: rounding of sums. bf16: the row's weight may be rounded
    (2^-8 of it at most) and so is the result."""
    return V.abs() * (1e-5 if fmt == "f32" else 2 * 2.0**-8) + 1e-9


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
@pytest.mark.parametrize("T", [64, 100])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("G,m", [(4, 4), (8, 4), (2, 300)])
def test_every_row_of_a_long_range(fmt, T, D, G, m):
    n, H = 5003, 2
    cols = -(-n // T)
    pool = sign_pool(fmt, cols + 2, H, T, D, T + G)
    table = R.shuffled_table(1, cols, cols + 2, m)
    K, V = (torch.stack([R.rows_of(pool, fmt, table, 0, 0, h, name)[:n] for h in range(H)]) for name in "KV")
    kind = torch.float32 if fmt == "f32" else torch.bfloat16
    ws = ipv.alloc_attend_workspace(pool, 1, H * G, m)
    print("needles", fmt, T, D, G, m, flush=True)
    for j0 in range(0, n, G * m):
        rows = torch.arange(j0, j0 + G * m, device="cuda") % n
        q = (8 * K[:, rows]).to(kind).view(1, H * G, m, D)
        out = torch.empty_like(q)
        ipv.ipv_attend(pool, table, n, n, 0, q, out, ws)
        want = V[:, rows].view(1, H * G, m, D)
        assert bool(((out.double() - want).abs() <= needle_limit(fmt, want)).all()), j0
    assert ipv.ipv_read_device_errors(ws) == 0


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
@pytest.mark.parametrize("T", [36, 128])
def test_rows_of_a_window(fmt, T):
    """The same under a window and first rows: each query at the oldest and newest row that it sees, and the first ones."""
    n, H, G, m, D, window, sinks = 4000, 2, 3, 256, 128, 700, 90
    cols = -(-n // T)
    pool = sign_pool(fmt, cols + 2, H, T, D, T)
    table = R.shuffled_table(1, cols, cols + 2, m)
    K, V = (torch.stack([R.rows_of(pool, fmt, table, 0, 0, h, name)[:n] for h in range(H)]) for name in "KV")
    kind = torch.float32 if fmt == "f32" else torch.bfloat16
    p = torch.arange(n - m, n, device="cuda")
    for some in (m, 5, 1):
        at = p[-some:]
        for rows in (at, at - window + 1, at - window // 2, at % sinks, torch.full_like(at, sinks - 1)):
            q = (8 * K[:, rows]).to(kind)[:, None].expand(H, G, some, D).reshape(1, H * G, some, D)
            out, ws = torch.empty_like(q), ipv.alloc_attend_workspace(pool, 1, H * G, some)
            ipv.ipv_attend(pool, table, n, n - some, 0, q, out, ws, window=window, sinks=sinks)
            want = V[:, rows][:, None].expand(H, G, some, D).reshape(1, H * G, some, D)
            assert bool(((out.double() - want).abs() <= needle_limit(fmt, want)).all())


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
@pytest.mark.parametrize("T", [64, 100])
@pytest.mark.parametrize("window,sinks", [(0, 0), (600, 30)])
def test_streams_with_different_numbers_of_queries(fmt, T, window, sinks):
    """A chunk beside single tokens, few tokens and a stream without any, over long ranges."""
    n, rows, D, H, G, M = [3000, 4100, 700, 2500, 0], [300, 1, 0, 5, 2], 128, 2, 3, 300
    cols = -(-max(n) // T)
    pool = R.filled_pool(fmt, 60 * 64 // T, 1, H, T, D, 4)
    table = (torch.randint(0, 60 * 64 // T, (5, cols), generator=torch.Generator().manual_seed(T))).int().cuda()
    q = queries(fmt, 5, H * G, M, D, 6)
    check(fmt, pool, table, n, [x - r if x else 0 for x, r in zip(n, rows)], 0, q, window, sinks, rows=rows)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("T", [64, 100])
def test_rows_of_streams_with_different_numbers_of_queries(fmt, T):
    """The same, row by row of V: every stream's queries at rows of its own, all over its range."""
    n, rows, D, H, G, M = [3000, 4100, 700, 2500], [300, 1, 0, 5], 128, 2, 3, 300
    cols = -(-max(n) // T)
    pool = sign_pool(fmt, 4 * cols, H, T, D, 4)
    table = R.shuffled_table(4, cols, 4 * cols, T)
    q = torch.zeros(4, H * G, M, D, dtype=torch.bfloat16, device="cuda")
    want = torch.zeros(4, H * G, M, D, dtype=torch.float64, device="cuda")
    for k in range(4):
        at = torch.zeros(4, H * G, M, dtype=torch.long)
        g = torch.Generator().manual_seed(k)
        for b in range(4):
            at[b, :, :rows[b]] = torch.randint(0, n[b], (H * G, rows[b]), generator=g)
            for a in range(H * G):
                K, V = (R.rows_of(pool, fmt, table, b, 0, a // G, name) for name in "KV")
                j = at[b, a, :rows[b]].cuda()
                q[b, a, :rows[b]] = (8 * K[j]).bfloat16()
                want[b, a, :rows[b]] = V[j]
        out, ws = torch.zeros_like(q), ipv.alloc_attend_workspace(pool, 4, H * G, M)
        ipv.ipv_attend(pool, table, n, n, 0, q, out, ws, q_rows=rows)
        assert bool(((out.double() - want).abs() <= needle_limit(fmt, want)).all())
