"""Selection of blocks with infinite bounds: the score is the sum of max(q lo, q hi), a product of 0 and an infinity counting
as 0, so that a channel in which every query has the other sign adds its finite product, and infinities count by their
signs; NaN is what a NaN bound or query, or infinities of both signs make. Every way of the selection, lists equal to the
last entry."""
import math

import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import blocks as X
from tests import paged as R
from tests.test_gpu_blocks import made_bounds, queries

pytestmark = pytest.mark.gpu


def defined(bounds, table, b, h, layer, q, blocks):
    """Scores [M, blocks] of one KV head by the definition, float64; q [G, M, D]."""
    q = q.double()

    def product(k):
        return torch.where(((q == 0) & k.isinf()) | (q.isinf() & (k == 0)), 0.0, q * k)

    return torch.stack([torch.maximum(product(k[0]), product(k[1])).sum((0, 2)) for k in
                        (X.bounds_at(bounds, table, b, layer, h, j).double() for j in range(blocks))], 1)


def ranked(score, count, top, first_blocks, last_blocks):
    """Lists [M, top]: those always picked, then NaN, then the highest, ties to the lower block."""
    j = torch.arange(score.shape[1], device=score.device)
    count = count[:, None]
    kind = torch.where(score.isnan(), 1, 0)
    kind = torch.where((j < first_blocks) | (j >= count - last_blocks), 2, kind)
    kind = torch.where(j < count, kind, -1)
    value = torch.where(score.isnan() | (kind != 0), 0.0, score)
    order = value.sort(dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, kind.gather(-1, order).sort(dim=-1, descending=True, stable=True).indices)[:, :top]
    order = torch.where(order < count, order, score.shape[1]).sort(-1).values
    return torch.nn.functional.pad(torch.where(order < score.shape[1], order, -1), (0, max(0, top - score.shape[1])), value=-1)


def check(fmt, pool, bounds, table, n, m, q, top, first_blocks, last_blocks):
    """The lists of the last m of n[b] positions."""
    B, A, _, D = q.shape
    H, R_ = pool.shape.kv_heads, bounds.block_rows
    print("infinite bounds", fmt, tuple(q.shape), n, R_, top, flush=True)
    ws = ipv.alloc_blocks_workspace(bounds, B, A, m, top, max(n))
    got = torch.full((B, H, m, top), 777, dtype=torch.int32, device="cuda")
    ipv.ipv_block_select(pool, table, bounds, n, [x - m for x in n], 0, q, got, ws, first_blocks=first_blocks, last_blocks=last_blocks)
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0 and bool((ws[256:4352] == 0).all())
    for b in range(B):
        blocks = -(-n[b] // R_)
        count = (torch.arange(n[b] - m, n[b], device="cuda") + R_) // R_
        for h in range(H):
            score = defined(bounds, table, b, h, 0, q[b, h * (A // H):(h + 1) * (A // H)], blocks)
            assert torch.equal(got[b, h].long(), ranked(score, count, top, first_blocks, last_blocks)), (b, h)
    return got


def test_a_channel_of_the_other_sign_adds_its_finite_product():
    """q = (-1, 2, 0, ..): a block of lo = (-1, -1), hi = (inf, 1) scores 1 + 2, less than others of 4 do."""
    T, D, N = 16, 32, 8
    pool = R.filled_pool("bf16", N, 1, 1, T, D, 3)
    table = torch.arange(N, dtype=torch.int32, device="cuda")[None]
    bounds, q = ipv.BlockBounds(pool, 16), torch.zeros((1, 1, 1, D), dtype=torch.bfloat16, device="cuda")
    q[..., 0], q[..., 1] = -1, 2
    bounds.values[:, 0, 0, 0, 0, 0] = -2
    bounds.values[:, 0, 0, 0, 1, 1] = 1  # 2 + 2
    bounds.values[2, 0, 0, 0, :, :2] = torch.tensor([[-1, -1], [math.inf, 1]])
    for top in (1, 3, 7):
        got = check("bf16", pool, bounds, table, [N * T], 1, q, top, 0, 0)
        assert 2 not in got.flatten().tolist()


def scattered(bounds, seed):
    """Random bounds with infinities of either sign, in either or both of them, in a few channels of a third of the blocks, NaN in a
    few, and one in eight of them a copy of another."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.randn(bounds.values.shape, generator=g, device="cuda").sort(dim=-2).values
    lo, hi = v.unbind(-2)
    p = torch.rand(lo.shape[:-1] + (1,), generator=g, device="cuda")
    x = torch.rand(lo.shape, generator=g, device="cuda")
    few = (p < 0.33) & (x < 2 / lo.shape[-1])
    kind = torch.randint(0, 5, lo.shape, generator=g, device="cuda")
    hi.masked_fill_(few & ((kind == 0) | (kind == 2)), math.inf)
    lo.masked_fill_(few & ((kind == 1) | (kind == 2)), -math.inf)
    for k, sign in ((3, 1), (4, -1)):  # all of a block's rows have that infinity there: now and then
        both = few & (kind == k) & (p < 0.03)
        lo.masked_fill_(both, sign * math.inf)
        hi.masked_fill_(both, sign * math.inf)
    hi.masked_fill_((p > 0.99) & (x < 1 / lo.shape[-1]), math.nan)
    flat = v.flatten(0, 3)
    copies = torch.rand(len(flat), generator=g, device="cuda") < 0.12
    flat[copies] = flat[torch.randint(0, len(flat), (int(copies.sum()),), generator=g, device="cuda")]
    bounds.values.copy_(flat.view(v.shape))


@pytest.mark.parametrize("fmt,D", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 128), ("f32", 256)])
@pytest.mark.parametrize("B,H,G,m,blocks", [
    (2, 2, 2, 1, 70),      # a workgroup a query
    (2, 2, 3, 3, 700),
    (1, 1, 2, 1, 2500),    # tiles of queries, their blocks shared out, scores read again
    (1, 2, 2, 40, 300),
    (1, 8, 2, 256, 150),   # tiles that take all blocks by themselves
    (1, 8, 1, 256, 600),
])
def test_infinities_anywhere(fmt, D, B, H, G, m, blocks):
    T, R_, n = 64, 16, [blocks * 16 - 5, blocks * 8 - 1][:B]
    cols = -(-n[0] // T)
    pool = R.filled_pool(fmt, B * cols, 1, H, T, D, 3)
    table = R.shuffled_table(B, cols, B * cols, 4)
    bounds = ipv.BlockBounds(pool, R_)
    scattered(bounds, blocks + D)
    q = queries(fmt, B, H * G, m, D, 9, token_major=True)
    q[:, ::2, ::3, 5] = 0  # of some heads, or of all (G = 1: of a group's only one)
    for top, first, last in ((9, 1, 2), (40, 0, 0)):
        check(fmt, pool, bounds, table, n, m, q, top, first, last)


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("m", [2, 300])
def test_queries_that_are_not_finite(value, m):
    """One head's element: NaN everywhere, or what an infinite query makes of either sign of a bound, and of a bound of 0."""
    T, D, H, G, blocks = 64, 64, 8, 2, 90
    n = blocks * 16 - 3
    pool, table = R.filled_pool("bf16", 23, 1, H, T, D, 3), R.shuffled_table(1, 23, 23, 4)
    bounds = ipv.BlockBounds(pool, 16)
    scattered(bounds, 5)
    lo, hi = bounds.values[..., 0, 7], bounds.values[..., 1, 7]  # [pages, 1, heads, blocks]
    lo[:, :, ::3], hi[:, :, ::3] = 0, hi[:, :, ::3].abs()
    lo[:, :, 1::3], hi[:, :, 1::3] = -lo[:, :, 1::3].abs(), -0.0
    q = queries("bf16", 1, H * G, m, D, 9)
    q[:, ::4, ::2, 7] = value
    check("bf16", pool, bounds, table, [n], m, q, 8, 1, 1)


@pytest.mark.parametrize("fmt", ("bf16", "f32"))
def test_keys_that_are_infinite(fmt):
    """Bounds as they are made of keys with infinities."""
    T, D, n, m = 64, 64, 900, 5
    pool, table = R.filled_pool(fmt, 15, 1, 2, T, D, 3), R.shuffled_table(1, 15, 15, 4)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.rand(pool.K.shape, generator=g, device="cuda")
    pool.K.masked_fill_(x < 3e-4, math.inf)
    pool.K.masked_fill_(x > 1 - 3e-4, -math.inf)
    bounds = made_bounds(pool, fmt, table, [n], 16)
    assert bool(torch.isinf(bounds.values).any())
    check(fmt, pool, bounds, table, [n], m, queries(fmt, 1, 4, m, D, 3), 12, 1, 1)
