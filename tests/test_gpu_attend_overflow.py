"""Quantised values beyond bf16's range (a scale of 2^127 and an element of 2, as another program may have
written it, or what the largest fp32 values round to): infinite to the queries that see them, nothing to the others."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R

pytestmark = pytest.mark.gpu

# (scale byte, code) pairs whose value is 2^128 or more, least ones first; and the largest that are not
BEYOND = {"fp8": [(247, 0x78), (247, 0x7e), (250, 0x60), (254, 0x40), (254, 0xc0), (254, 0x7e)], "fp4": [(253, 6), (253, 7), (254, 4), (254, 15)]}
WITHIN = {"fp8": [(246, 0x7e), (254, 0x3f), (250, 0x5f), (246, 0xfe)], "fp4": [(252, 7), (253, 5), (254, 3), (254, 11)]}


def attend(pool, table, n, first, q, window, sinks):
    ws = ipv.alloc_attend_workspace(pool, *q.shape[:3])
    out = torch.empty_like(q)
    ipv.ipv_attend(pool, table, n, first, 0, q, out, ws, window=window, sinks=sinks)
    assert ipv.ipv_read_device_errors(ws) == 0
    return out


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("T", [12, 64])
@pytest.mark.parametrize("m", [1, 4, 40])
def test_values_beyond_bf16(fmt, D, T, m):
    n, window, sinks, cols = 150, 20, 3, -(-192 // T)
    G = 4
    q = torch.randn((1, G, m, D), generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    table = R.shuffled_table(1, cols, cols + 1, 2)
    for kind, pairs in (("beyond", BEYOND[fmt]), ("within", WITHIN[fmt])):
        for byte, code in pairs:
            pool, plain = (R.filled_pool(fmt, cols + 1, 1, 1, T, D, 3) for _ in range(2))
            print("overflow", fmt, D, T, m, kind, byte, code, flush=True)
            # in rows past the last and before the window, and in a new token's own row, which later queries see
            own = n - 1 - m // 2
            hidden = [n, n + 1, min(n + 20, cols * T - 1), sinks, n - m - window]
            for row in hidden + [own] * (kind == "beyond"):
                at = (int(table[0, row // T]), 0, 0, row % T)
                pool.V[at][3] = code if fmt == "fp8" else (code | code << 4)
                pool.V_scales[at] = byte
                plain.V[at] = 0  # what the others make of it: nothing
            want, got = (attend(p, table, n, n - m, q, window, sinks) for p in (plain, pool))
            p = torch.arange(n - m, n, device="cuda")
            sees = (p >= own) & (own > p - window) & (kind == "beyond")
            assert torch.equal(got[:, :, ~sees], want[:, :, ~sees])
            if kind == "beyond":
                at = 3 if fmt == "fp8" else 6
                x = got[:, :, sees, at]
                assert bool((x == (-float("inf") if code & (0x80 if fmt == "fp8" else 8) else float("inf"))).all())


@pytest.mark.parametrize("fmt,least,below", [("fp8", 1.9375, 1.875), ("fp4", 1.75, 1.5)])
def test_the_largest_values_round_to_infinity(fmt, least, below):
    """From half a step below 2^128 on, as in every type of this exponent range."""
    D = 64
    x = torch.zeros(1, 1, 1, 4, D, device="cuda")
    x[..., 0, 5], x[..., 1, 40], x[..., 2, 7], x[..., 3, 63] = least * 2.0**127, -3.4e38, least * (1 - 2.0**-22) * 2.0**127, -least * (1 - 2.0**-20) * 2.0**127
    pool, ws = ipv.PagePool.empty(1, 1, 1, 4, D, R.FORMATS[fmt]), ipv.alloc_page_workspace("cuda")
    ipv.ipv_page_write(pool, None, 0, x, -x, ws)
    assert ipv.ipv_read_device_errors(ws) == 0
    want = torch.zeros_like(x)
    want[..., 0, 5], want[..., 1, 40], want[..., 2, 7], want[..., 3, 63] = float("inf"), -float("inf"), below * 2.0**127, -below * 2.0**127
    for kind in (torch.float32, torch.bfloat16):
        k, v = (torch.empty(1, 1, 1, 4, D, dtype=kind, device="cuda") for _ in range(2))
        ipv.ipv_page_read(pool, None, 0, k, v, ws)
        assert torch.equal(k, want.to(kind)) and torch.equal(v, -want.to(kind))
