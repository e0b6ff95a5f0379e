"""The largest weight of a softmax in the kernels of up to 32 rows: exactly 1, so that a row of V that outweighs the
others is not rounded before the result is."""
import math

import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("D", [64, 256])
@pytest.mark.parametrize("G", [16, 20, 32])
def test_the_largest_weight_is_not_rounded(fmt, D, G):
    """Keys of zero but for one, in a later tile, whose score is 1 to 5 above theirs; V zero but for it. So many streams that
    no key range is split: a wave has several tiles, and meets that key after others."""
    B, H, T, n, row = 64, 12, 64, 512, 437
    pool = ipv.PagePool.empty(n // T, 1, H, T, D, R.FORMATS[fmt])
    at = (row // T, 0, slice(None), row % T)
    g = torch.Generator(device="cuda").manual_seed(G)
    if fmt == "bf16":
        pool.K[at] = 1.0
        pool.V[at] = torch.randn(H, D, generator=g, device="cuda").bfloat16()
    else:
        pool.K[at] = 0x38 if fmt == "fp8" else 0x22
        pool.V[at] = torch.randint(1, 256, (H, pool.V.shape[-1]), generator=g, device="cuda", dtype=torch.uint8) & (0xbf if fmt == "fp8" else 0xff)
        pool.K_scales.fill_(127), pool.V_scales.fill_(127)
    table = torch.arange(n // T, device="cuda").int().expand(B, n // T).contiguous()
    step = (1 + 4 * torch.arange(H * G, device="cuda") / (H * G))  # scores
    q = torch.zeros(B, H * G, 1, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = (step * math.sqrt(D)).bfloat16()[:, None]
    x = q[0, :, 0, 0].double() / math.sqrt(D)
    out, ws = torch.empty_like(q), ipv.alloc_attend_workspace(pool, B, H * G, 1)
    print("weights", fmt, D, G, flush=True)
    ipv.ipv_attend(pool, table, n, n, 0, q, out, ws)
    V = torch.stack([R.rows_of(pool, fmt, table, 0, 0, h, "V")[row] for h in range(H)]).repeat_interleave(G, 0)
    want = V * (torch.exp(x) / (torch.exp(x) + n - 1))[:, None]
    # the result's rounding to bf16, half a step; scores, exponentials and sums in fp32
    half = torch.exp2(torch.floor(torch.log2(want.abs().clamp_min(1e-30))) - 8)
    off = (out[:, :, 0].double() - want).abs() - (half + 2e-5 * want.abs())
    assert float(off.max()) <= 0, float(off.max())
