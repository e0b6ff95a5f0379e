"""Arguments of the paged cache's calls at and beyond their ranges."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R

pytestmark = pytest.mark.gpu


def setup(fmt="fp8"):
    pool = R.filled_pool(fmt, 6, 2, 2, 16, 64, 3)
    table = R.shuffled_table(1, 3, 6, 1)
    q = torch.ones(1, 4, 3, 64, dtype=pool.dtype, device="cuda")
    return pool, table, q, torch.full_like(q, 3.0), ipv.alloc_attend_workspace(pool, 1, 4, 3), ipv.alloc_page_workspace("cuda")


@pytest.mark.parametrize("value", [2**32, -2**32, 2**32 + 1, 2**31, 2**63, 2**64])
def test_whole_numbers_beyond_32_bits(value):
    """Refused, not cut to their low 32 bits (a layer of 2^32 is not layer 0)."""
    pool, table, q, out, aws, ws = setup()
    K, V = (torch.ones(1, 1, 2, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    held = (pool.K, pool.V, pool.K_scales, pool.V_scales, K, V, out)
    before = [t.clone() for t in held]
    for f, args, kw in ((ipv.ipv_attend, (pool, table, 40, 37, value, q, out, aws), {}),
                        (ipv.ipv_attend, (pool, table, 40, 37, 0, q, out, aws), dict(window=value)),
                        (ipv.ipv_attend, (pool, table, 40, 37, 0, q, out, aws), dict(window=5, sinks=value)),
                        (ipv.ipv_attend, (pool, table, value, 37, 0, q, out, aws), {}),
                        (ipv.ipv_attend, (pool, table, [40], [value], 0, q, out, aws), {}),
                        (ipv.ipv_attend, (pool, table, 40, 37, 0, q, out, aws), dict(q_rows=[value])),
                        (ipv.ipv_page_write, (pool, table, 0, K, V, ws), dict(first_layer=value)),
                        (ipv.ipv_page_write, (pool, table, value, K, V, ws), {}),
                        (ipv.ipv_page_write, (pool, table, [value], K, V, ws), {}),
                        (ipv.ipv_page_write, (pool, table, 0, K, V, ws), dict(rows=value)),
                        (ipv.ipv_page_read, (pool, table, 0, K, V, ws), dict(rows=[value])),
                        (ipv.ipv_page_read, (pool, table, 0, K, V, ws), dict(first_layer=value)),
                        (ipv.attend_workspace_bytes, (pool, value, 4, 3), {}),
                        (ipv.attend_workspace_bytes, (pool, 1, value, 3), {}),
                        (ipv.attend_workspace_bytes, (pool, 1, 4, value), {})):
        with pytest.raises(ipv.IpvError) as e:
            f(*args, **kw)
        assert e.value.status in (ipv.ERR_SHAPE, ipv.ERR_ARG), (f.__name__, args[1:], kw)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(held, before))
