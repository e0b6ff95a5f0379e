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


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
def test_tensors_without_rows(fmt):
    """Nothing to write, to read or to ask: calls that do nothing, with the checks of the others."""
    pool, table, q, out, aws, ws = setup(fmt)
    before = [t.clone() for t in (pool.K, pool.V)]
    K, V = (torch.ones(1, 2, 2, 0, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for f in (ipv.ipv_page_write, ipv.ipv_page_read):
        f(pool, table, 5, K, V, ws)
        f(pool, table, 5, K, V, ws, rows=[0], rotary=R.angles(1, 64, "cuda"))
        f(pool, table, 5, *(torch.ones(1, 2, 2, 8, 64, device="cuda")[:, :, :, 8:] for _ in range(2)), ws)
        for args, kw in (((pool, table, 5, K, V, ws), dict(rows=1)), ((pool, table, 5, K, V, ws), dict(first_layer=1)),
                         ((pool, table, [5, 5], K, V, ws), {}), ((pool, table, -1, K, V, ws), {})):
            with pytest.raises(ipv.IpvError) as e:
                f(*args, **kw)
            assert e.value.status == ipv.ERR_SHAPE
    lse = torch.empty(1, 4, 0, device="cuda")
    for lse in (None, lse):
        ipv.ipv_attend(pool, table, 40, 40, 1, q[:, :, :0], out[:, :, :0], aws, lse=lse)
    for args in ((pool, table, 40, 40, 2), (pool, table, 49, 40, 0)):
        with pytest.raises(ipv.IpvError) as e:
            ipv.ipv_attend(*args, q[:, :, :0], out[:, :, :0], aws)
        assert e.value.status == ipv.ERR_SHAPE
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0 and ipv.ipv_read_device_errors(aws) == 0
    assert all(torch.equal(a, b) for a, b in zip((pool.K, pool.V), before)) and bool((out == 3.0).all())


def test_a_table_of_no_angles():
    """Rows cannot be turned by a table without positions (and are not left as they are)."""
    pool, table, q, out, aws, ws = setup("bf16")
    K, V = (torch.ones(1, 2, 2, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    before = pool.K.clone()
    for f in (ipv.ipv_page_write, ipv.ipv_page_read):
        with pytest.raises(ipv.IpvError) as e:
            f(pool, table, 0, K, V, ws, rotary=R.angles(10, 64, "cuda")[:0])
        assert e.value.status == ipv.ERR_ARG
    torch.cuda.synchronize()
    assert torch.equal(pool.K, before) and bool((K == 1).all())


def test_results_into_expanded_tensors():
    """Rows and queries may be expanded, results may not: their elements would be the same memory."""
    pool, table, q, out, aws, ws = setup("bf16")
    one = torch.ones(1, 2, 2, 1, 64, dtype=torch.bfloat16, device="cuda")
    ipv.ipv_page_write(pool, table, 0, *(one.expand(1, 2, 2, 8, 64),) * 2, ws)
    got = [torch.zeros(1, 2, 2, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ipv.ipv_page_read(pool, table, 0, *got, ws)
    assert all(bool((x == 1).all()) for x in got)
    ipv.ipv_attend(pool, table, 40, 37, 0, q[:, :, :1].expand(q.shape), out, aws)
    for f, args in ((ipv.ipv_page_read, (pool, table, 0, *(one.expand(1, 2, 2, 8, 64),) * 2, ws)),
                    (ipv.ipv_attend, (pool, table, 40, 37, 0, q, q[:, :, :1].expand(q.shape), aws)),
                    (ipv.ipv_attend, (pool, table, 40, 37, 0, q[:, :1].expand(q.shape), q[:, :1].expand(q.shape), aws))):
        with pytest.raises(ipv.IpvError) as e:
            f(*args)
        assert e.value.status == ipv.ERR_SHAPE
    torch.cuda.synchronize()
    assert bool((one == 1).all()) and bool((q == 1).all())
    # a dimension of one may have any stride
    ipv.ipv_attend(pool, table, 40, 39, 0, q[:, :, :1], out[:, :, :1].as_strided((1, 4, 1, 64), (0, 192, 0, 1)), aws)


def test_a_pools_tensors_stay():
    """A pool's addresses are taken when it is made, so its tensors cannot be exchanged under it."""
    pool, *_ = setup()
    held = [pool.K, pool.V, pool.K_scales, pool.V_scales]
    for name in ("K", "V", "K_scales", "V_scales"):
        with pytest.raises(AttributeError):
            setattr(pool, name, torch.zeros_like(pool.K))
    assert all(a is b for a, b in zip(held, (pool.K, pool.V, pool.K_scales, pool.V_scales)))
