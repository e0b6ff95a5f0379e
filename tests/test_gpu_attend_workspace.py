"""ipv_attend in a workspace of exactly the size it asks for: nothing is written past it, and only its first 4352 bytes
need be zero."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R
from tests.test_gpu_attend import queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("B,H,G,m", [(1, 1, 1, 1), (1, 4, 7, 1), (1, 2, 8, 4), (1, 4, 7, 35), (1, 1, 3, 400), (3, 2, 5, 1), (5, 1, 9, 60), (80, 1, 4, 1), (1, 8, 8, 150)])
def test_nothing_past_the_workspace(fmt, D, B, H, G, m):
    n, T = 9001 if B == 1 else 3000, 64
    cols = -(-n // T)
    pool = R.filled_pool(fmt, cols, 1, H, T, D, 3)
    table = torch.arange(cols, device="cuda").int().repeat(B, 1)
    q = queries(fmt, B, H * G, m, D, 4)
    size = ipv.attend_workspace_bytes(pool, B, H * G, m)
    room = torch.full((size + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    print("workspace", fmt, D, B, H, G, m, size, flush=True)
    got = []
    for fill in (0, 0xa5, 0xff):
        ws = room[:size]
        ws.fill_(fill)
        ws[:4352] = 0
        out, lse = torch.empty_like(q), torch.empty(B, H * G, m, device="cuda")
        for _ in range(2):
            ipv.ipv_attend(pool, table, n, n - m, 0, q, out, ws, lse=lse)
        assert ipv.ipv_read_device_errors(ws) == 0 and not bool(ws[:4352].any())
        got.append((out, lse))
    assert bool((room[size:] == 0xa5).all())
    for out, lse in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1])
    with pytest.raises(ipv.IpvError) as e:
        ipv.ipv_attend(pool, table, n, n - m, 0, q, out, room[:size - 1], lse=lse)
    assert e.value.status == ipv.ERR_WORKSPACE
