"""Compaction that keeps no row: a call that does nothing, and a stream's pages that all go back."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import blocks as X
from tests import paged as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("rows", [None, 0, [0, 0]])
def test_no_rows(fmt, rows):
    pool = R.filled_pool(fmt, 6, 2, 2, 32, 64, 3)
    table, bounds, ws = R.shuffled_table(2, 2, 6, 4), ipv.BlockBounds(pool, 16), ipv.alloc_page_workspace("cuda")
    bounds.values.fill_(777)
    before = [t.clone() for t in X.raw(pool)]
    keep = torch.empty((2, 2, 2, 0), dtype=torch.int32, device="cuda")
    ipv.ipv_page_compact(pool, table, table[:, :1].contiguous(), [40, 0], keep, ws, rows=rows, bounds=bounds, rotary=R.angles(64, 64, "cuda"))
    torch.cuda.synchronize()
    assert ipv.ipv_read_device_errors(ws) == 0 and bool((bounds.values == 777).all())
    assert all(torch.equal(x, y) for x, y in zip(before, X.raw(pool)))


def test_rows_of_no_room_are_refused():
    pool = R.filled_pool("bf16", 6, 2, 2, 32, 64, 3)
    table, ws = R.shuffled_table(2, 2, 6, 4), ipv.alloc_page_workspace("cuda")
    keep = torch.empty((2, 2, 2, 0), dtype=torch.int32, device="cuda")
    with pytest.raises(ipv.IpvError) as e:
        ipv.ipv_page_compact(pool, table, table, [40, 0], keep, ws, rows=[1, 0])
    assert e.value.status == ipv.ERR_SHAPE


def test_a_stream_that_keeps_nothing():
    pool = R.filled_pool("bf16", 6, 2, 2, 32, 64, 3)
    t, ws = ipv.PageTables(pool, 2, 3), ipv.alloc_page_workspace("cuda")
    t.reserve(0, [40, 10], ws)
    assert t.free_pages == 3
    t.compact([0], 40, torch.empty((1, 2, 2, 0), dtype=torch.int32, device="cuda"), ws)
    assert t.pages[0] == [] and len(t.pages[1]) == 1 and t.free_pages == 5
    assert t.table[0].tolist() == [-1] * 3 and ipv.ipv_read_device_errors(ws) == 0
