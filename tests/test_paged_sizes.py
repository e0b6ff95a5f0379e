"""Sizes of the paged cache's launches on the host: what no grid holds is refused before anything is launched.

No call here gets as far as a kernel (these tests run without a GPU)."""
import ctypes

import pytest

from paper_2506_15745_amd import ipv
from tests.test_paged_abi import attend_call, rows_call, shape


@pytest.mark.parametrize("fmt", [ipv.PAGES_BF16, ipv.PAGES_F32, ipv.PAGES_FP8, ipv.PAGES_FP4])
@pytest.mark.parametrize("heads,rows", [
    (2**26, (1,) * 64),                # 2^32 workgroups, one row each
    (2**27, (1,) * 64),
    (2**24, (1,)),                     # 2^24 of them: 2^32 threads
    (2**24 - 3, (1,)),                 # with those that make the number a multiple of eight
    (2**22, (1, 1, 0, 1, 1)),
    (2**18, (0,) * 64 + (1,) * 64),    # the second launch's
])
def test_more_workgroups_than_a_grid_holds(fmt, heads, rows):
    s = shape(pages=1, layers=1, kv_heads=heads, page_rows=1, head_dim=32, format=fmt)
    B = len(rows)
    assert attend_call(s=s, streams=B, cols=1, n=(1,) * B, first=(0,) * B, rows=rows, layer=0, heads=heads) == ipv.ERR_SHAPE


def test_a_launch_after_one_that_fits():
    """Single tokens in the first launch (2^31 threads), chunks of twice the threads a workgroup in the second."""
    s = shape(pages=1, layers=1, kv_heads=2**17, page_rows=64, head_dim=128, format=ipv.PAGES_BF16)
    rows = (1,) * 64 + (33,) * 64
    assert attend_call(s=s, streams=128, cols=1, n=(33,) * 128, first=(0,) * 128, rows=rows, layer=0, heads=2**17, most=33) == ipv.ERR_SHAPE


@pytest.mark.parametrize("name", ["ipv_page_write", "ipv_page_read"])
@pytest.mark.parametrize("D,rows", [(256, 2**28), (256, 2**28 - 15), (128, 2**29), (64, 2**30)])
def test_more_rows_than_a_grid_holds(name, D, rows):
    s = shape(pages=2, layers=1, kv_heads=1, page_rows=rows, head_dim=D, format=ipv.PAGES_FP4)
    for first, counts in (((0,), (rows,)), ((0,) * 129, (0,) * 128 + (rows,))):
        assert rows_call(name, s=s, streams=len(first), cols=1, first=first, rows=counts, layers=1) == ipv.ERR_SHAPE
