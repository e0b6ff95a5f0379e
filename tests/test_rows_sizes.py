"""Sizes of the launches of new tokens, block bounds and compaction on the host: what no grid holds is refused before
anything is launched, also where only a later launch would not fit.

No call here gets as far as a kernel (these tests run without a GPU)."""
import pytest

from paper_2506_15745_amd import ipv
from tests.test_paged_abi import FAKE, shape
from tests.test_rows_abi import block_bounds, compact, qkv


def large(rows, D=128, T=None):
    return shape(pages=2, layers=1, kv_heads=1, page_rows=rows if T is None else T, head_dim=D, format=ipv.PAGES_FP4)


def counts(rows):
    """Of one stream, and of the last of 129: a launch of its own."""
    return (rows,), (0,) * 128 + (rows,)


# a workgroup has 4096 / D rows: 2^24 of them are 2^32 threads
@pytest.mark.parametrize("bounds,block", [(None, 0), (FAKE, 1 << 20)])
@pytest.mark.parametrize("D,rows", [(256, 2**28), (256, 2**28 - 15), (128, 2**29), (64, 2**30)])
def test_new_tokens(D, rows, bounds, block):
    top = 1 << 30
    for n in counts(rows):
        kw = dict(streams=len(n), cols=1, first=(0,) * len(n), layer=0, heads=1, bounds=bounds, block=block)
        assert qkv(s=large(top, D), rows=n, **kw) == ipv.ERR_SHAPE
        assert qkv(s=large(top, D), rows=(0,) * len(n), **kw) == ipv.OK


@pytest.mark.parametrize("first,rows", [(0, 2**28), (15, 2**28 - 15), (2**29, 2**29)])
def test_blocks_of_new_tokens_and_of_bounds(first, rows):
    """2^24 blocks of 16 rows, a workgroup each; a stream's first position may lie in a block's middle."""
    for n in counts(rows):
        at = tuple(first if x else 0 for x in n)
        assert block_bounds(s=large(1 << 30), streams=len(n), cols=1, first=at, rows=n, layers=1, block=16) == ipv.ERR_SHAPE
        if rows < 2**29:
            assert qkv(s=large(1 << 30), streams=len(n), cols=1, first=at, rows=n, layer=0, heads=1, block=16) == ipv.ERR_SHAPE


@pytest.mark.parametrize("bounds,block", [(None, 0), (FAKE, 1 << 20), (FAKE, 16)])
@pytest.mark.parametrize("rows", [2**29, 2**29 - 31, 2**30])
def test_compaction(rows, bounds, block):
    """Runs of 32 rows of values, whatever the blocks of the keys."""
    for n in counts(rows):
        kw = dict(s=large(1 << 30), streams=len(n), cols=1, new_cols=1, n=n, C=1 << 30, bounds=bounds, block=block)
        assert compact(rows=n, **kw) == ipv.ERR_SHAPE
        assert compact(rows=(0,) * len(n), **kw) == ipv.OK
