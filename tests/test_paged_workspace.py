"""What ipv_attend's workspace takes: no more than the parts that calls of its sizes can make."""
import ctypes

import pytest

from paper_2506_15745_amd import ipv
from tests.test_paged_abi import shape

MIB = 1 << 20


def need(streams=1, heads=28, rows=1, **kw):
    size = ctypes.c_size_t(0)
    s = shape(**kw)
    assert ipv._paged().ipv_attend_workspace_bytes(ctypes.byref(s), streams, heads, rows, ctypes.byref(size)) == ipv.OK
    return size.value


def parts(streams, kv_heads, tiles, rows, D):
    """Bytes of the parts of `tiles` row tiles of `rows` rows a stream and KV head, each in 64 parts at most, 1024 in all."""
    return min(1024, min(streams, 64) * kv_heads * tiles * 64) * rows * (D + 2) * 4


@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("streams", [1, 3, 70])
def test_small_calls_take_little(D, streams):
    head = 256 + 4 * 1024
    tile = 256 if D <= 128 else 128
    for fmt in (ipv.PAGES_BF16, ipv.PAGES_FP8, ipv.PAGES_FP4):
        few1 = parts(streams, 4, 1, 16, D)
        few2 = parts(streams, 4, 1, 32, D)
        assert need(streams, 28, 1, head_dim=D, format=fmt) == head + few1                # 7 rows
        assert need(streams, 28, 4, head_dim=D, format=fmt) == head + max(few1, few2)     # 28 rows
        got = head + max(few1, few2, parts(streams, 4, -(-245 // tile), tile, D))         # 245 rows: a question
        assert need(streams, 28, 35, head_dim=D, format=fmt) == got
    assert need(streams, 28, 35, head_dim=D, format=ipv.PAGES_F32) == head + parts(streams, 4, 8, 32, D)


def test_a_question():
    """35 tokens of 28 query and 4 KV heads of 128, one stream."""
    assert need(1, 28, 35) < 33 * MIB
    assert need(1, 28, 1) < 3 * MIB


def test_a_workspace_serves_smaller_calls():
    """One for more streams, heads and rows is large enough for fewer of each."""
    for fmt in range(4):
        for D in (32, 256):
            for B in (1, 2, 5, 64, 200):
                for heads in (4, 8, 28):
                    for rows in (1, 2, 4, 5, 9, 33, 300):
                        n = need(B, heads, rows, head_dim=D, format=fmt)
                        for b, h, r in ((B + 1, heads, rows), (B, heads + 4, rows), (B, heads, rows + 1), (B, heads, 2 * rows)):
                            assert need(b, h, r, head_dim=D, format=fmt) >= n
