"""Attention over lists with a wave a query, at every head size and both widths of a group of heads."""
import pytest

from tests import paged as R
from tests.test_gpu_blocks import check, made_bounds, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "f32", "fp8", "fp4"])
@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("G", [3, 20, 33])
def test_every_head_size(fmt, D, G):
    """1280 queries over lists of three blocks of 48 rows: a wave each is the faster way for all of them (more queries than
    workgroups that the card holds, five key tiles), and a list's last key tile is half empty."""
    B, H, M, n = 2, 8, 80, [700, 395]
    pool, table = R.filled_pool(fmt, 24, 1, H, 96, D, D + G), R.shuffled_table(B, 8, 24, 3)
    check(fmt, pool, table, n, [x - M for x in n], 0, queries(fmt, B, H * G, M, D, 8, token_major=True), made_bounds(pool, fmt, table, n, 48),
          3, 1, 1)
