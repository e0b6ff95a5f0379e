"""Tensors without rows, on the host: calls that do nothing, or are refused where rows are asked for all the same. The
tensors are the host's own, their addresses stand for a GPU's, and nothing is launched."""
import ctypes

import pytest
import torch

from paper_2506_15745_amd import ipv


@pytest.fixture
def host(monkeypatch):
    """(pool, workspace): of six pages of 2 layers, 2 heads and 32 rows of 64."""
    monkeypatch.setattr(ipv, "_ptr", lambda t: None if t is None else t.data_ptr() or None)
    monkeypatch.setattr(ipv, "_pool_stream", lambda pool, stream: None)
    monkeypatch.setattr(ipv, "_stream", lambda stream: None)
    p = object.__new__(ipv.PagePool)
    p._tensors = tuple(torch.zeros(6, 2, 2, 32, 64, dtype=torch.bfloat16) for _ in range(2)) + (None, None)
    p.format, p.head_dim, p.device, p.dtype = ipv.PAGES_BF16, 64, p._tensors[0].device, torch.bfloat16
    p.shape, p._dev = ipv.PageShape(6, 2, 2, 32, 64, ipv.PAGES_BF16), -1
    p._args = (ctypes.byref(p.shape), p._tensors[0].data_ptr(), p._tensors[1].data_ptr(), None, None)
    room = torch.zeros(1 << 22, dtype=torch.uint8)
    return p, room[-room.data_ptr() % 256:][:(1 << 22) - 256]


@pytest.mark.parametrize("rows,status", [(None, ipv.OK), (0, ipv.OK), ([0], ipv.OK), ([1], ipv.ERR_SHAPE), (1, ipv.ERR_SHAPE), ([-1], ipv.ERR_SHAPE)])
def test_compaction(host, rows, status):
    pool, ws = host
    keep, table = torch.zeros((1, 2, 2, 0), dtype=torch.int32), torch.zeros((1, 3), dtype=torch.int32)
    got = ipv.OK
    try:
        ipv.ipv_page_compact(pool, table, table, [40], keep, ws, rows=rows)
    except ipv.IpvError as e:
        got = e.status
    assert got == status


def attend(pool, ws, q, blocks, lse, **kw):
    ipv.ipv_attend(pool, torch.zeros((1, 3), dtype=torch.int32), [40], [5], 0, q, q, ws, lse=lse, **kw)


def attend_blocks(pool, ws, q, blocks, lse, **kw):
    ipv.ipv_attend_blocks(pool, torch.zeros((1, 3), dtype=torch.int32), [40], [5], 0, q, blocks, q, ws, block_rows=16, lse=lse, **kw)


def select(pool, ws, q, blocks, lse, **kw):
    bounds = object.__new__(ipv.BlockBounds)
    bounds.pool, bounds.block_rows, bounds._at = pool, 16, ws.data_ptr()
    ipv.ipv_block_select(pool, torch.zeros((1, 3), dtype=torch.int32), bounds, [40], [5], 0, q, blocks, ws, **kw)


@pytest.mark.parametrize("call", [attend, attend_blocks, select])
@pytest.mark.parametrize("rows,status", [(None, ipv.OK), (0, ipv.OK), ([0], ipv.OK), ([1], ipv.ERR_SHAPE), (1, ipv.ERR_SHAPE), ([-1], ipv.ERR_SHAPE)])
def test_queries(host, call, rows, status):
    """A query of tensors that hold none would be read from the workspace, and its result written there."""
    pool, ws = host
    got = ipv.OK
    try:
        call(pool, ws, torch.zeros((1, 4, 0, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 0, 5), dtype=torch.int32), torch.zeros((1, 4, 0)), q_rows=rows)
    except ipv.IpvError as e:
        got = e.status
    assert got == status
