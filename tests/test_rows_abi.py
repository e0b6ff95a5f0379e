"""New tokens, block bounds, selection, lists, compaction and copies on the host: what the calls refuse, before
anything is launched.

Every call here carries at least one argument that the host checks reject, or
has nothing to do, so no kernel is enqueued (these tests run without a GPU)."""
import ctypes
import math

import pytest
import torch

from paper_2506_15745_amd import ipv
from tests.test_paged_abi import BIG, FAKE, ints, longs, shape

ROW = (1 << 16, 128, 4096)


def at(v, kind=ints):
    return None if v is None else kind(*v)


def qkv(s=None, K=FAKE, V=FAKE, Ks=FAKE, Vs=FAKE, bounds=FAKE, block=32, table=FAKE, cols=10, streams=2, first=(0, 5), rows=(7, 9), layer=3,
        q=FAKE, qs=ROW, heads=28, k=FAKE, v=FAKE, ks=ROW, dtype=ipv.BF16, qn=FAKE, kn=FAKE, eps=1e-6, rotary=None, angles=0, out=FAKE,
        os=ROW, ws=FAKE, ws_bytes=BIG):
    s = shape() if s is None else s
    return ipv._paged().ipv_qkv_write(ctypes.byref(s), K, V, Ks, Vs, bounds, block, table, cols, streams, at(first), at(rows), layer, q,
                                      at(qs, longs), heads, k, v, at(ks, longs), dtype, qn, kn, eps, rotary, angles, out, at(os, longs), ws,
                                      ws_bytes, None)


POOL = [
    (dict(K=None), ipv.ERR_NULL),
    (dict(Ks=None), ipv.ERR_NULL),
    (dict(K=FAKE + 8), ipv.ERR_ALIGN),
    (dict(table=FAKE + 2), ipv.ERR_ALIGN),
    (dict(bounds=FAKE + 8), ipv.ERR_ALIGN),
    (dict(block=0), ipv.ERR_SHAPE),
    (dict(block=-16), ipv.ERR_SHAPE),
    (dict(block=8), ipv.ERR_SHAPE),
    (dict(block=48), ipv.ERR_SHAPE),    # does not divide 64
    (dict(block=128), ipv.ERR_SHAPE),   # larger than a page
    (dict(s=shape(page_rows=24), block=24), ipv.ERR_SHAPE),  # no multiple of 16
    (dict(s=shape(format=4)), ipv.ERR_DTYPE),
    (dict(s=shape(head_dim=96)), ipv.ERR_SHAPE),
    (dict(streams=0), ipv.ERR_SHAPE),
    (dict(cols=0), ipv.ERR_SHAPE),
    (dict(table=None, cols=10), ipv.ERR_SHAPE),
    (dict(ws=None), ipv.ERR_WORKSPACE),
    (dict(ws=FAKE + 16), ipv.ERR_ALIGN),
    (dict(ws_bytes=255), ipv.ERR_WORKSPACE),
]


@pytest.mark.parametrize("case,status", POOL + [
    (dict(V=None), ipv.ERR_NULL),
    (dict(first=None), ipv.ERR_NULL),
    (dict(rows=None), ipv.ERR_NULL),
    (dict(q=None), ipv.ERR_NULL),
    (dict(k=None), ipv.ERR_NULL),
    (dict(v=None), ipv.ERR_NULL),
    (dict(out=None), ipv.ERR_NULL),
    (dict(qs=None), ipv.ERR_NULL),
    (dict(ks=None), ipv.ERR_NULL),
    (dict(os=None), ipv.ERR_NULL),
    (dict(q=FAKE + 8), ipv.ERR_ALIGN),
    (dict(out=FAKE + 8), ipv.ERR_ALIGN),
    (dict(qn=FAKE + 2), ipv.ERR_ALIGN),
    (dict(rotary=FAKE + 8, angles=100), ipv.ERR_ALIGN),
    (dict(qs=(100, 128, 4096)), ipv.ERR_ALIGN),
    (dict(os=(1 << 16, 128, 4100)), ipv.ERR_ALIGN),
    (dict(dtype=2), ipv.ERR_DTYPE),
    (dict(layer=4), ipv.ERR_SHAPE),
    (dict(layer=-1), ipv.ERR_SHAPE),
    (dict(heads=30), ipv.ERR_SHAPE),    # of 4 KV heads
    (dict(heads=0), ipv.ERR_SHAPE),
    (dict(heads=4 * 65535), ipv.ERR_SHAPE),
    (dict(first=(0, -1)), ipv.ERR_SHAPE),
    (dict(rows=(0, -1)), ipv.ERR_SHAPE),
    (dict(first=(0, 632), rows=(7, 9)), ipv.ERR_SHAPE),  # row 640 of ten pages of 64
    (dict(first=(0, 2**31 - 1)), ipv.ERR_SHAPE),
    (dict(eps=0.0), ipv.ERR_ARG),
    (dict(eps=-1.0), ipv.ERR_ARG),
    (dict(eps=math.nan), ipv.ERR_ARG),
    (dict(eps=math.inf), ipv.ERR_ARG),
    (dict(eps=1e-60, qn=None), ipv.ERR_ARG),
    (dict(rotary=FAKE, angles=13), ipv.ERR_ARG),
])
def test_new_tokens_refused(case, status):
    assert qkv(**case) == status


def test_no_new_tokens_are_fine():
    assert qkv(rows=(0, 0)) == ipv.OK
    assert qkv(rows=(0, 0), first=(640, 2**31 - 1), rotary=FAKE, angles=1) == ipv.OK
    assert qkv(rows=(0, 0), bounds=None, block=-7, qn=None, kn=None, eps=-1.0) == ipv.OK  # neither is looked at


def block_bounds(s=None, K=FAKE, Ks=FAKE, bounds=FAKE, block=32, table=FAKE, cols=10, streams=2, first=(0, 5), rows=(7, 9), layer=0, layers=4,
                 ws=FAKE, ws_bytes=BIG):
    s = shape() if s is None else s
    return ipv._paged().ipv_block_bounds(ctypes.byref(s), K, Ks, bounds, block, table, cols, streams, at(first), at(rows), layer, layers, ws,
                                         ws_bytes, None)


@pytest.mark.parametrize("case,status", POOL + [
    (dict(bounds=None), ipv.ERR_NULL),
    (dict(first=None), ipv.ERR_NULL),
    (dict(rows=None), ipv.ERR_NULL),
    (dict(layer=1), ipv.ERR_SHAPE),
    (dict(layer=-1), ipv.ERR_SHAPE),
    (dict(layers=0), ipv.ERR_SHAPE),
    (dict(rows=(1, -1)), ipv.ERR_SHAPE),
    (dict(first=(0, 632)), ipv.ERR_SHAPE),
    (dict(s=shape(layers=32768), layers=32768), ipv.ERR_SHAPE),  # a grid's second dimension
])
def test_bounds_refused(case, status):
    assert block_bounds(**case) == status
    assert block_bounds(rows=(0, 0)) == ipv.OK


def select(s=None, bounds=FAKE, block=32, table=FAKE, cols=10, streams=2, n=(600, 3), first=(599, 2), rows=(1, 1), layer=3, q=FAKE, qs=ROW,
           heads=28, most=1, keep_first=1, keep_last=1, top=5, blocks=FAKE, ws=FAKE, ws_bytes=BIG):
    s = shape() if s is None else s
    return ipv._paged().ipv_block_select(ctypes.byref(s), bounds, block, table, cols, streams, at(n), at(first), at(rows), layer, q,
                                         at(qs, longs), heads, most, keep_first, keep_last, top, blocks, ws, ws_bytes, None)


def attend(s=None, K=FAKE, V=FAKE, Ks=FAKE, Vs=FAKE, bounds=FAKE, block=32, table=FAKE, cols=10, streams=2, n=(600, 3), first=(599, 2),
           rows=(1, 1), layer=3, q=FAKE, qs=ROW, heads=28, most=1, scale=0.1, keep_first=1, keep_last=1, top=5, blocks=FAKE, out=FAKE, os=ROW,
           lse=None, ws=FAKE, ws_bytes=BIG):
    s = shape() if s is None else s
    return ipv._paged().ipv_attend_blocks(ctypes.byref(s), K, V, Ks, Vs, bounds, block, table, cols, streams, at(n), at(first), at(rows),
                                          layer, q, at(qs, longs), heads, most, scale, keep_first, keep_last, top, blocks, out, at(os, longs),
                                          lse, ws, ws_bytes, None)


LISTS = [(c, e) for c, e in POOL if not set(c) & {"K", "Ks"}] + [
    (dict(n=None), ipv.ERR_NULL),
    (dict(first=None), ipv.ERR_NULL),
    (dict(rows=None), ipv.ERR_NULL),
    (dict(q=None), ipv.ERR_NULL),
    (dict(qs=None), ipv.ERR_NULL),
    (dict(blocks=None), ipv.ERR_NULL),
    (dict(q=FAKE + 8), ipv.ERR_ALIGN),
    (dict(blocks=FAKE + 2), ipv.ERR_ALIGN),
    (dict(qs=(100, 128, 4096)), ipv.ERR_ALIGN),
    (dict(layer=4), ipv.ERR_SHAPE),
    (dict(heads=30), ipv.ERR_SHAPE),
    (dict(most=0), ipv.ERR_SHAPE),
    (dict(most=2**30), ipv.ERR_SHAPE),
    (dict(n=(641, 3)), ipv.ERR_SHAPE),
    (dict(n=(-1, 3)), ipv.ERR_SHAPE),
    (dict(rows=(2, 1)), ipv.ERR_SHAPE),
    (dict(rows=(-1, 1)), ipv.ERR_SHAPE),
    (dict(first=(-1, 2)), ipv.ERR_SHAPE),
    (dict(first=(2**30, 2)), ipv.ERR_SHAPE),
    (dict(top=0), ipv.ERR_SHAPE),
    (dict(top=-1), ipv.ERR_SHAPE),
    (dict(top=4097), ipv.ERR_SHAPE),
    (dict(top=4096, s=shape(page_rows=2**19), block=2**19), ipv.ERR_SHAPE),  # rows of a list in 31 bits
    (dict(keep_first=-1), ipv.ERR_ARG),
    (dict(keep_last=-1), ipv.ERR_ARG),
    (dict(keep_first=3, keep_last=3), ipv.ERR_ARG),
    (dict(keep_first=2**31 - 1, keep_last=2**31 - 1), ipv.ERR_ARG),
    (dict(ws_bytes=4352 + 2 * 4 * 32 * 8 - 1), ipv.ERR_WORKSPACE),  # 20 blocks, counted as 32, of two streams of four heads
]


@pytest.mark.parametrize("case,status", LISTS + [(dict(bounds=None), ipv.ERR_NULL)])
def test_selection_refused(case, status):
    assert select(**case) == status


@pytest.mark.parametrize("case,status", LISTS + [
    (dict(K=None), ipv.ERR_NULL),
    (dict(V=None), ipv.ERR_NULL),
    (dict(Vs=None), ipv.ERR_NULL),
    (dict(K=FAKE + 8), ipv.ERR_ALIGN),
    (dict(out=None), ipv.ERR_NULL),
    (dict(os=None), ipv.ERR_NULL),
    (dict(out=FAKE + 4), ipv.ERR_ALIGN),
    (dict(lse=FAKE + 1), ipv.ERR_ALIGN),
    (dict(scale=0.0), ipv.ERR_ARG),
    (dict(scale=-1.0), ipv.ERR_ARG),
    (dict(scale=math.nan), ipv.ERR_ARG),
    (dict(scale=math.inf), ipv.ERR_ARG),
    (dict(scale=1e-60), ipv.ERR_ARG),
    (dict(ws_bytes=4352 + 512 * 16 * 130 * 4 - 1), ipv.ERR_WORKSPACE),  # 64 parts of eight queries' heads
])
def test_lists_refused(case, status):
    assert attend(**case) == status


def test_no_queries_are_fine():
    for call in (select, attend):
        assert call(rows=(0, 0)) == ipv.OK
    assert attend(rows=(0, 0), bounds=None, keep_first=-1, keep_last=7, top=1) == ipv.OK  # only a selection looks at those


def blocks_ws(s, block, streams, heads, rows, top, n):
    out = ctypes.c_size_t(0)
    rc = ipv._paged().ipv_blocks_workspace_bytes(ctypes.byref(s), block, streams, heads, rows, top, n, ctypes.byref(out))
    return rc, out.value


def test_workspace_sizes():
    s = shape(format=ipv.PAGES_BF16)
    assert blocks_ws(s, 32, 1, 28, 1, 5, 600) == (ipv.OK, 4352 + 256 * 16 * 130 * 4)
    assert blocks_ws(s, 32, 1, 28, 4096, 5, 32768)[1] == 4352 + 4096 * 4 * 1024 * 8  # scores of all at once: 128 MiB
    assert blocks_ws(s, 32, 1, 28, 100000, 5, 32768)[1] == 4352 + 4096 * 4 * 1024 * 8
    for bad in ((s, 24, 1, 28, 1, 5, 600), (s, 32, 0, 28, 1, 5, 600), (s, 32, 1, 27, 1, 5, 600), (s, 32, 1, 28, 0, 5, 600),
                (s, 32, 1, 28, 1, 0, 600), (s, 32, 1, 28, 1, 5, -1), (s, 32, 1, 28, 1, 5, 2**30 + 1)):
        assert blocks_ws(*bad)[0] == ipv.ERR_SHAPE
    assert ipv._paged().ipv_blocks_workspace_bytes(ctypes.byref(s), 32, 1, 28, 1, 5, 600, None) == ipv.ERR_NULL


def test_a_workspace_is_enough_for_smaller_calls():
    """Calls of fewer streams, rows and tokens never ask for more than the workspace of the largest."""
    s = shape(format=ipv.PAGES_BF16, pages=1 << 20)
    for streams, rows, n in ((3, 300, 30000), (64, 40, 32768), (1, 5000, 9000)):
        room = blocks_ws(s, 16, streams, 28, rows, 7, n)[1]
        for b, r, t in ((1, 1, 1), (streams, 1, n), (streams, rows, n // 3), (max(1, streams // 2), rows, n), (1, rows, n)):
            kw = dict(s=s, block=16, table=FAKE, cols=1000, streams=b, n=(t,) * b, first=(0,) * b, rows=(0,) * b, heads=28, most=r, ws_bytes=room)
            assert attend(**kw, Ks=None, Vs=None) == ipv.OK and select(**kw) == ipv.OK


def compact(s=None, K=FAKE, V=FAKE, Ks=FAKE, Vs=FAKE, bounds=FAKE, block=32, table=FAKE, cols=10, new=FAKE, new_cols=5, streams=2, n=(600, 3),
            keep=FAKE, C=300, rows=(300, 3), rotary=None, angles=0, ws=FAKE, ws_bytes=BIG):
    s = shape() if s is None else s
    return ipv._paged().ipv_page_compact(ctypes.byref(s), K, V, Ks, Vs, bounds, block, table, cols, new, new_cols, streams, at(n), keep, C,
                                         at(rows), rotary, angles, ws, ws_bytes, None)


@pytest.mark.parametrize("case,status", POOL + [
    (dict(V=None), ipv.ERR_NULL),
    (dict(new=None), ipv.ERR_NULL),
    (dict(n=None), ipv.ERR_NULL),
    (dict(keep=None), ipv.ERR_NULL),
    (dict(rows=None), ipv.ERR_NULL),
    (dict(new=FAKE + 2), ipv.ERR_ALIGN),
    (dict(keep=FAKE + 2), ipv.ERR_ALIGN),
    (dict(rotary=FAKE + 8, angles=600), ipv.ERR_ALIGN),
    (dict(new_cols=0), ipv.ERR_SHAPE),
    (dict(C=0), ipv.ERR_SHAPE),
    (dict(n=(641, 3)), ipv.ERR_SHAPE),
    (dict(n=(-1, 3)), ipv.ERR_SHAPE),
    (dict(rows=(301, 3)), ipv.ERR_SHAPE),
    (dict(rows=(-1, 3)), ipv.ERR_SHAPE),
    (dict(C=400, rows=(321, 3)), ipv.ERR_SHAPE),  # five new pages of 64
    (dict(rotary=FAKE, angles=599), ipv.ERR_ARG),
    (dict(rotary=FAKE, angles=299, n=(200, 3)), ipv.ERR_ARG),
    (dict(s=shape(layers=8192)), ipv.ERR_SHAPE),  # a grid's second dimension
])
def test_compaction_refused(case, status):
    assert compact(**case) == status
    assert compact(rows=(0, 0)) == ipv.OK


def copy(s=None, K=FAKE, V=FAKE, Ks=FAKE, Vs=FAKE, bounds=FAKE, block=32, src=FAKE, dst=FAKE, count=3, rows=64, ws=FAKE, ws_bytes=BIG):
    s = shape() if s is None else s
    return ipv._paged().ipv_page_copy(ctypes.byref(s), K, V, Ks, Vs, bounds, block, src, dst, count, rows, ws, ws_bytes, None)


@pytest.mark.parametrize("case,status", [(c, e) for c, e in POOL if not set(c) & {"table", "cols", "streams"} and "page_rows" not in str(c)] + [
    (dict(V=None), ipv.ERR_NULL),
    (dict(src=None), ipv.ERR_NULL),
    (dict(dst=None), ipv.ERR_NULL),
    (dict(src=FAKE + 2), ipv.ERR_ALIGN),
    (dict(dst=FAKE + 1), ipv.ERR_ALIGN),
    (dict(count=-1), ipv.ERR_SHAPE),
    (dict(rows=0), ipv.ERR_SHAPE),
    (dict(rows=65), ipv.ERR_SHAPE),
    (dict(s=shape(pages=1, layers=2**15, kv_heads=2**6, page_rows=2**9, format=ipv.PAGES_F32)), ipv.ERR_SHAPE),  # a page in 32 bits
])
def test_copies_refused(case, status):
    assert copy(**case) == status
    assert copy(count=0) == ipv.OK


# ---------------------------------------------------------------- the binding
def pool(fmt=ipv.PAGES_BF16, **kw):
    """A pool on the host: its checks come before any address is taken of what a call is given."""
    p = object.__new__(ipv.PagePool)
    p._tensors = tuple(torch.zeros(6, 2, 2, 32, 64, dtype=torch.bfloat16) for _ in range(2)) + (None, None)
    p.format, p.head_dim, p.device, p.dtype = fmt, 64, p._tensors[0].device, torch.bfloat16
    p.shape, p._dev, p._args = ipv.PageShape(6, 2, 2, 32, 64, fmt), -1, (None,) * 5
    return p


def status(fn, *a, **kw):
    with pytest.raises(ipv.IpvError) as e:
        fn(*a, **kw)
    return e.value.status


def test_binding_checks_blocks():
    p = pool()
    for rows in (0, 8, 24, 48, 64, -16):
        assert status(ipv.BlockBounds, p, rows) == ipv.ERR_SHAPE
    assert status(ipv.BlockBounds, p, 16, torch.zeros(6, 2, 2, 1, 2, 64, dtype=torch.bfloat16)) == ipv.ERR_SHAPE
    assert status(ipv.BlockBounds, p, 16, torch.zeros(6, 2, 2, 2, 2, 64)) == ipv.ERR_DTYPE
    assert status(ipv.BlockBounds, p, 16) == ipv.ERR_ARG  # a host tensor


def test_binding_checks_new_tokens():
    p, ws = pool(), torch.zeros(256, dtype=torch.uint8)
    q, k = torch.zeros(1, 4, 3, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    call = lambda q=q, k=k, v=k, out=q, **kw: status(ipv.ipv_qkv_write, p, None, 0, 0, q, k, v, out, ws, **kw)  # noqa: E731
    assert call(q=q[0]) == ipv.ERR_SHAPE
    assert call(q=q[..., :32]) == ipv.ERR_SHAPE
    assert call(k=k[:, :1]) == ipv.ERR_SHAPE
    assert call(v=k[:, :, :2]) == ipv.ERR_SHAPE
    assert call(k=k.float()) == ipv.ERR_DTYPE
    assert call(out=q.float()) == ipv.ERR_DTYPE
    assert call(out=q[:, :2]) == ipv.ERR_SHAPE
    assert call(out=q[:, :, :1].expand(1, 4, 3, 64)) == ipv.ERR_SHAPE
    assert call(v=k.transpose(1, 2).contiguous().transpose(1, 2)) == ipv.ERR_SHAPE
    assert call(q=torch.zeros(1, 4, 64, 3, dtype=torch.bfloat16).transpose(2, 3)) == ipv.ERR_SHAPE
    assert call(rows=4) == ipv.ERR_SHAPE
    assert call() == ipv.ERR_ARG  # host tensors
    assert status(ipv.ipv_qkv_write, p, None, 0, 0, q, k, k, q, None) == ipv.ERR_WORKSPACE


def test_binding_checks_lists():
    p, ws = pool(), torch.zeros(256, dtype=torch.uint8)
    q, blocks = torch.zeros(1, 4, 3, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 3, 5, dtype=torch.int32)
    call = lambda q=q, blocks=blocks, out=q, **kw: status(ipv.ipv_attend_blocks, p, None, 3, 0, 0, q, blocks, out, ws, **kw)  # noqa: E731
    assert call() == ipv.ERR_ARG  # neither bounds nor block_rows
    assert call(block_rows=16, blocks=blocks.long()) == ipv.ERR_SHAPE
    assert call(block_rows=16, blocks=blocks[:, :1]) == ipv.ERR_SHAPE
    assert call(block_rows=16, blocks=blocks[0]) == ipv.ERR_SHAPE
    assert call(block_rows=16, q=q.float()) == ipv.ERR_DTYPE
    assert call(block_rows=16, out=q[:, :2]) == ipv.ERR_SHAPE
    assert call(block_rows=2**40) == ipv.ERR_ARG
    assert call(block_rows=16, lse=torch.zeros(1, 4, 2)) == ipv.ERR_SHAPE
    assert call(block_rows=16) == ipv.ERR_ARG  # host tensors
    assert status(ipv.ipv_block_select, p, None, None, 3, 0, 0, q, blocks, ws) == ipv.ERR_NULL
    assert status(ipv.ipv_block_select, p, None, None, 3, 0, 0, q.float(), blocks, ws) == ipv.ERR_DTYPE


def test_binding_checks_compaction_and_copies():
    p, ws = pool(), torch.zeros(256, dtype=torch.uint8)
    keep, table = torch.zeros(1, 2, 2, 5, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32)
    assert status(ipv.ipv_page_compact, p, None, table, 3, keep.long(), ws) == ipv.ERR_SHAPE
    assert status(ipv.ipv_page_compact, p, None, table, 3, keep[:, :1], ws) == ipv.ERR_SHAPE
    assert status(ipv.ipv_page_compact, p, None, None, 3, keep, ws) == ipv.ERR_NULL
    assert status(ipv.ipv_page_compact, p, None, torch.zeros(2, 1, dtype=torch.int32), 3, keep, ws) == ipv.ERR_SHAPE
    one = torch.zeros(2, dtype=torch.int32)
    assert status(ipv.ipv_page_copy, p, one, one[:1], ws) == ipv.ERR_SHAPE
    assert status(ipv.ipv_page_copy, p, one.long(), one, ws) == ipv.ERR_SHAPE
    assert status(ipv.ipv_page_copy, p, one[None], one, ws) == ipv.ERR_SHAPE
    assert status(ipv.ipv_page_copy, p, one, one, None) == ipv.ERR_WORKSPACE
