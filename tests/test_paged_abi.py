"""The paged cache's calls on the host: what they refuse, before anything is launched.

Every call here carries at least one argument that the host checks reject, or
has nothing to do, so no kernel is enqueued (these tests run without a GPU)."""
import ctypes

import pytest
import torch

from paper_2506_15745_amd import ipv

FAKE = 0x10000  # 256-aligned, never dereferenced
BIG = 1 << 40


def shape(**kw):
    d = dict(pages=100, layers=4, kv_heads=4, page_rows=64, head_dim=128, format=ipv.PAGES_FP8)
    d.update(kw)
    return ipv.PageShape(*[d[k] for k in ("pages", "layers", "kv_heads", "page_rows", "head_dim", "format")])


def ints(*v):
    return (ctypes.c_int32 * len(v))(*v)


def longs(*v):
    return (ctypes.c_int64 * len(v))(*v)


def rows_call(name="ipv_page_write", s=None, K=FAKE, V=FAKE, Ks=FAKE, Vs=FAKE, table=FAKE, cols=10, streams=2, first=(0, 5),
              rows=(7, 9), layer=0, layers=4, src=FAKE, src_V=FAKE, dtype=ipv.BF16, strides=(1 << 20, 1 << 16, 1 << 12, 128),
              rotary=None, rotary_rows=0, ws=FAKE, ws_bytes=BIG):
    s = shape() if s is None else s
    return getattr(ipv._paged(), name)(
        ctypes.byref(s), K, V, Ks, Vs, table, cols, streams, None if first is None else ints(*first),
        None if rows is None else ints(*rows), layer, layers, src, src_V, dtype, None if strides is None else longs(*strides),
        rotary, rotary_rows, ws, ws_bytes, None)


ROWS = [
    (dict(K=None), ipv.ERR_NULL),
    (dict(V=None), ipv.ERR_NULL),
    (dict(Ks=None), ipv.ERR_NULL),
    (dict(Vs=None), ipv.ERR_NULL),
    (dict(first=None), ipv.ERR_NULL),
    (dict(rows=None), ipv.ERR_NULL),
    (dict(src=None), ipv.ERR_NULL),
    (dict(src_V=None), ipv.ERR_NULL),
    (dict(strides=None), ipv.ERR_NULL),
    (dict(K=FAKE + 8), ipv.ERR_ALIGN),
    (dict(Vs=FAKE + 2), ipv.ERR_ALIGN),
    (dict(table=FAKE + 2), ipv.ERR_ALIGN),
    (dict(src=FAKE + 8), ipv.ERR_ALIGN),
    (dict(strides=(1 << 20, 1 << 16, 1 << 12, 100)), ipv.ERR_ALIGN),
    (dict(rotary=FAKE + 8, rotary_rows=100), ipv.ERR_ALIGN),
    (dict(dtype=2), ipv.ERR_DTYPE),
    (dict(s=shape(format=4)), ipv.ERR_DTYPE),
    (dict(s=shape(format=-1)), ipv.ERR_DTYPE),
    (dict(s=shape(head_dim=96)), ipv.ERR_SHAPE),
    (dict(s=shape(page_rows=0)), ipv.ERR_SHAPE),
    (dict(s=shape(pages=0)), ipv.ERR_SHAPE),
    (dict(s=shape(layers=0)), ipv.ERR_SHAPE),
    (dict(s=shape(kv_heads=0)), ipv.ERR_SHAPE),
    (dict(s=shape(pages=2**31 - 1, layers=2**20, kv_heads=64, page_rows=2**20)), ipv.ERR_SHAPE),  # 64-bit offsets
    (dict(streams=0), ipv.ERR_SHAPE),
    (dict(cols=0), ipv.ERR_SHAPE),
    (dict(layer=-1), ipv.ERR_SHAPE),
    (dict(layer=1), ipv.ERR_SHAPE),               # layers 1 .. 4 of 4
    (dict(layers=0), ipv.ERR_SHAPE),
    (dict(layers=5), ipv.ERR_SHAPE),
    (dict(first=(-1, 0)), ipv.ERR_SHAPE),
    (dict(rows=(-1, 0)), ipv.ERR_SHAPE),
    (dict(first=(0, 632), rows=(7, 9)), ipv.ERR_SHAPE),  # row 640 of ten pages of 64
    (dict(first=(0, 2**31 - 1), rows=(7, 1)), ipv.ERR_SHAPE),
    (dict(table=None, cols=10), ipv.ERR_SHAPE),   # without a table a stream has one page
    (dict(table=None, cols=1, s=shape(pages=1)), ipv.ERR_SHAPE),
    (dict(table=None, cols=1, first=(0, 60)), ipv.ERR_SHAPE),
    (dict(rotary=FAKE, rotary_rows=13), ipv.ERR_ARG),    # stream 1 ends at position 14
    (dict(ws=None), ipv.ERR_WORKSPACE),
    (dict(ws=FAKE + 16), ipv.ERR_ALIGN),
    (dict(ws_bytes=255), ipv.ERR_WORKSPACE),
]


@pytest.mark.parametrize("name", ["ipv_page_write", "ipv_page_read"])
@pytest.mark.parametrize("case,status", ROWS)
def test_rows_refused(name, case, status):
    assert rows_call(name, **case) == status


def test_rows_of_nothing_are_fine():
    for name in ("ipv_page_write", "ipv_page_read"):
        assert rows_call(name, rows=(0, 0)) == ipv.OK
        assert rows_call(name, rows=(0, 0), first=(640, 2**31 - 1), rotary=FAKE, rotary_rows=1) == ipv.OK  # no position is used
        assert rows_call(name, s=shape(format=ipv.PAGES_BF16), Ks=None, Vs=None, rows=(0, 0)) == ipv.OK


def attend_call(s=None, K=FAKE, V=FAKE, Ks=FAKE, Vs=FAKE, table=FAKE, cols=10, streams=2, n=(600, 3), first=(599, 2), rows=(1, 1),
                layer=3, q=FAKE, qs=(1 << 16, 128, 4096), heads=28, most=1, scale=0.1, window=0, sinks=0, out=FAKE,
                os=(1 << 16, 128, 4096), lse=None, ws=FAKE, ws_bytes=BIG):
    s = shape() if s is None else s
    return ipv._paged().ipv_attend(
        ctypes.byref(s), K, V, Ks, Vs, table, cols, streams, None if n is None else ints(*n), None if first is None else ints(*first),
        None if rows is None else ints(*rows), layer, q, None if qs is None else longs(*qs), heads, most, scale, window, sinks, out,
        None if os is None else longs(*os), lse, ws, ws_bytes, None)


@pytest.mark.parametrize("case,status", [
    (dict(K=None), ipv.ERR_NULL),
    (dict(Vs=None), ipv.ERR_NULL),
    (dict(n=None), ipv.ERR_NULL),
    (dict(first=None), ipv.ERR_NULL),
    (dict(rows=None), ipv.ERR_NULL),
    (dict(q=None), ipv.ERR_NULL),
    (dict(out=None), ipv.ERR_NULL),
    (dict(qs=None), ipv.ERR_NULL),
    (dict(os=None), ipv.ERR_NULL),
    (dict(q=FAKE + 8), ipv.ERR_ALIGN),
    (dict(out=FAKE + 4), ipv.ERR_ALIGN),
    (dict(lse=FAKE + 1), ipv.ERR_ALIGN),
    (dict(qs=(1 << 16, 4, 4096)), ipv.ERR_ALIGN),
    (dict(os=(1 << 16, 128, 4100)), ipv.ERR_ALIGN),
    (dict(s=shape(format=9)), ipv.ERR_DTYPE),
    (dict(s=shape(head_dim=64 + 32)), ipv.ERR_SHAPE),
    (dict(heads=30), ipv.ERR_SHAPE),              # not a multiple of 4 KV heads
    (dict(heads=0), ipv.ERR_SHAPE),
    (dict(most=0), ipv.ERR_SHAPE),
    (dict(most=2**30), ipv.ERR_SHAPE),
    (dict(rows=(2, 1)), ipv.ERR_SHAPE),           # more rows than max_rows
    (dict(rows=(-1, 1)), ipv.ERR_SHAPE),
    (dict(n=(641, 3)), ipv.ERR_SHAPE),            # more rows than the table covers
    (dict(n=(-1, 3)), ipv.ERR_SHAPE),
    (dict(first=(-1, 2)), ipv.ERR_SHAPE),
    (dict(first=(2**30, 2)), ipv.ERR_SHAPE),
    (dict(layer=4), ipv.ERR_SHAPE),
    (dict(layer=-1), ipv.ERR_SHAPE),
    (dict(table=None), ipv.ERR_SHAPE),
    (dict(scale=0.0), ipv.ERR_ARG),
    (dict(scale=-1.0), ipv.ERR_ARG),
    (dict(scale=float("nan")), ipv.ERR_ARG),
    (dict(scale=float("inf")), ipv.ERR_ARG),
    (dict(scale=1e300), ipv.ERR_ARG),
    (dict(scale=1e-300), ipv.ERR_ARG),
    (dict(window=-1), ipv.ERR_ARG),
    (dict(sinks=-1), ipv.ERR_ARG),
    (dict(ws=None), ipv.ERR_WORKSPACE),
    (dict(ws=FAKE + 128), ipv.ERR_ALIGN),
    (dict(ws_bytes=1024), ipv.ERR_WORKSPACE),
])
def test_attend_refused(case, status):
    assert attend_call(**case) == status


def test_attend_of_no_queries_is_fine():
    assert attend_call(rows=(0, 0)) == ipv.OK
    assert attend_call(rows=(0, 0), s=shape(format=ipv.PAGES_F32), Ks=None, Vs=None) == ipv.OK


def test_attend_workspace():
    size = ctypes.c_size_t(0)
    call = ipv._paged().ipv_attend_workspace_bytes

    def need(streams=1, heads=28, rows=1, **kw):
        assert call(ctypes.byref(shape(**kw)), streams, heads, rows, ctypes.byref(size)) == ipv.OK
        return size.value

    assert need() >= 256
    assert need(rows=500) >= need(rows=4) >= need()           # a workspace for more rows serves fewer
    assert need(rows=500, streams=64) == need(rows=500)       # what is split does not grow with the streams
    assert need(head_dim=256) >= need(head_dim=32)
    s = shape()
    assert call(ctypes.byref(s), 1, 28, 1, None) == ipv.ERR_NULL
    assert call(None, 1, 28, 1, ctypes.byref(size)) == ipv.ERR_NULL
    for bad in ((0, 28, 1), (1, 27, 1), (1, 0, 1), (1, 28, 0)):
        assert call(ctypes.byref(s), *bad, ctypes.byref(size)) == ipv.ERR_SHAPE


# ---------------------------------------------------------------- the binding
def refused(status, f, *a, **kw):
    with pytest.raises(ipv.IpvError) as e:
        f(*a, **kw)
    assert e.value.status == status


def test_pools_refused():
    Z = torch.zeros
    k = Z(2, 1, 2, 8, 64, dtype=torch.bfloat16)
    refused(ipv.ERR_SHAPE, ipv.PagePool, k[0], k[0])
    refused(ipv.ERR_SHAPE, ipv.PagePool, k, k[:1])
    refused(ipv.ERR_DTYPE, ipv.PagePool, k, k.float())
    refused(ipv.ERR_DTYPE, ipv.PagePool, k.half(), k.half())
    refused(ipv.ERR_ARG, ipv.PagePool, k, k)                   # not in GPU memory
    c, s = Z(2, 1, 2, 8, 64, dtype=torch.uint8), Z(2, 1, 2, 8, 2, dtype=torch.uint8)
    refused(ipv.ERR_NULL, ipv.PagePool, c, c)
    refused(ipv.ERR_ARG, ipv.PagePool, k, k, s, s)             # scales beside bf16
    refused(ipv.ERR_SHAPE, ipv.PagePool, c, c, s[..., :1], s[..., :1].repeat(1, 1, 1, 1, 2))
    refused(ipv.ERR_SHAPE, ipv.PagePool, c[..., :48], c[..., :48], s, s)
    refused(ipv.ERR_SHAPE, ipv.PagePool, c, c, s, s[:1])
    refused(ipv.ERR_DTYPE, ipv.PagePool, c, c, s, s.int())
    refused(ipv.ERR_DTYPE, ipv.PagePool.empty, 1, 1, 1, 8, 64, 7, device="cpu")


def test_host_arrays():
    assert list(ipv._host_counts(5, 3, "n")) == [5, 5, 5]
    assert list(ipv._host_counts([1, 2], 2, "n")) == [1, 2]
    refused(ipv.ERR_SHAPE, ipv._host_counts, [1, 2], 3, "n")
    x = torch.zeros(2, 3, 4, 8)
    assert list(ipv._stride_array(x.stride(), x.shape)) == [96, 32, 8]
    assert list(ipv._stride_array(x[:1].stride(), x[:1].shape)) == [0, 32, 8]
    refused(ipv.ERR_SHAPE, ipv._stride_array, x.transpose(2, 3).stride(), x.transpose(2, 3).shape)
