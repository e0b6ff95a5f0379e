"""PageTables on the host: which page is whose after reserving, forking, freeing and compacting. The pool is a plain
stand-in in CPU memory, and the copies that the calls would launch are written down instead."""
import random
from types import SimpleNamespace

import pytest
import torch

from paper_2506_15745_amd import ipv

T = 64


@pytest.fixture
def calls(monkeypatch):
    seen = []
    monkeypatch.setattr(ipv, "ipv_page_copy", lambda pool, old, new, ws, rows=None, bounds=None: seen.append(
        ("copy", old.tolist(), new.tolist(), rows, bounds)))
    monkeypatch.setattr(ipv, "ipv_page_compact", lambda pool, table, new, n, keep, ws, rows=None, rotary=None, bounds=None: seen.append(
        ("compact", table.tolist(), new.tolist(), n, rows, rotary, bounds)))
    return seen


def tables(pages=8, streams=3, columns=4):
    return ipv.PageTables(SimpleNamespace(shape=SimpleNamespace(pages=pages, page_rows=T), device="cpu"), streams, columns)


def consistent(t):
    """Every page is free or has as many users as streams name it; the table says what the lists say."""
    named = [p for x in t.pages for p in x]
    assert all(t._users[p] == named.count(p) for p in range(len(t._users)))
    assert sorted(t._free + sorted(set(named))) == list(range(len(t._users)))
    assert t.free_pages == len(t._users) - len(set(named))
    assert t.table.tolist() == [x + [-1] * (t.columns - len(x)) for x in t.pages]


def test_rows_get_pages(calls):
    t = tables()
    at = t.table.data_ptr()
    assert bool((t.table == -1).all()) and t.free_pages == 8
    t.reserve(0, [1, 0, 130], None)
    consistent(t)
    assert [len(x) for x in t.pages] == [1, 0, 3] and t.free_pages == 4 and calls == []
    t.reserve([1, 0, 130], [63, 0, 62], None)  # up to the pages' ends
    assert [len(x) for x in t.pages] == [1, 0, 3]
    t.reserve([64, 70, 0], [1, 1, 1], None)  # (stream 1: with the page before)
    consistent(t)
    assert [len(x) for x in t.pages] == [2, 2, 3] and calls == [] and t.table.data_ptr() == at


def test_a_shared_page_is_copied_before_it_is_written(calls):
    t = tables()
    t.reserve(0, [100, 0, 0], None)
    t.fork(0, 1, 100)
    t.fork(0, 2, 64)
    consistent(t)
    a, b = t.pages[0]
    assert t.pages == [[a, b], [a, b], [a]] and t.free_pages == 6
    t.reserve([100, 100, 64], 1, "ws", bounds="bounds")  # page b of two: one of them gets a copy
    consistent(t)
    assert calls == [("copy", [b], [t.pages[0][1]], None, "bounds")]
    assert t.pages[1] == [a, b] and t.pages[0][0] == t.pages[2][0] == a and len({b, t.pages[0][1], t.pages[2][1]}) == 3
    t.reserve([101, 101, 65], 1, None)
    assert len(calls) == 1
    t.reserve([0, 0, 0], [1, 1, 1], "ws")  # the shared first page: two of three get a copy, by one call
    consistent(t)
    assert calls[1] == ("copy", [a, a], [t.pages[0][0], t.pages[1][0]], None, None) and t.pages[2][0] == a


def test_freeing(calls):
    t = tables()
    t.reserve(0, [200, 0, 0], None)
    t.fork(0, 1, 200)
    t.free(0, 65)
    consistent(t)
    assert len(t.pages[0]) == 2 and len(t.pages[1]) == 4 and t.free_pages == 4
    t.free(1)
    consistent(t)
    assert t.pages[1] == [] and t.free_pages == 6
    t.free(0, 300)  # (more than it has)
    assert len(t.pages[0]) == 2
    t.fork(0, 0, 64)  # onto itself: what is left
    consistent(t)
    assert len(t.pages[0]) == 1 and t.free_pages == 7


def test_compaction_takes_pages_of_its_own(calls):
    t = tables(pages=10)
    t.reserve(0, [200, 64, 70], None)
    t.fork(0, 1, 130)
    old = [list(x) for x in t.pages]
    keep = torch.zeros((2, 1, 1, 66), dtype=torch.int32)
    t.compact([2, 0], [70, 200], keep, None, rows=[10, 66], rotary="rotary")
    consistent(t)
    assert calls == [("compact", [old[2] + [-1] * 2, old[0]], [t.pages[2] + [-1] * 3, t.pages[0] + [-1] * 2], [70, 200], [10, 66], "rotary", None)]
    assert t.pages[1] == old[1] and not set(t.pages[0] + t.pages[2]) & set(sum(old, []))
    t.compact([], [], keep[:0], None)
    t.compact([0], [66], keep[:1, ..., :0], None)  # nothing is kept
    consistent(t)
    assert t.pages[0] == []


def test_refusals_change_nothing(calls):
    t = tables(pages=4, columns=3)
    t.reserve(0, [100, 0, 0], None)
    t.fork(0, 1, 100)
    keep = torch.zeros((1, 1, 1, 130), dtype=torch.int32)
    before = [list(x) for x in t.pages]
    for call, status in (
            (lambda: t.reserve([100, 100, 0], [1, 1, 128], None), ipv.ERR_ARG),      # a copy and two pages: two are free
            (lambda: t.reserve(0, [193, 0, 0], None), ipv.ERR_SHAPE),                # four pages, three columns
            (lambda: t.reserve([-1, 0, 0], 1, None), ipv.ERR_SHAPE),
            (lambda: t.reserve(0, [0, 0, -1], None), ipv.ERR_SHAPE),
            (lambda: t.reserve([0, 0], 1, None), ipv.ERR_SHAPE),
            (lambda: t.fork(0, 3, 1), ipv.ERR_ARG),
            (lambda: t.fork(-1, 0, 1), ipv.ERR_ARG),
            (lambda: t.fork(2, 0, 1), ipv.ERR_SHAPE),
            (lambda: t.fork(0, 2, 129), ipv.ERR_SHAPE),
            (lambda: t.fork(0, 2, -1), ipv.ERR_SHAPE),
            (lambda: t.free(3), ipv.ERR_ARG),
            (lambda: t.free(0, -1), ipv.ERR_SHAPE),
            (lambda: t.compact([0], [100], keep, None), ipv.ERR_ARG),                # three pages
            (lambda: t.compact([0, 0], [100, 100], keep, None), ipv.ERR_ARG),
            (lambda: t.compact([0], [100], keep, None, rows=[-1]), ipv.ERR_SHAPE),
            (lambda: t.compact([0], [100], keep, None, rows=[193]), ipv.ERR_SHAPE),
            (lambda: tables(streams=0), ipv.ERR_SHAPE),
            (lambda: tables(columns=0), ipv.ERR_SHAPE)):
        with pytest.raises(ipv.IpvError) as e:
            call()
        assert e.value.status == status
        assert t.pages == before and calls == []
        consistent(t)


def test_a_call_that_is_refused_inside_changes_nothing(monkeypatch):
    def refuse(*_, **__):
        raise ipv.IpvError(ipv.ERR_WORKSPACE, "no workspace")
    monkeypatch.setattr(ipv, "ipv_page_copy", refuse)
    monkeypatch.setattr(ipv, "ipv_page_compact", refuse)
    t = tables()
    t.reserve(0, [100, 0, 0], None)
    t.fork(0, 1, 100)
    before = [list(x) for x in t.pages]
    for call in (lambda: t.reserve([100, 100, 0], [1, 1, 5], None),
                 lambda: t.compact([0], [100], torch.zeros((1, 1, 1, 20), dtype=torch.int32), None)):
        with pytest.raises(ipv.IpvError):
            call()
        assert t.pages == before
        consistent(t)


@pytest.mark.parametrize("seed", range(4))
def test_any_order_of_calls(calls, seed):
    r = random.Random(seed)
    t = tables(pages=20, streams=4, columns=5)
    rows = [0] * 4
    for _ in range(300):
        what, b, to = r.randrange(4), r.randrange(4), r.randrange(4)
        try:
            if what == 0:
                first, more = list(rows), [r.choice((0, 1, 5, 70)) for _ in rows]
                t.reserve(first, more, None)
                rows = [x + y for x, y in zip(rows, more)]
            elif what == 1:
                n = r.randint(0, rows[b])
                t.fork(b, to, n)
                rows[to] = n
            elif what == 2:
                rows[b] = r.randint(0, rows[b])
                t.free(b, rows[b])
            else:
                n = r.randint(0, rows[b])
                t.compact([b], [rows[b]], torch.zeros((1, 1, 1, n), dtype=torch.int32), None)
                rows[b] = n
        except ipv.IpvError as e:
            assert e.status in (ipv.ERR_ARG, ipv.ERR_SHAPE)
        consistent(t)
        assert all(len(x) * T >= n for x, n in zip(t.pages, rows))
    assert calls
