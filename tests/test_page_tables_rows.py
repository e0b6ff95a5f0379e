"""PageTables.compact on the host: rows that a stream does not have are refused, and then nothing changes."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests.test_page_tables import calls, consistent, tables  # noqa: F401 (calls: a fixture)


@pytest.mark.parametrize("streams,n_tokens,status", [
    ([0], [129], ipv.ERR_SHAPE),            # two pages of 64
    ([0], 129, ipv.ERR_SHAPE),
    ([0], [250], ipv.ERR_SHAPE),            # as many as the table's columns take
    ([0], [2**31 - 1], ipv.ERR_SHAPE),
    ([0], [2**31], ipv.ERR_SHAPE),
    ([0], [-1], ipv.ERR_SHAPE),
    ([1], [1], ipv.ERR_SHAPE),              # no pages at all
    ([0, 2], [100, 65], ipv.ERR_SHAPE),     # the second one
    ([2, 0], [64, 129], ipv.ERR_SHAPE),
    ([0, 2], [100], ipv.ERR_SHAPE),
])
def test_rows_that_a_stream_does_not_have(calls, streams, n_tokens, status):  # noqa: F811
    t = tables()
    t.reserve(0, [100, 0, 10], None)
    before = [list(x) for x in t.pages]
    with pytest.raises(ipv.IpvError) as e:
        t.compact(streams, n_tokens, torch.zeros((len(streams), 1, 1, 20), dtype=torch.int32), None)
    assert e.value.status == status and t.pages == before and calls == []
    consistent(t)


def test_after_freeing(calls):  # noqa: F811
    """The count that a stream had before its pages went back."""
    t = tables()
    t.reserve(0, [200, 0, 0], None)
    t.free(0, 64)
    with pytest.raises(ipv.IpvError):
        t.compact([0], [200], torch.zeros((1, 1, 1, 20), dtype=torch.int32), None)
    assert len(t.pages[0]) == 1 and t.free_pages == 7 and calls == []
    t.compact([0], [64], torch.zeros((1, 1, 1, 20), dtype=torch.int32), None)
    consistent(t)
    assert len(calls) == 1


def test_all_rows_of_the_pages_are_fine(calls):  # noqa: F811
    t = tables()
    t.reserve(0, [100, 0, 10], None)
    t.compact([2, 0], [64, 128], torch.zeros((2, 1, 1, 20), dtype=torch.int32), None)
    consistent(t)
    t.compact([0, 2], 0, torch.zeros((2, 1, 1, 20), dtype=torch.int32), None, rows=0)  # none of none
    consistent(t)
    assert [len(x) for x in t.pages] == [0, 0, 0] and [c[3] for c in calls] == [[64, 128], 0]
