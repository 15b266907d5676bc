"""Counts of pages at the end of a pool whose number of pages is no multiple of eight, changed by many entries at once."""
import pytest

from test_gpu_plan import INT_MIN, Steps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [10, 1100])
@pytest.mark.parametrize("n_pages", [9000, 9001, 9002, 9003, 9004, 9005, 9006, 9007])
def test_counts_of_the_last_pages(S, n_pages):
    """2000 entries and more change in a call, so counts are summed in LDS first: all pages but the last 300 are held."""
    x = Steps(S, 310, n_pages, 4, held=range(n_pages - 300))
    x.step([1200] + [0] * (S - 1))
    assert x.b.table[0][299] == n_pages - 1
    parent, shared = [0] * S, [1200] * S
    last = range(n_pages - 9, n_pages)
    x.step([0] * 10 + [INT_MIN] * (S - 10), parent=parent, shared=shared)    # 2700 entries are taken over
    assert [x.b.refs[p] for p in last] == [10] * 9
    x.step([0, 0] + [INT_MIN] * (S - 2))                  # ... 2400 given back
    assert [x.b.refs[p] for p in last] == [2] * 9
    # the first ends, with one that shares all and eight that begin with an odd number of its pages
    x.step([INT_MIN] * 2 + [0] * 8 + [INT_MIN] * (S - 10), parent=parent, shared=[1200 if s % 2 else 1188 for s in range(S)])
    assert [x.b.refs[p] for p in last] == [8] * 6 + [4] * 3
    x.step([INT_MIN] * S)
    assert sum(x.b.refs) == n_pages - 300 and not any(x.b.refs[-300:])
    x.step([1200] + [0] * (S - 1))                        # and all of them are free again
