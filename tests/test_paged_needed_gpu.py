"""Pages that a paged attention does not need: behind a sequence's end, and where a window has moved on.
Their entries may name nothing (a server that evicts them writes -1 there), and nothing is reported."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_paged_attention_gpu import BF, FP, Q8, Case, dev  # noqa: E402

pytestmark = pytest.mark.gpu


def needed(c):
    """bool [B, table length]: the pages with a row that a slot of the block sees."""
    some = np.zeros(c.table.shape, bool)
    for b in range(c.B):
        if c.counts[b] > 0:
            rows = np.flatnonzero(c.want(b)[4].any(0).numpy())
            some[b, np.unique(rows // c.page)] = True
    return some


def evicted(c, entry):
    """The table with `entry` in the place of every page that is not needed."""
    some = needed(c)
    assert not some.all()
    return np.where(some, c.table, entry).astype(np.int32)


FORMS = [(1, 4, False), (3, 5, False), (4, 4, True), (40, 2, False), (8, 4, True), (41, 4, True)]


@pytest.mark.parametrize("page", [1, 16, 24])
@pytest.mark.parametrize("window,sinks", [(50, 4), (100, 0), (33, 21), (64, 1), (31, 33), (9, 70)])
@pytest.mark.parametrize("S,group,tree", FORMS)
def test_pages_out_of_the_window(S, group, tree, window, sinks, page):
    """Windows and first rows that begin and end inside tiles, in both walks."""
    for entry, cache in ((-1, BF), (1 << 30, Q8)):
        c = Case(3, S, 2 * group, 2, 64, page, [150, 301, 97], counts=[S, S, max(1, S // 2)], tree=tree, window=window,
                 sinks=sinks, cache=cache, seed=S + page + window)
        print(S, group, tree, window, sinks, page, cache, flush=True)
        c.verify(page_table=dev(evicted(c, entry)))


@pytest.mark.parametrize("S,group,tree", FORMS)
def test_a_needed_page_is_reported(S, group, tree):
    """Each page that is seen, in turn, and nothing else."""
    c = Case(1, S, 2 * group, 2, 32, 24, [150], tree=tree, window=50, sinks=4, dtype=FP, seed=S)
    some, right = needed(c), evicted(c, -1)
    for j in range(right.shape[1]):
        table = right.copy()
        table[0, j] = -7
        c.run(page_table=dev(table))
        assert (c.ctx.device_status() != 0) == some[0, j], j
    c.ctx.close()


def test_pages_out_of_many_windows():
    """More row tiles than workgroups that run at once."""
    c = Case(40, 40, 64, 32, 16, 16, [30 * (b % 7) for b in range(40)], window=20, sinks=3, seed=2)
    c.verify(page_table=dev(evicted(c, -1)))
