"""Paged calls with columns of a wider table, which belongs to more sequences than the call's."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_20375_amd as G  # noqa: E402
from test_paged_attention_gpu import BF, Q8, Case, dev  # noqa: E402

pytestmark = pytest.mark.gpu


def wider(t):
    """The table as rows 0, 2, 4 .. and columns 3 .. of one whose other entries name nothing."""
    w = np.full((2 * t.shape[0] + 1, t.shape[1] + 8), -9, np.int32)
    w[:2 * t.shape[0]:2, 3:3 + t.shape[1]] = t
    w = dev(w)[::2, 3:3 + t.shape[1]]
    assert not w.is_contiguous() and w.shape[0] > t.shape[0]
    return w


@pytest.mark.parametrize("S", [1, 5, 40])
@pytest.mark.parametrize("cache", [BF, Q8])
@pytest.mark.parametrize("page", [16, 24])
def test_attention(S, cache, page):
    c = Case(3, S, 8, 2, 64, page, [100, 0, 333], cache=cache, seed=S)
    c.check(*c.run(page_table=wider(c.table)))
    one = Case(1, S, 8, 2, 64, page, [100], cache=cache, seed=S)
    one.verify(page_table=wider(one.table))
    c.ctx.close()


def test_write_and_commit():
    g = torch.Generator(device="cuda").manual_seed(3)
    table = np.array([[4, 1, 7], [0, 6, 2]], np.int32)
    k, v = (torch.randn(2, 20, 2, 64, dtype=BF, device="cuda", generator=g) for _ in range(2))
    start, n = dev(np.array([3, 20], np.int32)), dev(np.array([20, 17], np.int32))
    acc, nodes = dev(np.array([2, 3], np.int32)), dev(np.array([[1, 4, -1], [0, 5, 9]], np.int32))
    ctx = G.Context(2, 3, 64, 1, 20)
    pools = []
    for t in (dev(table), wider(table)):
        pool = G.paged_cache(8, 16, 2, 64, BF, planes=2)
        pool.fill_(5)
        ctx.paged_write((pool[0], pool[1]), t, k, v, n, start)
        ctx.paged_commit(pool, t, start, acc, nodes, with_root=True)
        assert ctx.device_status() == 0
        pools.append(pool)
    assert torch.equal(*pools) and not torch.all(pools[0] == 5)
    ctx.close()
