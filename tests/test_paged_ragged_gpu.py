"""Batches of the wide walk in which one sequence, or a few, are far longer than the others: with as many row tiles
as run at once, and with more, their walks are cut and joined."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_paged_attention_gpu import BF, FP, Q8, Case  # noqa: E402

pytestmark = pytest.mark.gpu


def lengths(B, at, long, short=30):
    lens = short + np.arange(B) % 7
    lens[list(at)] = long
    return lens


def twice(c):
    """The result against fp64, and the same bits from a workspace that holds NaN."""
    a = c.run()
    c.check(*a)
    x = c.args()
    need = c.ctx.paged_attention_workspace(**x)
    assert need > 0
    w = torch.full((need // 4 + 4,), float("nan"), device="cuda").view(torch.uint8)[:need]
    b = c.run(workspace=w)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    c.ctx.close()


@pytest.mark.parametrize("B", [50, 63, 64, 65, 100, 257])
@pytest.mark.parametrize("at", [(0,), (31,), (-1,), (3, 4, 40)])
def test_one_or_a_few_long_sequences(B, at):
    """400 to 2056 row tiles; up to 64 sequences every wave adds up for itself."""
    print(B, at, flush=True)
    twice(Case(B, 9, 16, 8, 16, 16, lengths(B, at, 6000), seed=B))


@pytest.mark.parametrize("cache,dtype", [(BF, BF), (FP, FP), (Q8, BF)])
@pytest.mark.parametrize("tree", [False, True])
def test_types_and_trees(cache, dtype, tree):
    """Three row tiles a sequence, of which some have fewer or none; most slots of a join's workgroups."""
    n = 65
    counts = np.array([n - 5 * (b % 13) for b in range(40)])
    counts[[7, 20]] = 1
    twice(Case(40, n, 32, 8, 64, 64, lengths(40, (5, 7, 39), 5000), counts=counts, tree=tree, cache=cache, dtype=dtype, seed=3,
               n_max=64))


def test_empty_and_lone_sequences():
    counts = np.zeros(64, np.int64)
    counts[[2, 63]] = 9
    twice(Case(64, 9, 16, 8, 16, 16, lengths(64, (2,), 9000), counts=counts, seed=4))
    Case(64, 9, 16, 8, 16, 16, lengths(64, (2,), 9000), counts=np.zeros(64, np.int64), seed=4).verify()


def test_all_long():
    twice(Case(66, 9, 16, 8, 16, 128, np.full(66, 4500), seed=5))


@pytest.mark.parametrize("window,sinks", [(4500, 70), (5000, 0)])
def test_long_windows(window, sinks):
    twice(Case(64, 9, 16, 8, 16, 24, lengths(64, (0, 50), 7000, 2000), window=window, sinks=sinks, seed=6))


def test_prompts():
    """Row tiles in the thousands, whose joins go over the rows in turns."""
    twice(Case(4, 700, 32, 8, 16, 64, [9000, 0, 64, 4000], counts=[700, 700, 1, 350], seed=7, n_max=8))
    twice(Case(1, 2100, 32, 8, 16, 64, [5000], seed=8, n_max=8))


def test_many_pieces():
    """The longest walk is of more pieces than a join holds, unless they are made longer."""
    twice(Case(64, 17, 8, 8, 16, 128, lengths(64, (9,), 150000, 0), seed=9))
