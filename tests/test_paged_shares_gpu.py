"""How the paged attention shares its rounds: more sequences than threads, sequences that take none,
more pieces than a merge holds, row tiles that a piece leaves nothing, and groups that no rounds are left
for."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_paged_attention_gpu import BF, Q8, Case  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [255, 256, 257, 600])
@pytest.mark.parametrize("S,group", [(1, 2), (9, 5)])
def test_more_sequences_than_threads(B, S, group):
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 400, B)
    lens[::7] = 0
    counts = np.where(rng.random(B) < 0.2, 0, S)
    counts[-1] = S
    Case(B, S, 2 * group, 2, 16, 16, lens, counts=counts, seed=B).verify()


@pytest.mark.parametrize("S", [1, 3, 40])
@pytest.mark.parametrize("cache", [BF, Q8])
def test_one_long_sequence(S, cache):
    """One key head: more even pieces than the merge takes, so longer ones."""
    Case(1, S, 2, 1, 16, 128, [70000], cache=cache, seed=S).verify()
    Case(2, S, 2, 1, 64, 64, [30000, 3], cache=cache, seed=S).verify()


@pytest.mark.parametrize("n,S", [(0, 600), (10, 600), (700, 600), (0, 1000), (63, 129), (64, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 5)])
def test_prompts_from_the_first_row_on(n, S, window, sinks):
    """The first row tiles see one tile of keys, the last ones many."""
    Case(1, S, 4, 1, 32, 16, [n], window=window, sinks=sinks, seed=n + S).verify()
    Case(2, S, 2, 1, 64, 24, [n, n // 2], counts=[S, S // 3], window=window, sinks=sinks, seed=n + S).verify()


def test_one_sequence_among_empty_ones():
    for S, group in ((1, 4), (20, 4)):
        counts = np.zeros(64, np.int64)
        counts[37] = S
        lens = np.arange(64) * 11
        lens[37] = 5000
        Case(64, S, group, 1, 32, 16, lens, counts=counts, seed=1).verify()
        Case(64, S, group, 1, 32, 16, lens, counts=np.zeros(64, np.int64), seed=1).verify()


def test_many_units_take_no_pieces():
    """1024 row tiles and more: a workgroup each."""
    Case(40, 40, 64, 32, 16, 16, [30 * (b % 5) for b in range(40)], counts=[40 - b % 3 for b in range(40)], seed=2).verify()
    Case(1, 1100, 128, 64, 16, 16, [50], seed=3, n_max=8).verify()
