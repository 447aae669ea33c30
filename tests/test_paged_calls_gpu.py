"""Calls of the paged operators that the other files do not make: chains behind a root, graphs whose lengths
change between replays, calls of several contexts in flight where walks are cut."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_paged_attention_gpu import BF, Q8, Case, dev  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [1, 4, 40])
def test_chains_behind_a_root(S):
    """with_root without a mask: one slot more than the nodes; n_nodes None: all slots."""
    c = Case(3, S, 8, 2, 64, 16, [60, 0, 201], counts=[S, 1, max(1, S - 2)], seed=S)
    c.check(*c.run(with_root=True, n_nodes=dev(c.counts - 1)))
    c.ctx.close()
    c = Case(3, S, 8, 2, 64, 16, [60, 0, 201], seed=S)
    c.check(*c.run(with_root=True, n_nodes=None))
    c.ctx.close()


def lengths(at, long):
    lens = 40 + np.arange(64) % 11
    lens[at] = long
    return lens.astype(np.int32)


@pytest.mark.parametrize("cache", [BF, Q8])
def test_replays_with_other_lengths(cache):
    """One graph, whose replays cut other sequences, or none: each as an eager call of these lengths."""
    S = 9
    c = Case(64, S, 16, 8, 16, 64, np.full(64, 4500), cache=cache, seed=1)
    lens, n = dev(lengths(0, 4500)), dev(np.full(64, S, np.int32))
    out, lse = torch.zeros_like(c.q, device="cuda"), torch.zeros(c.q.shape[:3], device="cuda")
    a = dict(c.args(), cache_len=lens, n_nodes=n, out=out, lse=lse)
    a["workspace"] = torch.full((c.ctx.paged_attention_workspace(**a),), 0xFF, dtype=torch.uint8, device="cuda")
    c.ctx.paged_attention(**a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.ctx.paged_attention(**a)
    for k, x in enumerate([lengths(0, 4500), lengths([3, 63], 4500), np.full(64, 4500), lengths(0, 0), np.zeros(64), lengths(31, 4000)]):
        c.lens = np.asarray(x, np.int32)
        c.counts = np.full(64, S, np.int32)
        c.counts[k::7] = 0
        lens.copy_(torch.from_numpy(c.lens)), n.copy_(torch.from_numpy(c.counts))
        eager = c.run()
        out.fill_(7), lse.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1]), k
    assert c.ctx.device_status() == 0
    c.lens = lengths(31, 4000)
    c.check(out, lse)
    del g
    c.ctx.close()


def test_cut_calls_in_flight():
    """Three contexts on streams of their own, some calls behind one another in each."""
    cases = [Case(64, 9, 16, 8, 16, 64, lengths(at, 5000), seed=at) for at in (0, 30, 63)]
    args = [c.args() for c in cases]
    want = [c.run() for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], [[] for _ in cases]
    for turn in range(4):
        for i, (c, a, s) in enumerate(zip(cases, args, streams)):
            with torch.cuda.stream(s):
                out, lse = torch.full_like(want[i][0], 7.0), torch.full_like(want[i][1], 7.0)
                c.ctx.paged_attention(**a, out=out, lse=lse)
                got[i].append((out, lse))
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
        c.check(*want[i])
        c.ctx.close()
