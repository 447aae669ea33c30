"""The accepted path's rows moved up in the pages (paged_commit), byte for byte."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paged_ref as R  # noqa: E402
import paper_2608_20375_amd as G  # noqa: E402

pytestmark = pytest.mark.gpu

BF, FP, Q8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def parts(p):
    return (p.codes, p.scales) if isinstance(p, G.QuantRows) else (p.view(torch.int16),)


def check(B, L, N, planes, H, D, page, cache=BF, root=True, starts=None, paths=None, pool=None, seed=0):
    rng = np.random.default_rng(seed)
    starts = np.asarray(starts if starts is not None else rng.integers(0, 4 * page, B), np.int32)
    if paths is None:
        paths = [np.sort(rng.choice(N, min(L, rng.integers(0, L + 1), N), replace=False)) for _ in range(B)]
    t, pages = R.table(rng, page, starts + N + 1)
    p = G.paged_cache(pages + 1, page, H, D, cache, planes=planes) if pool is None else pool(pages + 1)
    for x in parts(p):
        x.copy_(torch.randint(0, 120, x.shape, dtype=x.dtype, device="cuda"))
    want = [x.cpu().clone() for x in parts(p)]
    nodes = np.full((B, L), -1, np.int32)
    for b in range(B):
        nodes[b, :len(paths[b])] = paths[b]
        first = int(starts[b]) + (1 if root else 0)
        at = lambda r: (int(t[b][r // page]), r % page)
        for x in want:
            old = x.clone()
            for i, j in enumerate(paths[b]):
                (p0, r0), (p1, r1) = at(first + int(j)), at(first + i)
                x[:, p1, r1] = old[:, p0, r0]
    ctx = G.Context(B, L, 64, 1, N)
    got = ctx.paged_commit(p, dev(t), dev(starts), dev(np.array([len(x) for x in paths], np.int32)), dev(nodes), with_root=root)
    assert got is p and ctx.device_status() == 0
    for x, y in zip(parts(p), want):
        assert torch.equal(x.cpu(), y)
    ctx.close()


@pytest.mark.parametrize("cache", [BF, FP, Q8])
@pytest.mark.parametrize("D,H", [(16, 1), (48, 3), (80, 4), (128, 8)])
@pytest.mark.parametrize("page", [1, 7, 16, 64])
def test_paths(cache, D, H, page):
    check(3, 12, 40, 5, H, D, page, cache=cache, seed=D + page)


@pytest.mark.parametrize("L,N", [(1, 1), (4, 4), (16, 16), (17, 64), (33, 100), (64, 64), (64, 1024)])
def test_depths(L, N):
    """Paths over more than one group of rows; chains, whose rows stay; rows that are source and
    destination both."""
    check(4, L, N, 3, 2, 64, 16, seed=L)
    up = [np.arange(L), np.arange(L) + min(1, N - L), np.arange(L) + (N - L), np.arange(0, L)]
    check(4, L, N, 3, 2, 64, 16, paths=up, seed=L)
    check(4, L, N, 2, 2, 64, 24, paths=[x[x.size // 2:] for x in up], root=False, cache=Q8, seed=L)


def test_batches_and_planes():
    check(64, 16, 128, 72, 8, 128, 64, starts=[64] * 64, seed=1)
    check(1, 16, 64, 200, 1, 16, 16, seed=2)
    check(2, 8, 64, 3, 1000, 16, 16, seed=2, cache=Q8)


def test_empty_paths():
    check(3, 4, 9, 2, 2, 32, 8, paths=[[], [], []])
    check(3, 4, 9, 2, 2, 32, 8, paths=[[], [3, 8], []], starts=[0, 0, 0])


def test_layouts():
    check(2, 8, 30, 4, 2, 64, 16, pool=lambda n: torch.empty(4, n, 16, 2, 64, dtype=BF, device="cuda"))
    check(2, 8, 30, 4, 2, 64, 16, pool=lambda n: torch.empty(n, 2, 16, 4, 80, dtype=BF, device="cuda")[..., :64].permute(3, 0, 2, 1, 4))
    check(2, 8, 30, 4, 2, 64, 16, cache=Q8, pool=lambda n: G.QuantRows.empty(4, n, 16, 2, 64))


def test_no_start():
    ctx = G.Context(1, 4, 64, 1, 9)
    p = torch.arange(12, device="cuda").view(1, 3, 4, 1, 1).expand(1, 3, 4, 1, 16).to(BF).contiguous()
    t = dev(np.array([[2, 0, 1]], np.int32))
    ctx.paged_commit(p, t, None, dev(np.array([2], np.int32)), dev(np.array([[1, 6, -1, -1]], np.int32)))
    assert p[0, 2, :, 0, 0].tolist() == [9, 2, 10, 11] and p[0, 0, :, 0, 0].tolist() == [0, 1, 2, 3]
    assert ctx.device_status() == 0
    ctx.close()


def test_what_is_outside_is_skipped_and_reported():
    """Node indices, rows and pages that there are none of."""
    base = torch.arange(24, device="cuda").view(1, 6, 4, 1, 1).expand(1, 6, 4, 1, 16).to(BF)
    cases = [([0], [[0, 1]], [3], [[2, -1, 5, 0]], [3], {0: 2, 2: 5}),          # a negative node
             ([0], [[0, 1]], [3], [[3, 9, 7, 0]], [3], {0: 3, 2: 7}),           # a node past max_nodes
             ([4], [[0, 1]], [2], [[1, 6, 0, 0]], [2], {4: 5}),                 # a row past the table
             ([-1], [[0, 1]], [2], [[1, 5, 0, 0]], [2], {0: 4}),                # a row before it
             ([0], [[0, 6]], [2], [[1, 5, 0, 0]], [2], {0: 1}),                 # a page past the pool
             ([0], [[0, -1]], [2], [[1, 5, 0, 0]], [2], {0: 1})]
    for start, table, n, nodes, _, moved in cases:
        ctx = G.Context(1, 4, 64, 1, 9)
        p = base.contiguous()
        ctx.paged_commit(p, dev(np.array(table, np.int32)), dev(np.array(start, np.int32)), dev(np.array(n, np.int32)),
                         dev(np.array(nodes, np.int32)))
        assert ctx.device_status() != 0 and ctx.device_status() == 0
        want = base.contiguous()
        for to, src in moved.items():
            want[0, table[0][to // 4], to % 4] = base[0, table[0][src // 4], src % 4]
        assert torch.equal(p, want), (start, table, nodes)
        ctx.close()


def test_lengths_outside_are_clamped():
    ctx = G.Context(2, 2, 64, 1, 9)
    p = torch.arange(24, device="cuda").view(1, 6, 4, 1, 1).expand(1, 6, 4, 1, 16).to(BF).contiguous()
    t = dev(np.array([[0, 1, 2], [3, 4, 5]], np.int32))
    ctx.paged_commit(p, t, None, dev(np.array([-1, 9], np.int32)), dev(np.array([[3, 4], [3, 4]], np.int32)))
    assert p[0, 0, :, 0, 0].tolist() == [0, 1, 2, 3] and p[0, 3, :, 0, 0].tolist() == [15, 16, 14, 15]
    ctx.close()
