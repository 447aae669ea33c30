"""Context.accept_sampled at sizes where its kernel takes other turns: rows of more than one
vector a lane and run, trees of more nodes than a wave looks at at once, paths that are long,
two calls in flight.  Compared as in test_accept_sampled_gpu."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_accept_sampled_gpu import call, check, context, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,V", [("float32", 262143), ("float32", 262147), ("float32", 300001),
                                     ("float32", 1100003), ("bfloat16", 524287), ("bfloat16", 600011),
                                     ("float16", 1300001)])
def test_long_rows(dtype, V):
    print("long rows", dtype, V, flush=True)
    c = make(3, 4, 3, V, dtype, seed=V % 1000, T=[1.0, 0.0, 0.7])
    ctx = context(c)
    acc = check(c, call(ctx, c))
    for u in (0.0, 1.0 - 2.0 ** -53, 2.0):
        c["u"][:] = u
        check(c, call(ctx, c))
    assert ctx.device_status() == 0 and acc.max() > 0
    ctx.close()


@pytest.mark.parametrize("V", [262147, 600011])
def test_long_rows_of_few_tokens(V):
    """Masked everywhere but at a few places, at a row's ends among them; ties of the largest."""
    c = make(2, 3, 2, V, "float32" if V < 500000 else "bfloat16", seed=9, T=[1.0, 0.0])
    z = c["z"]
    z[:] = float("-inf")
    rng = np.random.default_rng(4)
    for b in range(2):
        for r in range(z.shape[1]):
            z[b, r, [0, V - 1]] = 1.0
            z[b, r, torch.from_numpy(rng.integers(0, V, 3))] = 0.5
    for u in (0.0, 0.3, 0.6, 0.999999):
        c["u"][:] = u
        ctx = context(c)
        check(c, call(ctx, c))
        ctx.close()


@pytest.mark.parametrize("nodes", [255, 256, 257, 300, 700, 1024])
def test_large_trees(nodes):
    c = make(3, nodes, 8, 2003, "bfloat16", seed=nodes, n=[nodes, nodes - 1, nodes // 2], mass=0.97)
    ctx = context(c)
    check(c, call(ctx, c))
    ctx.close()


def test_a_long_path_through_late_nodes():
    """A path of 60 nodes whose tokens are all but certain, each the last of five."""
    L, n, V = 60, 300, 611
    rng = np.random.default_rng(3)
    tokens = rng.integers(0, V - 1, (2, n)).astype(np.int32)
    parents = np.full((2, n), -1, np.int32)
    path = np.arange(4, n, 5)
    parents[:, path[1:]] = path[:-1]
    tokens[:, np.setdiff1d(np.arange(n), path)] = V - 1
    z = torch.from_numpy(rng.normal(size=(2, n + 1, V)).astype(np.float32))
    for b in range(2):
        rows = torch.from_numpy(np.concatenate([[-1], path[:-1]]) + 1)
        z[b, rows, torch.from_numpy(tokens[b, path]).long()] = 60.0
    c = dict(z=z, parents=parents, tokens=tokens, n=np.asarray([n, 280], np.int32),
             u=rng.random((2, L + 1)), T=np.ones(2, np.float32), L=L, V=V)
    ctx = context(c)
    acc = check(c, call(ctx, c))
    assert acc.tolist() == [60, 56]
    ctx.close()


def test_two_calls_at_once():
    cs = [make(6, 40, 7, 9001, "bfloat16", seed=1), make(3, 20, 9, 33333, "float32", seed=2)]
    ctxs = [context(c) for c in cs]
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    args = []
    for c in cs:
        z = c["z"].cuda()
        args.append(dict(n_nodes=cu(c["n"]), tokens=cu(c["tokens"]), parents=cu(c["parents"]),
                         root_logits=z[:, 0], node_logits=z[:, 1:], uniform=cu(c["u"]),
                         temperature=cu(c["T"])))
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = ctxs[i].accept_sampled(**args[i])
    torch.cuda.synchronize()
    for ctx, c, g in zip(ctxs, cs, got):
        check(c, g)
        ctx.close()
