"""Context.tree_attention and Context.accept_sampled: what a call reports, and that calls in flight
write all of their results, each into memory that held something else."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_accept_sampled_gpu as W  # noqa: E402
from test_tree_attention_gpu import call, check, context, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes", [6, 40])
def test_cache_lengths_of_sequences_without_slots_are_reported(nodes):
    """Both walks: a sequence without a node and a root writes nothing, but its length counts."""
    c = make(2, nodes, [9, 12], 0, 2, 2, 64, "bfloat16", False, 0, n=[0, nodes], extra=0)
    ctx = context(c)
    good, zg, _ = call(ctx, c)
    check(c, good, zg)
    assert ctx.device_status() == 0
    for n in (-1, 13, 2 ** 31 - 1):
        lens = torch.tensor([n, 12], dtype=torch.int32, device="cuda")
        out, lse, _ = call(ctx, c, cache_len=lens)
        assert torch.equal(out, good) and torch.equal(lse, zg)
        assert ctx.device_status() == 5 and ctx.device_status() == 0, n
    ctx.close()


def test_attention_calls_in_flight_write_everything():
    """Two contexts on two streams, four calls each behind one another, with a workspace a context
    and outputs of their own that nothing has written."""
    cs = [make(3, 20, [900, 64, 333], 129, 8, 2, 128, "bfloat16", True, 1, seed=1),
          make(4, 0, [3000, 64, 2000, 1], 500, 8, 2, 64, "float16", False, 1, seed=2, chain=True,
               n=[0] * 4)]
    ctxs = [context(c) for c in cs]
    firsts = [call(ctx, c) for ctx, c in zip(ctxs, cs)]
    spaces, fresh = [], []
    for ctx, (out, lse, a) in zip(ctxs, firsts):
        need = ctx.tree_attention_workspace(**a)
        spaces.append(torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda"))
        fresh.append([(torch.full_like(out, 7.0), torch.full_like(lse, 7.0)) for _ in range(4)])
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for turn in range(4):
        for st, ctx, (_, _, a), w, f in zip(streams, ctxs, firsts, spaces, fresh):
            with torch.cuda.stream(st):
                ctx.tree_attention(**{**a, "workspace": w, "out": f[turn][0], "lse": f[turn][1]})
    torch.cuda.synchronize()
    for ctx, c, (first, z, _), f in zip(ctxs, cs, firsts, fresh):
        for out, lse in f:
            check(c, out, lse)
            assert torch.equal(out, first) and torch.equal(lse, z)
        assert ctx.device_status() == 0
        ctx.close()


def test_walks_in_flight_write_everything():
    cs = [W.make(6, 40, 7, 9001, "bfloat16", seed=1), W.make(3, 20, 9, 33333, "float32", seed=2)]
    ctxs = [W.context(c) for c in cs]
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    args, fresh = [], []
    for c in cs:
        z, B, L = c["z"].cuda(), len(c["n"]), c["L"]
        args.append(dict(n_nodes=cu(c["n"]), tokens=cu(c["tokens"]), parents=cu(c["parents"]),
                         root_logits=z[:, 0], node_logits=z[:, 1:], uniform=cu(c["u"]),
                         temperature=cu(c["T"])))
        full = lambda *s: torch.full(s, -77, dtype=torch.int32, device="cuda")
        fresh.append([dict(acc_len=full(B), acc_nodes=full(B, L), bonus=full(B),
                           logp=torch.full((B, L + 1), 7.0, device="cuda")) for _ in range(4)])
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for turn in range(4):
        for st, ctx, a, f in zip(streams, ctxs, args, fresh):
            with torch.cuda.stream(st):
                ctx.accept_sampled(**a, **f[turn])
    torch.cuda.synchronize()
    for ctx, c, f in zip(ctxs, cs, fresh):
        for o in f:
            W.check(c, (o["acc_len"], o["acc_nodes"], o["bonus"], o["logp"]))
        assert ctx.device_status() == 0
        ctx.close()
