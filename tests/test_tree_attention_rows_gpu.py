"""Context.tree_attention: a row depends on its own query and on the keys it sees, to the bit.
Other rows' queries, other sequences' queries in the shared prefix's own pass, and large finite
keys that a row does not see change none of its bits, in either walk."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_tree_attention_gpu import call, check, context, make  # noqa: E402

pytestmark = pytest.mark.gpu

# nodes, query heads, key heads, keys: up to 16 and 32 rows of a key head (the narrow walk, whose
# parts take several rounds of tiles from 64 * 128 keys on), 33 to 64 and more (the wide one)
WALKS = [(14, 2, 2, 17000), (13, 4, 2, 17000), (40, 2, 2, 400), (67, 2, 1, 400)]
KINDS = ["bfloat16", "float16", "e4m3"]


def inputs(kind, seed, batch, nodes, lens, shared, Hq, H, D, **kw):
    c = make(batch, nodes, lens, shared, Hq, H, D, "bfloat16" if kind == "e4m3" else kind,
             kind == "e4m3", 1, seed=seed, **kw)
    c["k"] *= 1.5           # maxima rise again in the block, by less than a rescaling takes
    return c


def bits(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


def same(a, b):
    return torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("walk", WALKS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shared", [0, 1])
def test_other_rows_queries(walk, kind, shared):
    """Half of the queries of a sequence are made 10 times as large: the others' rows stay."""
    nodes, Hq, H, keys = walk
    for seed in range(4):
        print("rows", walk, kind, shared, seed, flush=True)
        c = inputs(kind, seed, 2, nodes, [keys, 129], shared * keys // 2, Hq, H, 64, chain=True,
                   n=[nodes, nodes])
        ctx = context(c)
        out, lse, _ = call(ctx, c)
        if seed == 0:
            check(c, out, lse)
        c["q"][:, 1::2] *= 10.0
        far, zfar, _ = call(ctx, c)
        assert same(far[:, ::2].contiguous(), out[:, ::2].contiguous()), seed
        assert same(zfar[:, ::2].contiguous(), lse[:, ::2].contiguous()), seed
        ctx.close()


@pytest.mark.parametrize("nodes,Hq,H", [(0, 8, 2), (3, 8, 2), (11, 8, 2), (31, 2, 1)])
@pytest.mark.parametrize("kind", KINDS)
def test_other_sequences_queries(nodes, Hq, H, kind):
    """The shared prefix's own pass takes rows of several sequences into a tile."""
    for seed in range(4):
        print("sequences", nodes, Hq, H, kind, seed, flush=True)
        c = inputs(kind, seed, 6, nodes, [5, 70, 0, 200, 1, 64], 9000, Hq, H, 64, chain=True,
                   n=[nodes] * 6)
        ctx = context(c)
        out, lse, _ = call(ctx, c)
        c["q"][1::2] *= 10.0
        far, zfar, _ = call(ctx, c)
        assert same(far[::2].contiguous(), out[::2].contiguous()), seed
        assert same(zfar[::2].contiguous(), lse[::2].contiguous()), seed
        ctx.close()


@pytest.mark.parametrize("walk", WALKS)
@pytest.mark.parametrize("kind", KINDS)
def test_large_finite_hidden_keys(walk, kind):
    """The chain's last slots get keys 20 times as large: the slots before them, which do not see
    them, stay."""
    nodes, Hq, H, keys = walk
    for seed in range(4):
        print("hidden keys", walk, kind, seed, flush=True)
        c = inputs(kind, seed, 2, nodes, [keys + 100, 20], 0, Hq, H, 64, chain=True, n=[nodes, nodes - 1])
        ctx = context(c)
        out, lse, _ = call(ctx, c)
        hurt = nodes - 3
        c["k"][:, hurt:] *= 20.0
        far, zfar, _ = call(ctx, c)
        assert same(far[:, :hurt].contiguous(), out[:, :hurt].contiguous()), seed
        assert same(zfar[:, :hurt].contiguous(), lse[:, :hurt].contiguous()), seed
        ctx.close()
