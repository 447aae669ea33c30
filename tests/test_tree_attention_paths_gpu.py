"""Context.tree_attention where sequences of one batch take different ways through it: caches
of very different lengths (one part beside many), the shared prefix's own pass for wide
blocks, every head size in both walks, two calls at once.  Bounds as in verifier_ref."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_tree_attention_gpu import call, check, context, make  # noqa: E402

pytestmark = pytest.mark.gpu


def run(c):
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    assert ctx.device_status() == 0
    ctx.close()


@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("nodes", [2, 9, 40])
@pytest.mark.parametrize("quant", [False, True])
def test_every_head_size(D, nodes, quant):
    """16, 32 and more rows a key head: the narrow walk of one and two column tiles, the wide."""
    print("head size", D, nodes, quant, flush=True)
    run(make(2, nodes, [75, 31], 40, 6, 2, D, "bfloat16", quant, 1, seed=D + nodes))


@pytest.mark.parametrize("kind", ["bfloat16", "float16", "e4m3"])
@pytest.mark.parametrize("nodes", [0, 5, 30])
def test_short_and_long_caches_in_one_batch(kind, nodes):
    """Sequences of one part write their rows themselves, the others' parts are joined."""
    print("mixed lengths", kind, nodes, flush=True)
    run(make(5, nodes, [10, 3900, 0, 64, 700], 0, 8, 2, 128, "bfloat16" if kind == "e4m3" else kind,
             kind == "e4m3", 1, seed=nodes, n=[nodes, nodes, nodes // 2, nodes, 0], chain=nodes == 0))


@pytest.mark.parametrize("kind", ["bfloat16", "float16", "e4m3"])
@pytest.mark.parametrize("nodes,Hq,H", [(11, 8, 2), (15, 4, 1), (8, 14, 2), (31, 2, 1)])
def test_the_shared_prefix_of_wide_blocks(kind, nodes, Hq, H):
    """33 to 64 rows a sequence and key head: the wide walk's pass of the shared prefix, whose
    row tiles hold rows of several sequences."""
    print("shared, wide", kind, nodes, Hq, H, flush=True)
    run(make(5, nodes, [0, 5, 800, 64, 129], 777, Hq, H, 96, "bfloat16" if kind == "e4m3" else kind,
             kind == "e4m3", 1, seed=nodes, n=[nodes, 0, nodes, 1, nodes - 1]))


@pytest.mark.parametrize("shared", [1, 31, 128, 129, 1000])
def test_shared_prefix_and_no_cache(shared):
    run(make(3, 6, [], shared, 4, 4, 64, "float16", False, 1, seed=shared))
    run(make(1, 6, [], shared, 4, 4, 64, "bfloat16", True, 1, seed=shared))


@pytest.mark.parametrize("quant", [False, True])
def test_more_sequences_than_parts_fill(quant):
    """Many short sequences of every length around a tile."""
    lens = [i % 70 for i in range(96)]
    run(make(96, 1, lens, 0, 4, 1, 64, "bfloat16", quant, 1, seed=5, n=[i % 2 for i in range(96)]))


def test_two_calls_at_once():
    """Two contexts' calls in flight on two streams, each with a workspace of its own."""
    cs = [make(3, 20, [900, 64, 333], 129, 8, 2, 128, "bfloat16", True, 1, seed=1),
          make(4, 0, [3000, 64, 2000, 1], 500, 8, 2, 64, "float16", False, 1, seed=2, chain=True,
               n=[0] * 4)]
    ctxs = [context(c) for c in cs]
    firsts = [call(ctx, c) for ctx, c in zip(ctxs, cs)]
    streams = [torch.cuda.Stream() for _ in cs]
    spaces = []
    for ctx, (_, _, a) in zip(ctxs, firsts):
        need = ctx.tree_attention_workspace(**a)
        spaces.append(torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(4):
        for st, ctx, (_, _, a), w in zip(streams, ctxs, firsts, spaces):
            with torch.cuda.stream(st):
                ctx.tree_attention(**{**a, "workspace": w})
    torch.cuda.synchronize()
    for ctx, c, (out, lse, _) in zip(ctxs, cs, firsts):
        check(c, out, lse)
        ctx.close()


def test_small_quantised_keys_and_values():
    """Keys of size 2^-100 (scores of nothing) and values of size 2^-20."""
    import verifier_ref as R
    c = make(1, 4, [40], 0, 2, 1, 32, "bfloat16", True, 1, seed=3)
    for i, e in enumerate((-100, -20)):
        x = torch.randn(1, c["cache"][0][0].shape[1], 1, 32,
                        generator=torch.Generator().manual_seed(i)).to(torch.bfloat16)
        c["cache"][i] = R.quantise((x.double() * 2.0 ** e).to(torch.bfloat16))
    run(c)


def test_slots_past_the_block_are_not_read():
    """NaN in every tensor's unused places: slots behind the block, rows behind the cache,
    neighbours of a strided row."""
    c = make(2, 12, [33, 90], 17, 4, 2, 64, "bfloat16", False, 1, seed=8, n=[12, 3])
    wide = {}
    for name in ("q", "k", "v"):
        t = c[name]
        w = torch.full((*t.shape[:-1], 96), float("nan"), dtype=t.dtype, device="cuda")
        w[..., 16:80] = t.cuda()
        for b in range(2):
            w[b, int(c["n"][b]) + 1:] = float("nan")
        wide[name] = w[..., 16:80]
    ctx = context(c)
    out, lse, _ = call(ctx, c, **wide)
    check(c, out, lse)
    ctx.close()


@pytest.mark.parametrize("nodes", [1, 40])
@pytest.mark.parametrize("quant", [False, True])
def test_one_sequence_past_32_bit_offsets(nodes, quant):
    """Rows 4 MB apart, so that a sequence's later tiles start more than 2^31 bytes after its
    first."""
    rows = 600
    c = make(1, nodes, [rows], 0, 2, 1, 64, "bfloat16", quant, 1, seed=nodes, extra=0)
    import paper_2608_20375_amd as G
    space = torch.empty(rows * (1 << 22), dtype=torch.uint8, device="cuda")
    pair = []
    for i, x in enumerate(c["cache"]):
        codes = x[0] if quant else x
        at = space.view(codes.dtype)
        per = at.numel() // rows
        far = at.as_strided((1, rows, 1, 64), (0, per, 64, 1), 128 * i)
        far.copy_(codes.cuda())
        pair.append(G.QuantRows(far, x[1].cuda()) if quant else far)
    ctx = context(c)
    out, lse, _ = call(ctx, c, cache=tuple(pair))
    check(c, out, lse)
    ctx.close()
