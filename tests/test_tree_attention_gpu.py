"""Context.tree_attention against the same attention in 64 bits: types, head layouts,
lengths from none to long ones, odd sizes, strides, masks, splits, and what hidden slots
hold.  Tolerances are verifier_ref.attention's, derived there."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import verifier_ref as R  # noqa: E402

pytestmark = pytest.mark.gpu


def make(batch, nodes, lens, shared, Hq, H, D, dtype, quant, root, seed=0, chain=False, n=None,
         depth=6, qscale=2.0, extra=3):
    """Inputs of one call on the GPU and their CPU copies."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed + 1)
    dt = getattr(torch, dtype)
    S = nodes + root
    norm = lambda *s: torch.randn(*s, generator=g).to(dt)
    c = dict(q=norm(batch, S, Hq, D) * qscale, k=norm(batch, S, H, D), v=norm(batch, S, H, D))
    N = max(nodes, 1)
    n = np.asarray(n if n is not None else
                   [nodes - (i * 7) % max(1, nodes) for i in range(batch)], np.int32)
    mask = np.zeros((batch, N, (N + 63) // 64), np.int64)
    seen = []
    for b in range(batch):
        nb = int(n[b])
        bits = (np.tril(np.ones((nb, nb), bool)) if chain
                else R.random_tree(rng, nb, depth)[2])
        mask[b] = R.pack_mask(bits, N)
        full = np.zeros((nb + root, nb + root), bool)
        full[root:, root:] = bits
        if root:
            full[:, 0] = True
        seen.append(full)
    lens = np.asarray(lens, np.int32)
    rows = int(lens.max(initial=0)) + extra if len(lens) else 0
    cache = shared_kv = None
    val = lambda pair: [R.values(*x) if quant else x.double() for x in pair]
    if rows:
        cache = [norm(batch, rows, H, D) for _ in range(2)]
        if quant:
            cache = [R.quantise(x) for x in cache]
    if shared:
        shared_kv = [norm(shared, H, D) for _ in range(2)]
        if quant:
            shared_kv = [R.quantise(x) for x in shared_kv]
    c.update(n=n, mask=mask, seen=seen, lens=lens, cache=cache, shared=shared_kv, quant=quant,
             root=root, val=val, chain=chain, dt=dt, H=H, D=D)
    return c


def context(c):
    import paper_2608_20375_amd as G
    B, S = c["q"].shape[:2]
    return G.Context(B, 8, 64, 1, max(1, S - c["root"]))


def call(ctx, c, lse=True, **kw):
    import paper_2608_20375_amd as G
    cu = lambda t: None if t is None else t.cuda()
    pair = lambda p: None if p is None else tuple(
        G.QuantRows(*[t.cuda() for t in x]) if c["quant"] else x.cuda() for x in p)
    B, S, Hq, _ = c["q"].shape
    a = dict(q=cu(c["q"]), k=cu(c["k"]), v=cu(c["v"]), n_nodes=torch.from_numpy(c["n"]).cuda(),
             mask=None if c["chain"] else torch.from_numpy(c["mask"]).cuda(), cache=pair(c["cache"]),
             cache_len=torch.from_numpy(c["lens"]).cuda() if c["cache"] is not None else None,
             shared=pair(c["shared"]), with_root=bool(c["root"]),
             out=torch.full_like(c["q"], 7.0).cuda(),
             lse=torch.full((B, S, Hq), 7.0, device="cuda") if lse else None)
    a.update(kw)
    out = ctx.tree_attention(**a)
    return out, a["lse"], a


def check(c, out, lse, scale=None):
    D, H = c["D"], c["H"]
    scale = D ** -0.5 if scale is None else scale
    eps = torch.finfo(c["dt"]).eps
    out, lse = out.cpu().double(), None if lse is None else lse.cpu().double()
    none = torch.zeros(0, H, D, dtype=torch.float64)
    shared = c["val"](c["shared"]) if c["shared"] is not None else [none, none]
    for b in range(len(c["n"])):
        m = int(c["n"][b]) + c["root"]
        own = [none, none]
        if c["cache"] is not None:
            L = int(c["lens"][b])
            own = [x[b, :L] for x in c["val"](c["cache"])]
        ref, z, tol, ztol = R.attention(
            c["q"][b, :m].double(), c["k"][b, :m].double(), c["v"][b, :m].double(), c["seen"][b],
            torch.cat([shared[0], own[0]]), torch.cat([shared[1], own[1]]), scale, eps)
        far = (out[b, :m] - ref).abs() - tol
        assert not torch.isnan(out[b, :m]).any(), b
        assert (far <= 0).all(), (b, float(far.max()))
        assert (out[b, m:] == 7.0).all(), b
        if lse is not None:
            same = (lse[b, :m] == z) | ((lse[b, :m] - z).abs() <= ztol)
            assert same.all(), b
            assert (lse[b, m:] == 7.0).all(), b


SHAPES = [
    # batch, nodes, cache lengths, shared, Hq, H, D
    (1, 1, [0], 0, 1, 1, 16),            # a node alone: it sees itself
    (1, 1, [1], 0, 4, 4, 64),
    (2, 5, [63, 64], 0, 8, 2, 128),      # around a tile of keys
    (3, 70, [65, 1, 0], 0, 5, 1, 80),    # odd group, odd dimension, an empty cache
    (2, 64, [130, 7], 3, 4, 2, 32),      # a shared prefix that fills no tile
    (1, 130, [200], 64, 14, 2, 48),      # rows of several tiles, group 7
    (5, 3, [10, 300, 64, 129, 1], 257, 8, 8, 128),   # shared prefix's own pass, rows of all
    (2, 200, [100, 33], 130, 2, 2, 112),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "b%d_n%d_D%d" % (s[0], s[1], s[6]))
@pytest.mark.parametrize("kind", ["bfloat16", "float16", "e4m3"])
@pytest.mark.parametrize("root", [0, 1])
def test_shapes(shape, kind, root):
    print("attention", shape, kind, root, flush=True)
    batch, nodes, lens, shared, Hq, H, D = shape
    c = make(batch, nodes, lens, shared, Hq, H, D, "bfloat16" if kind == "e4m3" else kind,
             kind == "e4m3", root, seed=nodes + D)
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    assert ctx.device_status() == 0
    ctx.close()


@pytest.mark.parametrize("batch,lens,shared", [(1, [1], 0), (1, [2000], 0), (3, [5, 0, 4100], 0),
                                               (40, None, 513), (2, [1, 1], 4000)])
@pytest.mark.parametrize("quant", [False, True])
def test_single_tokens(batch, lens, shared, quant):
    """The root alone (no nodes): ordinary decoding, over long caches split into parts."""
    print("single", batch, lens, shared, quant, flush=True)
    lens = [(37 * i) % 301 for i in range(batch)] if lens is None else lens
    c = make(batch, 0, lens, shared, 8, 2, 64, "bfloat16", quant, 1, seed=batch, chain=True,
             n=[0] * batch)
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    ctx.close()


@pytest.mark.parametrize("root", [0, 1])
def test_chain_without_a_mask(root):
    c = make(2, 67, [9, 64], 5, 4, 2, 64, "float16", False, root, chain=True, n=[67, 0])
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    ctx.close()


def test_every_word_of_a_full_mask():
    """max_nodes a multiple of 64 with the root: the block's last slot is in a tile whose
    mask word does not exist."""
    c = make(1, 128, [3], 0, 2, 1, 64, "bfloat16", False, 1, n=[128])
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    ctx.close()


def test_fewer_slots_than_the_context_has():
    """slots below max_nodes: the mask keeps the context's rows and words."""
    import paper_2608_20375_amd as G
    c = make(2, 40, [12, 80], 0, 4, 2, 64, "bfloat16", False, 1)
    ctx = G.Context(3, 8, 64, 1, 200)
    mask = np.zeros((2, 200, 4), np.int64)
    mask[:, :40, :1] = c["mask"]
    out, lse, _ = call(ctx, c, mask=torch.from_numpy(mask).cuda())
    check(c, out, lse)
    ctx.close()


def test_large_scores_and_another_scale():
    """Scores of several hundred: exp of nothing but differences from the maximum."""
    c = make(2, 20, [100, 64], 70, 4, 2, 128, "bfloat16", False, 1, qscale=40.0)
    ctx = context(c)
    out, lse, _ = call(ctx, c, scale=0.3)
    check(c, out, lse, scale=0.3)
    ctx.close()


def test_strided_tensors():
    """q, k, v as slices of one projection, keys and values of one interleaved cache, heads
    before rows, an output inside a wider one."""
    c = make(2, 33, [70, 130], 20, 8, 2, 64, "bfloat16", False, 1)
    B, S = c["q"].shape[:2]
    ctx = context(c)
    fused = torch.zeros(B, S, 12, 64, dtype=torch.bfloat16, device="cuda")
    fused[:, :, :8], fused[:, :, 8:10], fused[:, :, 10:] = (c[n].cuda() for n in ("q", "k", "v"))
    rows = c["cache"][0].shape[1]
    both = torch.zeros(B, 2, 2, rows, 64, dtype=torch.bfloat16, device="cuda")   # b, k/v, head, row
    for i in range(2):
        both[:, i] = c["cache"][i].cuda().transpose(1, 2)
    wide = torch.full((B, S, 8, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    out, lse, _ = call(ctx, c, q=fused[:, :, :8], k=fused[:, :, 8:10], v=fused[:, :, 10:],
                       cache=(both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)),
                       out=wide[..., :64])
    check(c, out, lse)
    assert (wide[..., 64:] == 7.0).all()
    ctx.close()


def test_strided_quantised_cache():
    import paper_2608_20375_amd as G
    c = make(2, 9, [70, 130], 20, 4, 2, 64, "bfloat16", True, 1)
    ctx = context(c)
    rows = c["cache"][0][0].shape[1]
    codes = torch.zeros(4, 2, rows, 3, 64, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(4, 2, rows, 3, dtype=torch.uint8, device="cuda")
    for i in range(2):
        codes[1 + i, :, :, 1:] = c["cache"][i][0].cuda()
        scales[1 + i, :, :, 1:] = c["cache"][i][1].cuda()
    every = G.QuantRows(codes, scales)
    view = lambda p: G.QuantRows(every[p].codes[:, :, 1:], every[p].scales[:, :, 1:])
    out, lse, _ = call(ctx, c, cache=(view(1), view(2)))
    check(c, out, lse)
    ctx.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3.0e38])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_hidden_slots_and_unused_rows_do_not_reach_a_row(bad, dtype):
    """Infinite, NaN and largest keys and values in slots that a row does not see, in rows
    past the block and past the cache."""
    c = make(2, 40, [30, 64], 0, 4, 2, 64, dtype, False, 1, depth=3, n=[40, 20])
    hurt = 5                                    # a node; slot 6
    kids = [i for i in range(c["n"][0] + 1) if c["seen"][0][i, hurt + 1]]
    clean, zc, _ = call(context(c), c)
    c["k"][0, hurt + 1] = bad
    c["v"][0, hurt + 1] = bad
    c["k"][1, 21:] = bad
    c["v"][1, 21:] = bad
    c["q"][1, 21:] = bad
    for x in c["cache"]:
        x[0, 30:] = bad
        x[1, 64:] = bad
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    rest = [i for i in range(41) if i not in kids]
    assert torch.equal(out[0, rest], clean[0, rest]) and torch.equal(lse[0, rest], zc[0, rest])
    assert torch.equal(out[1], clean[1]) and torch.equal(lse[1], zc[1])
    ctx.close()


def test_visible_infinite_values_arrive():
    """An infinite value of a slot that rows see makes those entries infinite, opposite ones
    NaN, and leaves the other entries as they are."""
    c = make(1, 8, [20], 0, 2, 1, 64, "bfloat16", False, 1, chain=True, n=[8])
    clean, _, _ = call(context(c), c)
    c["v"][0, 2, 0, 3] = float("inf")
    c["v"][0, 4, 0, 3] = float("-inf")
    c["v"][0, 5, 0, 9] = float("nan")
    ctx = context(c)
    out, _, _ = call(ctx, c)
    out, clean = out.cpu().float(), clean.cpu().float()
    assert torch.equal(out[0, :2], clean[0, :2])
    assert (out[0, 2:4, :, 3] == float("inf")).all() and torch.isnan(out[0, 4:, :, 3]).all()
    assert torch.isnan(out[0, 5:, :, 9]).all() and torch.isfinite(out[0, :5, :, 9]).all()
    other = [i for i in range(64) if i not in (3, 9)]
    assert torch.equal(out[..., other], clean[..., other])
    ctx.close()


@pytest.mark.parametrize("lens", [[0, 0], [40, 0]])
def test_rows_that_see_nothing(lens):
    """Without a root a mask row may be empty: with no prefix the row gets zeros and -inf."""
    c = make(2, 10, lens, 0, 2, 1, 64, "bfloat16", False, 0, n=[10, 10])
    for b in range(2):
        c["mask"][b, 4] = 0
        c["seen"][b][4] = False
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    assert (out[1, 4] == 0).all() and (lse[1, 4] == -float("inf")).all()
    ctx.close()


def test_mask_bits_past_the_tree_are_ignored():
    c = make(1, 70, [5], 0, 2, 1, 64, "bfloat16", False, 1, n=[30])
    c["mask"][0, :, 0] |= np.int64(-1) << np.int64(30)
    c["mask"][0, :, 1] = -1
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    ctx.close()


def test_no_nodes_and_no_root_leaves_everything():
    c = make(2, 6, [9, 9], 0, 2, 1, 64, "bfloat16", False, 0, n=[0, 6])
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    ctx.close()


def test_sizes_outside_their_range_are_clamped_and_reported():
    c = make(2, 6, [9, 12], 0, 2, 1, 64, "bfloat16", False, 1, n=[6, 6], extra=0)
    ctx = context(c)
    good, zg, _ = call(ctx, c)
    assert ctx.device_status() == 0
    n = torch.tensor([7, 6], dtype=torch.int32, device="cuda")
    out, lse, _ = call(ctx, c, n_nodes=n)
    assert torch.equal(out, good) and torch.equal(lse, zg)
    assert ctx.device_status() == 5 and ctx.device_status() == 0
    lens = torch.tensor([9, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out, lse, _ = call(ctx, c, cache_len=lens)
    assert torch.equal(out, good) and torch.equal(lse, zg)
    assert ctx.device_status() == 5
    out, lse, _ = call(ctx, c, n_nodes=torch.tensor([-3, 6], dtype=torch.int32, device="cuda"))
    assert torch.equal(out[1], good[1]) and (out[0, 1:] == 7.0).all()
    assert ctx.device_status() == 5
    ctx.close()


def test_caches_past_32_bit_offsets():
    """The second sequence's rows start more than 2^31 elements after the first's."""
    c = make(2, 3, [70, 90], 0, 2, 1, 64, "bfloat16", False, 1)
    rows = c["cache"][0].shape[1]
    far = 2 ** 31 + 1024
    caches = []
    for x in c["cache"]:
        buf = torch.empty(far + rows * 64, dtype=torch.bfloat16, device="cuda")
        view = buf.as_strided((2, rows, 1, 64), (far, 64, 64, 1))
        view.copy_(x)
        caches.append(view)
    ctx = context(c)
    out, lse, _ = call(ctx, c, cache=tuple(caches))
    check(c, out, lse)
    ctx.close()


def test_the_same_bits_every_time_and_without_lse():
    c = make(3, 40, [900, 64, 333], 129, 8, 2, 128, "bfloat16", True, 1)
    ctx = context(c)
    first, z, _ = call(ctx, c)
    for _ in range(5):
        out, lse, _ = call(ctx, c)
        assert torch.equal(out, first) and torch.equal(lse, z)
    out, _, _ = call(ctx, c, lse=False)
    assert torch.equal(out, first)
    ctx.close()


def test_another_stream_and_two_captured_graphs():
    """A call on a side stream; two graphs with workspaces of their own replayed with eager
    calls between them and new inputs in place."""
    c = make(4, 20, [500, 64, 333, 0], 200, 8, 2, 64, "bfloat16", False, 1)
    ctx = context(c)
    want, z, a = call(ctx, c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = torch.full_like(want, 7.0)
        ctx.tree_attention(**{**a, "out": out})
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    args = {k: v for k, v in a.items()}
    need = ctx.tree_attention_workspace(**{k: v for k, v in a.items()})
    assert need > 0
    graphs = []
    for i in range(2):
        o = torch.full_like(want, 7.0)
        w = torch.empty(need, dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.tree_attention(**{**args, "out": o, "workspace": w})
        graphs.append((g, o, w))
    for turn in range(3):
        a["q"].copy_(torch.randn_like(a["q"], dtype=torch.float32))
        eager = torch.full_like(want, 7.0)
        ctx.tree_attention(**{**args, "out": eager})
        for g, o, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, o, _ in graphs:
            assert torch.equal(o, eager), turn
    ctx.close()


def test_refusals_with_real_tensors():
    import paper_2608_20375_amd as G
    c = make(2, 6, [9, 9], 4, 4, 2, 64, "bfloat16", False, 1)
    ctx = context(c)
    _, _, a = call(ctx, c)
    flat = torch.zeros(2 * 7 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    bad = [dict(q=flat[1:1 + 2 * 7 * 4 * 64].view(2, 7, 4, 64)),        # misaligned
           dict(scale=0.0), dict(scale=float("nan")), dict(scale=-1.0),
           dict(q=torch.zeros(2, 7, 4, 68, dtype=torch.bfloat16, device="cuda")[..., :64])]
    for kw in bad:
        with pytest.raises((G.GraftError, ValueError)):
            ctx.tree_attention(**{**a, **kw})
    small = torch.empty(8, dtype=torch.uint8, device="cuda")
    if ctx.tree_attention_workspace(**a):
        with pytest.raises(ValueError):
            ctx.tree_attention(**{**a, "workspace": small})
    with pytest.raises(TypeError):
        ctx.tree_attention(**{**a, "cache_len": a["cache_len"].cpu()})
    with pytest.raises(TypeError):
        ctx.tree_attention(**{**a, "n_nodes": a["n_nodes"].long()})
    quant = G.QuantRows.empty(2, 12, 2, 64)
    with pytest.raises(ValueError):                                     # one type for both
        ctx.tree_attention(**{**a, "cache": (quant, quant)})
    half = {n: a[n].half() for n in ("q", "k", "v", "out")}
    with pytest.raises(G.GraftError):                                   # e4m3 with fp16
        ctx.tree_attention(**{**a, **half, "cache": (quant, quant), "shared": None})
    ctx.close()
