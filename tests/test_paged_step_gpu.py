"""The paged operators together as a serving loop runs them: a tree is built, its block's rows are
rotated into the pages, the block attends over them, the walk draws tokens, and the accepted path's
rows move up.  Every stage is checked against 64 bits, or byte for byte, on what the stage before it
gave."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paged_ref as R  # noqa: E402
import paper_2608_20375_amd as G  # noqa: E402

pytestmark = pytest.mark.gpu

BF, Q8 = torch.bfloat16, torch.float8_e4m3fn


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def numbers(pool):
    return R.values(pool.codes.cpu(), pool.scales.cpu()) if isinstance(pool, G.QuantRows) else pool.cpu().double()


def bits(pool):
    return [x.cpu().clone() for x in ((pool.codes, pool.scales) if isinstance(pool, G.QuantRows) else (pool.view(torch.int16),))]


@pytest.mark.parametrize("kind", [BF, Q8])
@pytest.mark.parametrize("window", [None, 30])
def test_rounds_of_a_serving_loop(kind, window):
    B, L, V, K, N, Hq, H, D, page = 3, 5, 300, 6, 40, 4, 2, 32, 16
    E, width = 24, 12
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    ctx = G.Context(B, L, V, K, N)
    ctx.set_scorer(rnd(V, 16), 0.1 * rnd(16, 8), 0.1 * rnd(16, 8))
    ctx.set_history(torch.zeros(B, 4, dtype=torch.int32, device="cuda"))
    emb, head = rnd(V, E), 1.5 * rnd(Hq * D, V)
    wq, wk, wv = (rnd(E, h * D).mul_(0.4) for h in (Hq, H, H))
    row = lambda tok, w, h: (emb[tok] @ w).to(BF).view(*tok.shape, h, D)
    freq = 100.0 ** -(np.arange(D // 2) / (D // 2))
    rng = np.random.default_rng(1)
    table = rng.permutation(B * width).astype(np.int32).reshape(B, width)
    t, f = dev(table), dev(freq)
    pool = G.paged_cache(B * width, page, H, D, kind, planes=2)
    for x in ((pool.codes, pool.scales) if kind == Q8 else (pool.view(torch.int16),)):
        x.fill_(-1 if x.dtype == torch.int16 else 255)         # NaN everywhere
    length = torch.tensor([20, 0, 33], dtype=torch.int32, device="cuda")
    prompt = torch.randint(0, V, (B, 33), device="cuda", generator=gen)
    ctx.paged_write((pool[0], pool[1]), t, row(prompt, wk, H), row(prompt, wv, H), length, freq=f)
    root = torch.randint(0, V, (B,), device="cuda", generator=gen, dtype=torch.int32)
    moved = 0
    for r in range(5):
        out = ctx.build_tree(rnd(B, L, V).mul_(2).to(BF), root, length,
                             fixed_budget=torch.full((B,), 25 + r, dtype=torch.int32, device="cuda"))
        block = torch.cat([root[:, None], out.tokens], 1).long().clamp_min(0)
        q, k, v = row(block, wq, Hq), row(block, wk, H), row(block, wv, H)
        # position ids: the root's, then one more a level
        pos = torch.cat([length[:, None], out.pos_ids], 1).to(torch.int32).contiguous()
        rq = ctx.paged_write((pool[0], pool[1]), t, k, v, out.n_nodes + 1, length, q=q, freq=f, positions=pos)
        att = ctx.paged_attention(rq, (pool[0], pool[1]), t, length, out.n_nodes, out.mask, with_root=True, window=window,
                                  sinks=2 if window else 0)
        n, lens, own = out.n_nodes.cpu().numpy(), length.cpu().numpy(), numbers(pool)
        mask, p = out.mask.cpu().numpy().view(np.uint64), pos.cpu().numpy()
        for b in range(B):
            m = int(n[b]) + 1
            seen = np.zeros((m, m), bool)
            seen[:, 0] = True
            for j in range(m - 1):
                seen[1:, 1 + j] = (mask[b, :m - 1, j >> 6] >> np.uint64(j & 63)) & np.uint64(1)
            # a node's depth is its place behind the cache
            assert (seen.sum(1) - 1 + lens[b] == p[b, :m]).all()
            y, tol = R.rotate(q[b, :m].cpu().double(), p[None, b, :m], freq)
            assert ((rq[b, :m].cpu().double() - y).abs() <= tol + 2.0 ** -8 * 1.001 * (y.abs() + tol)).all()
            kv = [R.rows_of(own[i], table[b], page, int(lens[b]) + m) for i in range(2)]
            y, tol = R.rotate(k[b, :m].cpu().double(), p[None, b, :m], freq)
            err = (kv[0][lens[b]:] - y).abs()
            step = 2.0 ** -4 * y.abs() + 2.0 ** -17 * y.abs().amax(-1, keepdim=True) if kind == Q8 else 2.0 ** -8 * y.abs()
            assert (err <= 1.001 * step + tol).all()
            see = R.visible(int(lens[b]), m, window or 0, 2, seen)
            ref, _, tol, _ = R.attention(rq[b, :m].cpu().double(), *kv, see, D ** -0.5, 2.0 ** -7)
            assert ((att[b, :m].cpu().double() - ref).abs() <= tol).all(), (r, b)
        logits = att.float().view(B, N + 1, -1) @ head
        tok, par = out.tokens.cpu().numpy(), out.parents.cpu().numpy()
        for b in range(B):
            for i in range(int(n[b])):
                logits[b, par[b, i] + 1, tok[b, i]] += 12.0
        u = torch.rand(B, L + 1, dtype=torch.float64, device="cuda", generator=gen)
        acc, nodes, bonus, _ = ctx.accept_sampled(out.n_nodes, out.tokens, out.parents, logits[:, 0], logits[:, 1:], u)
        want = bits(pool)
        a, path = acc.cpu().numpy(), nodes.cpu().numpy()
        for b in range(B):
            first = int(lens[b]) + 1
            at = lambda x: (int(table[b, x // page]), x % page)
            for x in want:
                old = x.clone()
                for i in range(int(a[b])):
                    (p0, r0), (p1, r1) = at(first + int(path[b, i])), at(first + i)
                    x[:, p1, r1] = old[:, p0, r0]
            moved += int((path[b, :a[b]] != np.arange(a[b])).sum())
        ctx.paged_commit(pool, t, length, acc, nodes, with_root=True)
        assert all(torch.equal(x, y) for x, y in zip(bits(pool), want))
        length = length + 1 + acc
        root = bonus
    assert moved > 0 and ctx.device_status() == 0
    ctx.close()


def test_a_step_in_a_graph():
    """Write, attention and commit captured together and replayed between eager work: each replay gives
    the bits of the same calls made one by one."""
    B, S, Hq, H, D, page, width = 2, 9, 8, 2, 64, 16, 20
    rng = np.random.default_rng(2)
    rnd = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(BF).cuda()
    table = dev(rng.permutation(B * width).astype(np.int32).reshape(B, width))
    seen = [R.tree_block(rng, S - 1)[1] for _ in range(B)]
    mask = dev(np.stack([R.pack_mask(x, S - 1) for x in seen]))
    ctx = G.Context(B, 4, 64, 1, S - 1)
    pool = G.paged_cache(B * width, page, H, D, BF, planes=2)
    pool.copy_(rnd(*pool.shape))
    q, k, v = rnd(B, S, Hq, D), rnd(B, S, H, D), rnd(B, S, H, D)
    freq = dev(10.0 ** -np.linspace(0, 3, D // 2))
    n = torch.full((B,), S, dtype=torch.int32, device="cuda")
    lens = torch.tensor([100, 37], dtype=torch.int32, device="cuda")
    acc, nodes = torch.tensor([2, 3], dtype=torch.int32, device="cuda"), dev(np.array([[1, 4, -1, -1], [2, 5, 7, -1]], np.int32))
    rq, out, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(B, S, Hq, device="cuda")
    kv = (pool[0], pool[1])
    need = ctx.paged_attention_workspace(q, kv, table, lens, n - 1, mask, with_root=True)
    w = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
    nn = n - 1

    def step():
        ctx.paged_write(kv, table, k, v, n, lens, q=q, q_out=rq, freq=freq)
        ctx.paged_attention(rq, kv, table, lens, nn, mask, with_root=True, out=out, lse=lse, workspace=w)
        ctx.paged_commit(pool, table, lens, acc, nodes, with_root=True)

    start = pool.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for lengths in ([100, 37], [0, 200], [299, 1]):
        lens.copy_(dev(np.array(lengths, np.int32)))
        k.copy_(rnd(*k.shape))
        pool.copy_(start)
        step()
        torch.cuda.synchronize()
        eager = [x.clone() for x in (pool, rq, out, lse)]
        pool.copy_(start)
        for x in (rq, out, lse):
            x.fill_(7.0)
        w.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((pool, rq, out, lse), eager)), lengths
    assert ctx.device_status() == 0
    ctx.close()


def test_steps_in_flight():
    """Two contexts' steps on two streams at once, into memory that nothing has written."""
    B, S, Hq, H, D, page = 3, 40, 8, 2, 64, 32
    rng = np.random.default_rng(4)
    rnd = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(BF).cuda()
    runs = []
    for i in range(2):
        lens = np.array([500, 60, 1200], np.int32) - 30 * i
        t, pages = R.table(rng, page, lens + S)
        c = dict(ctx=G.Context(B, 4, 64, 1, 64), lens=lens, t=t, kv=(G.paged_cache(pages, page, H, D), G.paged_cache(pages, page, H, D)),
                 q=rnd(B, S, Hq, D), k=rnd(B, S, H, D), v=rnd(B, S, H, D), stream=torch.cuda.Stream())
        for x in c["kv"]:
            x.copy_(rnd(*x.shape))
        c.update(td=dev(t), ld=dev(lens), out=torch.empty(B, S, Hq, D, dtype=BF, device="cuda"))
        need = c["ctx"].paged_attention_workspace(c["q"], c["kv"], c["td"], c["ld"])
        c["w"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        runs.append(c)
    torch.cuda.synchronize()
    for _ in range(3):
        for c in runs:
            with torch.cuda.stream(c["stream"]):
                c["ctx"].paged_write(c["kv"], c["td"], c["k"], c["v"], start=c["ld"])
                c["ctx"].paged_attention(c["q"], c["kv"], c["td"], c["ld"], out=c["out"], workspace=c["w"])
    torch.cuda.synchronize()
    for c in runs:
        for b in range(B):
            n = int(c["lens"][b])
            k, v = (R.rows_of(x.cpu().double(), c["t"][b], page, n + S) for x in c["kv"])
            assert torch.equal(k[n:], c["k"][b].cpu().double()) and torch.equal(v[n:], c["v"][b].cpu().double())
            ref, _, tol, _ = R.attention(c["q"][b].cpu().double(), k, v, R.visible(n, S), D ** -0.5, 2.0 ** -7)
            assert ((c["out"][b].cpu().double() - ref).abs() <= tol).all()
        assert c["ctx"].device_status() == 0
        c["ctx"].close()
