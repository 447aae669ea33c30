"""The verifier's side of several rounds as a serving loop runs it: a tree is built, the
block attends over a quantised cache, the walk draws tokens from the logits, and the root
and the accepted path are appended.  Every stage is checked against 64 bits on what the
stage before it gave."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import verifier_ref as R  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quant", [True, False])
def test_rounds_of_a_serving_loop(quant):
    import paper_2608_20375_amd as G
    B, L, V, K, N, Hq, H, D, P, rows = 3, 5, 300, 6, 40, 4, 2, 32, 9, 80
    E = 24
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    ctx = G.Context(B, L, V, K, N)
    ctx.set_scorer(rnd(V, 16), 0.1 * rnd(16, 8), 0.1 * rnd(16, 8))
    ctx.set_history(torch.zeros(B, 4, dtype=torch.int32, device="cuda"))
    emb, head = rnd(V, E), 1.5 * rnd(Hq * D, V)
    wq, wk, wv = (rnd(E, h * D).mul_(0.4) for h in (Hq, H, H))
    kv = lambda tok: [(emb[tok] @ w).to(torch.bfloat16).view(*tok.shape, H, D) for w in (wk, wv)]

    prompt = torch.randint(0, V, (B, 20), device="cuda", generator=gen)
    shared_tok = torch.randint(0, V, (1, P), device="cuda", generator=gen)
    if quant:
        cache = G.QuantRows.empty(2, B, rows, H, D)
        shared = G.QuantRows.empty(2, 1, P, H, D)
    else:
        cache = torch.zeros(2, B, rows, H, D, dtype=torch.bfloat16, device="cuda")
        shared = torch.zeros(2, 1, P, H, D, dtype=torch.bfloat16, device="cuda")
    length = torch.tensor([20, 0, 13], dtype=torch.int32, device="cuda")
    ctx.cache_write(cache, torch.stack(kv(prompt)), length)
    ctx.cache_write(shared, torch.stack(kv(shared_tok)),
                    torch.tensor([P], dtype=torch.int32, device="cuda"))
    root = torch.randint(0, V, (B,), device="cuda", generator=gen, dtype=torch.int32)
    texts = [prompt[b, :int(length[b])].tolist() for b in range(B)]
    accepted = 0
    for r in range(4):
        out = ctx.build_tree(rnd(B, L, V).mul_(2).to(torch.bfloat16), root, length,
                             fixed_budget=torch.full((B,), 25 + r, dtype=torch.int32, device="cuda"))
        block = torch.cat([root[:, None], out.tokens], 1).long().clamp_min(0)
        q = (emb[block] @ wq).to(torch.bfloat16).view(B, N + 1, Hq, D)
        k, v = kv(block)
        att = ctx.tree_attention(q, k, v, out.n_nodes, out.mask, cache=(cache[0], cache[1]),
                                 cache_len=length, shared=(shared[0, 0], shared[1, 0]), with_root=True)
        n = out.n_nodes.cpu().numpy()
        number = ((lambda t: R.values(t.codes.cpu(), t.scales.cpu())) if quant
                  else (lambda t: t.cpu().double()))
        own, sh = number(cache), number(shared)
        mask = out.mask.cpu().numpy().view(np.uint64)
        for b in range(B):
            m = int(n[b]) + 1
            seen = np.zeros((m, m), bool)
            seen[:, 0] = True
            for j in range(m - 1):
                seen[1:, 1 + j] = (mask[b, :m - 1, j >> 6] >> np.uint64(j & 63)) & np.uint64(1)
            c = int(length[b])
            ref, _, tol, _ = R.attention(
                q[b, :m].cpu().double(), k[b, :m].cpu().double(), v[b, :m].cpu().double(), seen,
                torch.cat([sh[0, 0], own[0, b, :c]]), torch.cat([sh[1, 0], own[1, b, :c]]),
                D ** -0.5, torch.finfo(torch.bfloat16).eps)
            assert ((att[b, :m].cpu().double() - ref).abs() <= tol).all(), (r, b)
        logits = att.float().view(B, N + 1, -1) @ head
        # the drafted children get a good share, so that paths are accepted
        tok, par = out.tokens.cpu().numpy(), out.parents.cpu().numpy()
        for b in range(B):
            for i in range(int(n[b])):
                logits[b, par[b, i] + 1, tok[b, i]] += 12.0
        u = torch.rand(B, L + 1, dtype=torch.float64, device="cuda", generator=gen)
        acc, nodes, bonus, logp = ctx.accept_sampled(out.n_nodes, out.tokens, out.parents, logits[:, 0],
                                                     logits[:, 1:], u, update_history=True)
        z = logits.double().cpu().numpy()
        for b in range(B):
            a, path, x, lp = R.walk(z[b], par[b], tok[b], int(n[b]), L, u[b].cpu().numpy(), 1.0)
            assert (int(acc[b]), int(bonus[b])) == (a, x) and nodes[b].tolist() == path.tolist(), (r, b)
            texts[b] += [int(root[b])] + [int(tok[b, i]) for i in path[:a]]
            accepted += a
        ctx.cache_write(cache, torch.stack([k, v]), acc, rows=nodes, start=length, with_root=True)
        length = length + acc + 1
        root = bonus
        # the cache is the text's keys and values
        for b in range(B):
            t = torch.tensor(texts[b], device="cuda")
            assert len(texts[b]) == int(length[b])
            want = torch.stack(kv(t))
            got = number(cache)[:, b, :len(t)]
            assert torch.equal(got, R.values(*R.quantise(want.cpu())) if quant else want.cpu().double())
    assert accepted > 0 and ctx.device_status() == 0
    ring, pos = ctx.get_history(B)
    assert pos.tolist() == [0] * B
    ctx.close()
