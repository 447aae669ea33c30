"""The verifier's side of a decoding round, as measurable cases.

Three groups of operators, each with a plain form in elementary torch
operations and the calls that a user makes of paper_2608_20375_amd:

attend   Context.tree_attention: attention of a draft block (the last committed
         token and the nodes of its tree, under the ancestor mask; or that token
         alone) over a prefix that the whole batch shares, each sequence's own
         cache (plain or e4m3 with a power-of-two scale a row and head) and the
         block itself.
sample   Context.accept_sampled: the walk down a draft tree that follows tokens
         drawn from the target model's probabilities with given random numbers.
cache    Context.cache_write and Context.cache_read: key/value rows quantised into a
         cache as they are appended, and rows of it read back ("write" cases do
         both, "read" cases take a long span back as bf16).

Inputs are drawn from the seed alone.  Lengths and tree sizes are a fixed
spread of the case's range in an order that the seed draws, so a case's work
does not depend on the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # One user's next token without a draft: one query row over a short plain
        # cache.  The smallest call, where launches and latency count.
        dict(name="attend_b1_single", kind="attend", batch=1, nodes=0, depth=1, q_heads=32,
             kv_heads=8, dim=128, dtype="bfloat16", cache="same", length=700, shared=0),
        # A serving batch at one token a sequence, a system prompt shared by all of
        # it, ragged quantised caches: bound by the cache's bytes.
        dict(name="attend_b64_shared_e4m3", kind="attend", batch=64, nodes=0, depth=1, q_heads=32,
             kv_heads=8, dim=128, dtype="bfloat16", cache="e4m3", length=8192, shared=4096),
        # Odd sizes: five sequences, a tree that fills no tile, five query heads a
        # key head, 80 dimensions, half precision.
        dict(name="attend_b5_odd_fp16", kind="attend", batch=5, nodes=70, depth=12, q_heads=20,
             kv_heads=4, dim=80, dtype="float16", cache="same", length=1531, shared=133),
        # The 16-sequence round's trees (up to 256 nodes) over plain caches.
        dict(name="attend_b16_n256", kind="attend", batch=16, nodes=256, depth=16, q_heads=32,
             kv_heads=8, dim=128, dtype="bfloat16", cache="same", length=4096, shared=0),
        # The batch-64 round's trees (up to 512 nodes) over quantised caches: the
        # largest attention, bound by matrix products.
        dict(name="attend_b64_n512_e4m3", kind="attend", batch=64, nodes=512, depth=16, q_heads=32,
             kv_heads=8, dim=128, dtype="bfloat16", cache="e4m3", length=4096, shared=1024),
        # One sequence, small vocabulary, small tree: latency.
        dict(name="sample_b1_v32k", kind="sample", batch=1, nodes=32, depth=8, vocab=32000,
             dtype="bfloat16", mixed=False),
        # Odd sizes: rows that start at any alignment, fp32 logits, temperatures of
        # 0 among others.
        dict(name="sample_b5_odd_fp32", kind="sample", batch=5, nodes=100, depth=12, vocab=70001,
             dtype="float32", mixed=True),
        # The batch-64 round's vocabulary and depth.
        dict(name="sample_b64_v128k", kind="sample", batch=64, nodes=128, depth=16, vocab=128256,
             dtype="bfloat16", mixed=True),
        # The largest batch and depth.
        dict(name="sample_b128_v152k", kind="sample", batch=128, nodes=64, depth=32, vocab=151936,
             dtype="bfloat16", mixed=False),
        # One sequence's accepted path appended to a 16-layer cache.
        dict(name="write_b1_append", kind="write", batch=1, planes=32, heads=4, dim=128, slots=33,
             most=9, paths=True),
        # The batch-64 round's accepted paths, 36 layers of keys and values.
        dict(name="write_b64_append", kind="write", batch=64, planes=72, heads=8, dim=128,
             slots=129, most=17, paths=True),
        # A layer's cache of the batch read back for a path that wants bf16.
        dict(name="read_b64_span", kind="read", batch=64, planes=2, heads=8, dim=128, length=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: attention in five of ten draws, then the sampled walk, writes and reads."""
    u = rng.random()
    if u < 0.5:
        kv = rng.choice((1, 2, 4, 8, 8))
        q = kv * rng.choice((1, 2, 4, 4, 5, 7, 8))
        dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 128))
        dtype = rng.choice(("bfloat16", "bfloat16", "float16"))
        cache = rng.choice(("same", "e4m3")) if dtype == "bfloat16" else "same"
        nodes = rng.choice((0, 0, _log_int(rng, 1, 512), _log_int(rng, 16, 512)))
        length, shared = _log_int(rng, 16, 16384), rng.choice((0, 0, _log_int(rng, 16, 8192)))
        most = int(64 * 272 * 32 * 128 * 3400 / ((nodes * 0.53 + 1) * q * dim * (shared + length / 2 + nodes)))
        cells = int(2.5e8 / (kv * dim * (length + nodes + 64)))       # a cache of at most 1 GB
        rows = int(1.4e8 / (q * dim * (nodes + 1)))
        batch = max(1, min(_log_int(rng, 1, 64), most, cells, rows))
        return dict(kind="attend", batch=batch, nodes=nodes, depth=rng.choice((8, 12, 16, 32)),
                    q_heads=q, kv_heads=kv, dim=dim, dtype=dtype, cache=cache, length=length,
                    shared=shared)
    if u < 0.75:
        dtype = rng.choice(("bfloat16", "bfloat16", "float16", "float32"))
        V = rng.choice((_log_int(rng, 8000, 151936), 32000, 128256, 151936))
        nodes = _log_int(rng, 8, 256)
        batch = max(1, min(_log_int(rng, 1, 128),
                           int(2.4e9 / ((nodes + 1) * V * (4 if dtype == "float32" else 2)))))
        return dict(kind="sample", batch=batch, nodes=nodes, depth=rng.choice((4, 8, 12, 16, 32)),
                    vocab=V, dtype=dtype, mixed=rng.random() < 0.5)
    if u < 0.9:
        heads, dim = rng.choice((1, 2, 4, 5, 8)), rng.choice((32, 64, 80, 128, 128))
        if rng.random() < 0.6:
            return dict(kind="write", batch=_log_int(rng, 1, 64), planes=rng.randint(2, 72),
                        heads=heads, dim=dim, slots=rng.randint(20, 129),
                        most=rng.choice((5, 9, 17)), paths=True)
        most = _log_int(rng, 16, 4096)                                # a prompt's rows
        return dict(kind="write", batch=_log_int(rng, 1, 16), planes=2, heads=heads, dim=dim,
                    slots=most, most=most, paths=False)
    return dict(kind="read", batch=_log_int(rng, 1, 64), planes=2, heads=rng.choice((1, 4, 5, 8)),
                dim=rng.choice((32, 64, 80, 128)), length=_log_int(rng, 16, 4096))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

CHILD_MASS = 0.8        # target probability of a drafted node's children together, at temperature 1
SPINE = 6.0             # weight of a child that has children itself, against 0..1


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 9973 + 41)


def _spread(count, lo, hi, rng=None):
    """count sizes spread evenly over lo..hi (the largest among them), in an order drawn by rng."""
    v = np.array([hi - (hi - lo) * i // max(1, count) for i in range(count)], np.int32)
    return v if rng is None else rng.permutation(v).astype(np.int32)


def _node_counts(case, rng=None):
    n = case["nodes"]
    return _spread(case["batch"], min(n, max(1, n // 16)), n, rng)


def _tree(rng, n, depth, vocab):
    """parents, tokens and depths of a tree of n nodes in canonical order (depth, then the
    parents' order, then token); every depth's first node has children."""
    depth = min(depth, n)
    if n == 0:
        return (np.zeros(0, np.int32),) * 3
    share = np.exp(-np.arange(depth) / 6.0) * np.minimum(np.arange(depth) + 1, 4)
    count = 1 + np.floor((n - depth) * share / share.sum()).astype(int)
    count[min(1, depth - 1)] += n - count.sum()
    toks = np.unique(rng.integers(0, vocab, 2 * n + 64))
    toks = rng.permutation(toks)[:n].astype(np.int32)
    parents, tokens, depths = [], [], []
    first, before = -1, 1
    at = 0
    for d in range(depth):
        c = int(count[d])
        p = np.sort(rng.integers(0, before, c)) + first if d else np.full(c, -1)
        if d:
            p[0] = first
            p.sort()
        t = toks[at:at + c]
        order = np.lexsort((t, p))
        parents.append(p[order])
        tokens.append(t[order])
        depths.append(np.full(c, d + 1))
        first, before = at, c
        at += c
    return tuple(np.concatenate(x).astype(np.int32) for x in (parents, tokens, depths))


def _trees(case, rng, counts, vocab):
    """Padded arrays of the batch's trees, and the ancestor bitsets."""
    B, N = case["batch"], max(1, case["nodes"])
    parents = np.full((B, N), -1, np.int32)
    tokens = np.full((B, N), -1, np.int32)
    mask = np.zeros((B, N, (N + 63) // 64), np.uint64)
    for b in range(B):
        n = int(counts[b])
        p, t, d = _tree(rng, n, case["depth"], vocab)
        parents[b, :n], tokens[b, :n] = p, t
        i = np.arange(n)
        mask[b, i, i >> 6] = np.uint64(1) << (i & 63).astype(np.uint64)
        for depth in range(2, int(d.max(initial=0)) + 1):
            level = np.flatnonzero(d == depth)
            mask[b, level] |= mask[b, p[level]]
    return parents, tokens, mask


def _pow2(e):
    """2^e in fp32, exactly (a library power need not be): integers e in -126..127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _pow2_64(e):
    """2^e in fp64, exactly: integers e in -1022..1023."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _quantise(x):
    """e4m3 codes of the last axis' values over 2^e, and e + 127: e is the smallest integer from
    -118 on with max|x| <= 448 * 2^e."""
    x = x.float()
    part, power = torch.frexp(x.abs().amax(-1))
    e = torch.where(part <= 0.875, power - 9, power - 8)
    e = torch.where(part == 0, -118, e).clamp_min(-118).to(torch.int32)
    codes = (x * _pow2(-e)[..., None]).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The numbers that codes and scales stand for, in fp32."""
    return codes.float() * _pow2(scales.to(torch.int32) - 127)[..., None]


def _attend_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    B, S, Hq, H, D = (case["batch"], case["nodes"] + 1, case["q_heads"], case["kv_heads"],
                      case["dim"])
    dt = getattr(torch, case["dtype"])
    lens = _spread(B, max(1, case["length"] // 16), case["length"], rng)
    counts = _node_counts(case, rng)
    parents, _, mask = _trees(case, rng, counts, 50000)
    rows = (case["length"] + S + 63) // 64 * 64

    def normal(*shape):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g)

    s = dict(q=normal(B, S, Hq, D).mul_(2.0), k=normal(B, S, H, D), v=normal(B, S, H, D))
    for name, lead in (("cache", (B, rows)), ("shared", (case["shared"],))):
        if lead[-1] == 0 or (name == "shared" and not case["shared"]):
            s[name] = None
            continue
        pair = (normal(*lead, H, D), normal(*lead, H, D))
        s[name] = tuple(_quantise(x) for x in pair) if case["cache"] == "e4m3" else pair
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    s.update(n_nodes=dev(counts), mask=dev(mask.view(np.int64)), cache_len=dev(lens), lens=lens,
             counts=counts, parents=parents)
    return s


def _sample_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    B, N, V, L = case["batch"], case["nodes"], case["vocab"], case["depth"]
    counts = _node_counts(case, rng)
    parents, tokens, _ = _trees(case, rng, counts, V)
    logits = torch.empty(B, N + 1, V, dtype=getattr(torch, case["dtype"]), device="cuda")
    logits.normal_(generator=g)
    # children of a node share CHILD_MASS of its row's probability
    bb, ii = np.nonzero(np.arange(N)[None, :] < counts[:, None])
    row = parents[bb, ii] + 1
    has = np.zeros((B, N + 1), bool)
    has[bb, row] = True
    w = rng.uniform(0.05, 1.0, len(bb)) + SPINE * has[bb, ii + 1]
    total = np.zeros((B, N + 1))
    np.add.at(total, (bb, row), w)
    z = np.log(w / total[bb, row] * CHILD_MASS / (1 - CHILD_MASS)) + math.log(V) + 0.5
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    logits[dev(bb), dev(row).long(), dev(tokens[bb, ii]).long()] = dev(z).to(logits.dtype)
    temper = np.ones(B, np.float32)
    if case["mixed"]:
        temper = rng.choice(np.array([0.0, 0.6, 0.8, 1.0, 1.2], np.float32), B)
    u = torch.rand(B, L + 1, dtype=torch.float64, device="cuda", generator=g)
    return dict(logits=logits, n_nodes=dev(counts), tokens=dev(tokens), parents=dev(parents),
                temperature=dev(temper), uniform=u, counts=counts)


def _write_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    P, B, H, D, M = case["planes"], case["batch"], case["heads"], case["dim"], case["most"]
    src = torch.empty(P, B, case["slots"], H, D, dtype=torch.bfloat16, device="cuda")
    src.normal_(generator=g)
    # a few dimensions of each head are larger, as keys are
    src.mul_(torch.exp(torch.randn(H, D, device="cuda", generator=g)).to(torch.bfloat16))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    s = dict(src=src)
    if case["paths"]:       # the root and an accepted path of 0 .. most - 1 nodes
        n = _spread(B, 0, M - 1, rng) * 4 // 10
        nodes = np.full((B, M - 1), -1, np.int32)
        for b in range(B):
            nodes[b, :n[b]] = np.sort(rng.choice(case["slots"] - 1, n[b], replace=False))
        s.update(n=dev(n), nodes=dev(nodes))
    else:
        n = _spread(B, max(1, M // 4), M, rng)
        s.update(n=dev(n), nodes=None)
    start = rng.integers(0, 64, B).astype(np.int32)
    rows = M + 64
    s.update(start=dev(start), start_h=start, n_h=n,
             codes=torch.zeros(P, B, rows, H, D, dtype=torch.float8_e4m3fn, device="cuda"),
             scales=torch.zeros(P, B, rows, H, dtype=torch.uint8, device="cuda"),
             out=torch.zeros(P, B, M, H, D, dtype=torch.bfloat16, device="cuda"))
    return s


def _read_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    P, B, H, D, M = case["planes"], case["batch"], case["heads"], case["dim"], case["length"]
    x = torch.empty(P, B, M + 64, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    codes, scales = [], []
    for p in range(P):
        c, s = _quantise(x[p])
        codes.append(c)
        scales.append(s)
    n = _spread(B, max(1, M // 8), M, rng)
    start = rng.integers(0, 64, B).astype(np.int32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return dict(codes=torch.stack(codes), scales=torch.stack(scales), n=dev(n), start=dev(start),
                n_h=n, start_h=start,
                out=torch.zeros(P, B, M, H, D, dtype=torch.bfloat16, device="cuda"))


_INPUTS = dict(attend=_attend_inputs, sample=_sample_inputs, write=_write_inputs,
               read=_read_inputs)


def prepare(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    s["case"] = case
    B = case["batch"]
    if case["kind"] == "attend":
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(s["q"].shape[:3], dtype=torch.float32, device="cuda")
    if case["kind"] == "sample":
        i32 = dict(dtype=torch.int32, device="cuda")
        s.update(acc_len=torch.empty(B, **i32), acc_nodes=torch.empty(B, case["depth"], **i32),
                 bonus=torch.empty(B, **i32),
                 logp=torch.empty(B, case["depth"] + 1, dtype=torch.float32, device="cuda"))
    if own:
        s["ctx"] = _context(case)
        _wrap(s)
    return s


def _context(case):
    import paper_2608_20375_amd as G
    kind = case["kind"]
    nodes = max(1, case["nodes"]) if kind in ("attend", "sample") else max(1, case.get("slots", 1) - 1)
    depth = case.get("depth", max(1, case.get("most", 2) - 1) if case.get("paths") else 1)
    return G.Context(case["batch"], depth, case.get("vocab", 64), 1, min(nodes, 1024))


def _wrap(s):
    """The caches as the framework takes them: codes and scales in one object."""
    import paper_2608_20375_amd as G
    kind = s["case"]["kind"]
    if kind in ("write", "read"):
        s["cache"] = G.QuantRows(s["codes"], s["scales"])
    elif kind == "attend" and s["case"]["cache"] == "e4m3":
        for name in ("cache", "shared"):
            if s[name] is not None:
                s[name] = tuple(G.QuantRows(c, e) for c, e in s[name])


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    return (_RUN_OWN if own else _RUN_PLAIN)[s["case"]["kind"]](s)


def _attend_own(s):
    tree = s["case"]["nodes"] > 0
    s["ctx"].tree_attention(s["q"], s["k"], s["v"], s["n_nodes"], s["mask"] if tree else None,
                            cache=s["cache"], cache_len=s["cache_len"], shared=s["shared"],
                            with_root=True, out=s["out"], lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


def _sample_own(s):
    a, n, t, lp = s["ctx"].accept_sampled(
        s["n_nodes"], s["tokens"], s["parents"], s["logits"][:, 0], s["logits"][:, 1:],
        s["uniform"], temperature=s["temperature"], acc_len=s["acc_len"],
        acc_nodes=s["acc_nodes"], bonus=s["bonus"], logp=s["logp"])
    return dict(acc_len=a, acc_nodes=n, bonus=t, logp=lp)


def _write_own(s):
    ctx, case = s["ctx"], s["case"]
    if case["paths"]:
        ctx.cache_write(s["cache"], s["src"], s["n"], rows=s["nodes"], start=s["start"],
                        with_root=True)
        n = s["n"] + 1
    else:
        ctx.cache_write(s["cache"], s["src"], s["n"], start=s["start"])
        n = s["n"]
    return ctx.cache_read(s["cache"], n, start=s["start"], out=s["out"])


def _read_own(s):
    return s["ctx"].cache_read(s["cache"], s["n"], start=s["start"], out=s["out"])


def _attend_plain(s):
    case, q = s["case"], s["q"]
    B, S, Hq, D = q.shape
    H = case["kv_heads"]
    G = Hq // H
    quant = case["cache"] == "e4m3"
    plain = (lambda x: _values(*x)) if quant else (lambda x: x.float())
    cut = (lambda x, b, n: (x[0][b, :n], x[1][b, :n])) if quant else (lambda x, b, n: x[b, :n])
    shared = [plain(x) for x in s["shared"]] if s["shared"] is not None else None
    # visible slots: the root's for all, a node's ancestors and itself
    j = torch.arange(S - 1, device=q.device)
    seen = torch.zeros(B, S, S, dtype=torch.bool, device=q.device)
    seen[:, :, 0] = True
    seen[:, 1:, 1:] = ((s["mask"][:, :S - 1, j >> 6] >> (j & 63)) & 1) == 1
    live = torch.arange(S, device=q.device)[None, :] <= s["n_nodes"][:, None]
    seen &= live[:, None, :]
    out, lse = torch.zeros_like(q), torch.zeros(B, S, Hq, device=q.device)
    for b in range(B):
        n, m = int(s["lens"][b]), int(s["counts"][b]) + 1
        own_k, own_v = (plain(cut(x, b, n)) for x in s["cache"])
        k = torch.cat(([shared[0]] if shared else []) + [own_k, s["k"][b, :m].float()])
        v = torch.cat(([shared[1]] if shared else []) + [own_v, s["v"][b, :m].float()])
        qb = q[b, :m].float().reshape(m, H, G, D).transpose(0, 1).reshape(H, m * G, D)
        score = torch.matmul(qb, k.permute(1, 2, 0).contiguous()) / math.sqrt(D)
        score = score.view(H, m, G, -1)
        score[..., -m:] = torch.where(seen[b, :m, None, :m], score[..., -m:], -math.inf)
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul((p / total).view(H, m * G, -1), v.permute(1, 0, 2).contiguous())
        out[b, :m] = o.view(H, m, G, D).transpose(0, 1).reshape(m, Hq, D).to(q.dtype)
        lse[b, :m] = (top + torch.log(total)).view(H, m, G).transpose(0, 1).reshape(m, Hq)
    return dict(out=out, lse=lse)


def _sample_plain(s):
    z, u = s["logits"], s["uniform"]
    B, _, V = z.shape
    L = u.shape[1] - 1
    dev = z.device
    pick = torch.arange(B, device=dev)
    index = torch.arange(s["tokens"].shape[1], device=dev)
    listed_ = index[None, :] < s["n_nodes"][:, None]
    T = s["temperature"].double()
    greedy = T == 0
    inverse = 1.0 / torch.where(greedy, 1.0, T)
    cur = torch.full((B,), -1, dtype=torch.long, device=dev)
    going = torch.ones(B, dtype=torch.bool, device=dev)
    acc = torch.zeros(B, dtype=torch.long, device=dev)
    nodes = torch.full((B, L), -1, dtype=torch.long, device=dev)
    bonus = torch.zeros(B, dtype=torch.long, device=dev)
    logp = torch.zeros(B, L + 1, dtype=torch.float64, device=dev)
    for d in range(L + 1):
        row = z[pick, cur + 1].double()
        top = row.amax(-1, keepdim=True)
        best = (row == top).to(torch.int8).argmax(-1)
        e = torch.exp((row - top) * inverse[:, None])
        total = torch.cumsum(e, -1)
        x = (total <= u[:, d, None] * total[:, -1:]).sum(-1).clamp_max(V - 1)
        x = torch.where(greedy, best, x)
        lp = torch.where(greedy, 0.0, torch.log(e[pick, x] / total[:, -1]))
        logp[:, d] = torch.where(going, lp, 0.0)
        bonus = torch.where(going, x, bonus)
        hit = listed_ & (s["parents"] == cur[:, None]) & (s["tokens"] == x[:, None])
        found = hit.any(-1) & going & (d < L)
        child = hit.to(torch.int8).argmax(-1)
        if d < L:
            nodes[:, d] = torch.where(found, child, -1)
        acc += found
        cur = torch.where(found, child, cur)
        going = found
    return dict(acc_len=acc.int(), acc_nodes=nodes.int(), bonus=bonus.int(), logp=logp.float())


def _write_plain(s):
    case = s["case"]
    B, M = case["batch"], case["most"]
    i = torch.arange(M, device=s["src"].device)
    if case["paths"]:
        count = s["n"] + 1
        row = torch.cat([torch.zeros_like(s["nodes"][:, :1]), s["nodes"] + 1], 1).long()
    else:
        count = s["n"]
        row = i.expand(B, M)
    pick = torch.arange(B, device=row.device)[:, None]
    live = (i[None, :] < count[:, None])[None, :, :, None]
    codes, scales = _quantise(s["src"][:, pick, row.clamp_min(0)])
    at = s["start"][:, None] + i[None, :]
    old = s["codes"].view(torch.uint8)[:, pick, at]
    s["codes"].view(torch.uint8)[:, pick, at] = torch.where(live[..., None], codes.view(torch.uint8), old)
    s["scales"][:, pick, at] = torch.where(live, scales, s["scales"][:, pick, at])
    back = _values(s["codes"].view(torch.uint8)[:, pick, at].view(torch.float8_e4m3fn),
                   s["scales"][:, pick, at])
    return torch.where(live[..., None], back, 0.0).to(torch.bfloat16)


def _read_plain(s):
    M = s["case"]["length"]
    i = torch.arange(M, device=s["codes"].device)
    pick = torch.arange(s["case"]["batch"], device=i.device)[:, None]
    at = s["start"][:, None] + i[None, :]
    live = (i[None, :] < s["n"][:, None])[None, :, :, None, None]
    back = _values(s["codes"].view(torch.uint8)[:, pick, at].view(torch.float8_e4m3fn),
                   s["scales"][:, pick, at])
    return torch.where(live, back, 0.0).to(torch.bfloat16)


_RUN_OWN = dict(attend=_attend_own, sample=_sample_own, write=_write_own, read=_read_own)
_RUN_PLAIN = dict(attend=_attend_plain, sample=_sample_plain, write=_write_plain,
                  read=_read_plain)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _visited_rows(case):
    """Rows of logits that the walk reads, as an expectation: a node's children together have
    CHILD_MASS, and nine in ten of it goes to children that have children."""
    return case["batch"] * sum((0.9 * CHILD_MASS) ** d for d in range(case["depth"] + 1))


def work(case):
    B = case["batch"]
    if case["kind"] == "attend":
        Hq, H, D, P = case["q_heads"], case["kv_heads"], case["dim"], case["shared"]
        lens = _spread(B, max(1, case["length"] // 16), case["length"]).astype(np.int64)
        slots = _node_counts(case).astype(np.int64) + 1
        keys = P + lens + slots
        per_row = D + 1 if case["cache"] == "e4m3" else 2 * D
        queries = int(slots.sum())
        return dict(bytes=queries * Hq * (4 * D + 4) + queries * H * 4 * D
                    + 2 * H * per_row * (int(lens.sum()) + P),
                    flops=4 * D * Hq * int((slots * keys).sum()))
    if case["kind"] == "sample":
        rows = _visited_rows(case)
        es = 4 if case["dtype"] == "float32" else 2
        return dict(bytes=rows * case["vocab"] * es + 8 * B * case["nodes"],
                    flops=rows * case["vocab"] * 4)
    P, H, D = case["planes"], case["heads"], case["dim"]
    if case["kind"] == "write":
        if case["paths"]:
            n = int((_spread(B, 0, case["most"] - 1) * 4 // 10 + 1).sum())
        else:
            n = int(_spread(B, max(1, case["most"] // 4), case["most"]).sum())
        # read bf16, write codes and scales; the rows read back
        return dict(bytes=P * H * n * (2 * D + 2 * (D + 1) + 2 * D), flops=P * H * n * D * 4)
    n = int(_spread(B, max(1, case["length"] // 8), case["length"]).astype(np.int64).sum())
    return dict(bytes=P * H * n * (D + 1 + 2 * D), flops=P * H * n * D)


# ---------------------------------------------------------------------------
# The same results in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    return _EXACT[case["kind"]](case, _INPUTS[case["kind"]](case, seed))


def _decode(pair):
    """A quantised pair's numbers in 64 bits, from the bits: sign, 4 exponent bits (bias 7), 3 of
    the fraction."""
    c = pair[0].view(torch.uint8).to(torch.int64)
    ex, fr = (c >> 3) & 15, c & 7
    sub = fr.double() * 2.0 ** -9
    nor = (8 + fr).double() * _pow2_64(ex - 10)
    mag = torch.where(ex == 0, sub, nor) * _pow2_64(pair[1].to(torch.int64) - 127)[..., None]
    return torch.where(c >= 128, -mag, mag)


def _attend_exact(case, s):
    """Row by row of the key heads; a node's visible slots from the parents, not the bitset."""
    q = s["q"].double()
    B, S, Hq, D = q.shape
    H = case["kv_heads"]
    G = Hq // H
    number = _decode if case["cache"] == "e4m3" else (lambda x: x.double())
    out = torch.zeros(B, S, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.zeros(B, S, Hq, dtype=torch.float64, device=q.device)
    for b in range(B):
        n, m = int(s["lens"][b]), int(s["counts"][b]) + 1
        see = np.zeros((m, m), bool)
        for i in range(m):
            see[i, 0] = see[i, i] = True
            p = s["parents"][b, i - 1] if i else -1
            if p >= 0:
                see[i] |= see[p + 1]
        hide = torch.from_numpy(~see).to(q.device)
        for h in range(H):
            def side(i):
                own_ = s["cache"][i]
                own_ = (tuple(x[b, :n, h] for x in own_) if case["cache"] == "e4m3"
                        else own_[b, :n, h])
                parts = [number(own_), (s["k"], s["v"])[i][b, :m, h].double()]
                if s["shared"] is not None:
                    x = s["shared"][i]
                    x = tuple(y[:, h] for y in x) if case["cache"] == "e4m3" else x[:, h]
                    parts.insert(0, number(x))
                return torch.cat(parts)
            k, v = side(0), side(1)
            for g in range(G):
                a = q[b, :m, h * G + g] @ k.T.contiguous() * D ** -0.5
                a[:, -m:].masked_fill_(hide, -math.inf)
                z = torch.logsumexp(a, -1)
                lse[b, :m, h * G + g] = z
                out[b, :m, h * G + g] = torch.exp(a - z[:, None]) @ v
    return dict(out=out, lse=lse)


def _sample_exact(case, s):
    B, L, V = case["batch"], case["depth"], case["vocab"]
    tokens, parents = s["tokens"].cpu().numpy(), s["parents"].cpu().numpy()
    u, T = s["uniform"].cpu().numpy(), s["temperature"].cpu().numpy()
    acc, bonus = np.zeros(B, np.int32), np.zeros(B, np.int32)
    nodes, logp = np.full((B, L), -1, np.int32), np.zeros((B, L + 1))
    for b in range(B):
        below = {}
        for i in range(int(s["counts"][b]) - 1, -1, -1):
            below[(int(parents[b, i]), int(tokens[b, i]))] = i
        at = -1
        for d in range(L + 1):
            row = s["logits"][b, at + 1].float().cpu().numpy().astype(np.float64)
            if T[b] == 0:
                x, lp = int(np.argmax(row)), 0.0
            else:
                a = (row - row.max()) / np.float64(T[b])
                e = np.exp(a)
                c = np.cumsum(e)
                x = min(int(np.searchsorted(c, u[b, d] * c[-1], side="right")), V - 1)
                lp = a[x] - math.log(c[-1])
            logp[b, d], bonus[b] = lp, x
            at = below.get((at, x), -2) if d < L else -2
            if at < 0:
                break
            nodes[b, d] = at
            acc[b] += 1
    t = torch.from_numpy
    return dict(acc_len=t(acc), acc_nodes=t(nodes), bonus=t(bonus), logp=t(logp))


def _round_e4m3(x):
    """x (64 bits, at most 448 in magnitude) to the nearest e4m3 number, ties to even."""
    _, power = torch.frexp(x)
    step = _pow2_64((power - 1).clamp_min(-6) - 3)
    return torch.round(x / step) * step


def _write_exact(case, s):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    nodes = s["nodes"].cpu().numpy() if case["paths"] else None
    for b in range(case["batch"]):
        n = int(s["n_h"][b])
        rows = [0] + [int(v) + 1 for v in nodes[b, :n]] if case["paths"] else list(range(n))
        x = s["src"][:, b, torch.tensor(rows, device="cuda")].double()
        top = x.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(top / 448.0))
        e = torch.where(top > 448.0 * _pow2_64(e), e + 1, e)
        e = torch.where(top <= 448.0 * _pow2_64(e - 1), e - 1, e).clamp_min(-118)
        unit = _pow2_64(e)
        out[:, b, :len(rows)] = _round_e4m3(x / unit) * unit
    return out


def _read_exact(case, s):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        n, a = int(s["n_h"][b]), int(s["start_h"][b])
        out[:, b, :n] = _decode((s["codes"].view(torch.uint8)[:, b, a:a + n],
                                 s["scales"][:, b, a:a + n]))
    return out


_EXACT = dict(attend=_attend_exact, sample=_sample_exact, write=_write_exact, read=_read_exact)
