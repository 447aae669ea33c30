"""A target model's layer around a paged key/value cache, as measurable cases.

Three groups of operators, each with a plain form in elementary torch operations
and the calls that a user makes of paper_2608_20375_amd:

attend   Context.paged_attention: attention of a block of new rows (one token, a
         drafted chain, a draft tree under its ancestor mask, a piece of a prompt)
         over a cache in pages, the block's own rows behind it; with a sliding
         window and a few first rows that stay visible where the case has one.
write    Context.paged_write: a block's queries and keys rotated by their positions
         (one axis, or three), keys and values appended to the pages, plain or
         quantised.  Quantised pages are read back with Context.cache_read, as the
         numbers that they stand for.
commit   Context.paged_commit: the rows of the accepted path moved up in the pages of
         all layers.

Inputs are drawn from the seed alone.  Lengths and counts are a fixed spread of the
case's range in an order that the seed draws, so a case's work does not depend on
the seed; pages lie in the pool in a drawn order.
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
        # One user's next token over a short cache: the smallest attention, where
        # launches and latency count.
        dict(name="attend_b1_token", kind="attend", batch=1, slots=1, tree=False, q_heads=32, kv_heads=8,
             dim=128, dtype="bfloat16", cache="same", page=16, length=700, window=0, sinks=0),
        # A serving batch at one token a sequence over ragged quantised caches: bound by
        # the cache's bytes.
        dict(name="attend_b64_token_e4m3", kind="attend", batch=64, slots=1, tree=False, q_heads=32,
             kv_heads=8, dim=128, dtype="bfloat16", cache="e4m3", page=64, length=8192, window=0, sinks=0),
        # Odd sizes: five sequences, chains of up to three, five query heads a key head, 80
        # numbers a head, pages that end inside every tile, half precision.
        dict(name="attend_b5_odd_fp16", kind="attend", batch=5, slots=3, tree=False, q_heads=20, kv_heads=4,
             dim=80, dtype="float16", cache="same", page=24, length=1531, window=500, sinks=3),
        # Long conversations of a model with a sliding window: only the window and the
        # first rows are visible.
        dict(name="attend_b32_window", kind="attend", batch=32, slots=1, tree=False, q_heads=32, kv_heads=8,
             dim=128, dtype="bfloat16", cache="same", page=16, length=16384, window=4096, sinks=4),
        # The verifier's pass: draft trees of up to 64 nodes with the root.
        dict(name="attend_b16_tree64", kind="attend", batch=16, slots=65, tree=True, q_heads=32, kv_heads=8,
             dim=128, dtype="bfloat16", cache="same", page=32, length=4096, window=0, sinks=0),
        # Prompts in pieces of 1024 tokens, windowed: bound by matrix products.
        dict(name="attend_b8_piece1024", kind="attend", batch=8, slots=1024, tree=False, q_heads=32,
             kv_heads=8, dim=128, dtype="bfloat16", cache="same", page=64, length=4096, window=2048, sinks=4),
        # One token's row: the smallest write.
        dict(name="write_b1_token", kind="write", batch=1, slots=1, q_heads=32, kv_heads=8, dim=128, rot=128,
             axes=1, interleaved=False, dtype="bfloat16", cache="same", page=16, start=700),
        # The batch-64 round's blocks into quantised pages, at the tree's positions.
        dict(name="write_b64_tree_e4m3", kind="write", batch=64, slots=65, q_heads=32, kv_heads=8, dim=128,
             rot=128, axes=1, interleaved=False, dtype="bfloat16", cache="e4m3", page=64, start=8192),
        # Odd sizes: part of a head rotated, neighbouring numbers as pairs, half precision.
        dict(name="write_b5_odd_fp16", kind="write", batch=5, slots=37, q_heads=20, kv_heads=4, dim=80, rot=48,
             axes=1, interleaved=True, dtype="float16", cache="same", page=24, start=120000),
        # Prompts with pictures: positions of three axes (time, height, width).
        dict(name="write_b4_prompt_axes3", kind="write", batch=4, slots=2048, q_heads=32, kv_heads=8, dim=128,
             rot=128, axes=3, interleaved=False, dtype="bfloat16", cache="same", page=16, start=2048),
        # One sequence's accepted path in a 16-layer cache.
        dict(name="commit_b1_path", kind="commit", batch=1, slots=33, planes=32, kv_heads=4, dim=128, most=8,
             dtype="bfloat16", page=16, start=700),
        # The batch-64 round's accepted paths, 36 layers of keys and values.
        dict(name="commit_b64_path", kind="commit", batch=64, slots=129, planes=72, kv_heads=8, dim=128, most=16,
             dtype="bfloat16", page=64, start=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case: attention in six of ten draws, then writes, then commits."""
    u = rng.random()
    page = rng.choice((8, 16, 16, 24, 32, 64, 64, 100, 128))
    if u < 0.6:
        kv = rng.choice((1, 2, 4, 8, 8))
        q = kv * rng.choice((1, 2, 4, 4, 5, 7, 8))
        dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 128))
        dtype = rng.choice(("bfloat16", "bfloat16", "float16"))
        cache = rng.choice(("same", "e4m3")) if dtype == "bfloat16" else "same"
        tree = rng.random() < 0.3
        slots = (_log_int(rng, 4, 130) if tree
                 else rng.choice((1, 1, 1, rng.randint(2, 8), _log_int(rng, 16, 1024))))
        length = _log_int(rng, 16, 65536)
        window, sinks = 0, 0
        if rng.random() < 0.4:
            window, sinks = _log_int(rng, 64, 8192), rng.choice((0, 1, 4, 4, 64))
        seen = min(length / 2, window + sinks) if window else length / 2
        most = int(8 * 1024 * 32 * 128 * 2048 / (slots * q * dim * (seen + slots)))
        cells = int(2.5e8 / (kv * dim * (length + slots + page)))     # a cache of at most 1 GB
        batch = max(1, min(_log_int(rng, 1, 64), most, cells, int(7e7 / (q * dim * slots))))
        return dict(kind="attend", batch=batch, slots=slots, tree=tree, q_heads=q, kv_heads=kv, dim=dim,
                    dtype=dtype, cache=cache, page=page, length=length, window=window, sinks=sinks)
    if u < 0.85:
        kv = rng.choice((1, 2, 4, 5, 8))
        q = kv * rng.choice((1, 2, 4, 5, 8))
        dim = rng.choice((32, 64, 80, 96, 128, 128))
        rot = rng.choice((dim, dim, dim, 16 * rng.randint(1, dim // 16)))
        dtype = rng.choice(("bfloat16", "bfloat16", "float16"))
        cache = rng.choice(("same", "e4m3")) if dtype == "bfloat16" else "same"
        slots = rng.choice((1, _log_int(rng, 2, 130), _log_int(rng, 16, 2048)))
        batch = max(1, min(_log_int(rng, 1, 64), int(4 * 2048 * 32 * 128 / (slots * q * dim))))
        return dict(kind="write", batch=batch, slots=slots, q_heads=q, kv_heads=kv, dim=dim, rot=rot,
                    axes=rng.choice((1, 1, 2, 3)), interleaved=rng.random() < 0.4, dtype=dtype, cache=cache,
                    page=page, start=_log_int(rng, 1, 200000))
    heads, dim, slots, start = (rng.choice((1, 2, 4, 8)), rng.choice((32, 64, 80, 128)), rng.randint(34, 129),
                                _log_int(rng, 1, 256))
    planes = rng.randint(2, 72)
    batch = max(1, min(_log_int(rng, 1, 64), int(9e8 / ((start + slots + page) * planes * heads * dim))))
    return dict(kind="commit", batch=batch, slots=slots, planes=planes, kv_heads=heads, dim=dim,
                most=rng.choice((4, 8, 16)), dtype=rng.choice(("bfloat16", "float16")), page=page, start=start)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 23)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _spread(count, lo, hi, rng=None):
    """count sizes spread evenly over lo..hi (the largest among them), in an order drawn by rng."""
    v = np.array([hi - (hi - lo) * i // max(1, count) for i in range(count)], np.int32)
    return v if rng is None else rng.permutation(v).astype(np.int32)


def _lengths(case, rng=None):
    return _spread(case["batch"], max(1, case["length"] // 16), case["length"], rng)


def _slot_counts(case, rng=None):
    """New rows of each sequence: all of a prompt's piece or token, a spread of chains and trees."""
    s = case["slots"]
    if case["kind"] == "attend" and not case["tree"] and s > 8:
        return np.full(case["batch"], s, np.int32)
    return _spread(case["batch"], max(1, s // 2), s, rng)


def _table(rng, page, rows, pages=None):
    """Page tables of sequences of `rows` rows each (-1 behind them), pages in a drawn order, and
    the pool's size (`pages`, or as many as are needed)."""
    need = -(-rows.astype(np.int64) // page)
    pool = rng.permutation(pages or int(need.sum())).astype(np.int32)
    table = np.full((len(rows), int(need.max())), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = pool[at:at + n]
        at += n
    return table, len(pool)


def _pow2(e):
    """2^e in fp32, exactly: integers e in -126..127."""
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
    return (x * _pow2(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The numbers that codes and scales stand for, in fp32."""
    return codes.float() * _pow2(scales.to(torch.int32) - 127)[..., None]


def _pool(*shape, dtype):
    """Zeros [.., pages, rows, heads, dim] whose pages hold a head's rows side by side."""
    *lead, rows, heads, dim = shape
    return torch.zeros(*lead, heads, rows, dim, dtype=dtype, device="cuda").transpose(-2, -3)


def _tree(rng, n, depth):
    """parents of a tree of n nodes in canonical order (by depth); every depth's first node has
    children."""
    depth = min(depth, n)
    count = np.full(depth, n // max(1, depth), int)
    count[-1:] += n - count.sum()
    parents, before, first = [], 1, -1
    at = 0
    for d in range(depth):
        p = np.sort(rng.integers(0, before, count[d])) + first if d else np.full(count[d], -1)
        if d:
            p[0] = first
            p.sort()
        parents.append(p)
        first, before = at, count[d]
        at += count[d]
    return np.concatenate(parents).astype(np.int32) if parents else np.zeros(0, np.int32)


def _ancestors(parents):
    n = len(parents)
    seen = np.eye(n, dtype=bool)
    for i in range(n):
        if parents[i] >= 0:
            seen[i] |= seen[parents[i]]
    return seen


def _attend_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    B, S, Hq, H, D = case["batch"], case["slots"], case["q_heads"], case["kv_heads"], case["dim"]
    dt = getattr(torch, case["dtype"])
    lens, counts = _lengths(case, rng), _slot_counts(case, rng)
    table, pages = _table(rng, case["page"], lens + counts)
    s = dict(q=torch.empty(B, S, Hq, D, dtype=dt, device="cuda").normal_(generator=g).mul_(2.0))
    pools = [_pool(pages, case["page"], H, D, dtype=dt) for _ in range(2)]
    for x in pools:
        x.transpose(1, 2).normal_(generator=g)
    if case["cache"] == "e4m3":
        flat = [_quantise(x.transpose(1, 2)) for x in pools]
        s["k"], s["v"] = ((c.transpose(1, 2), e.transpose(1, 2)) for c, e in flat)
    else:
        s["k"], s["v"] = pools
    mask = parents = None
    if case["tree"]:        # slot 0 is the root, nodes follow
        N = S - 1
        mask = np.zeros((B, N, (N + 63) // 64), np.uint64)
        parents = []
        for b in range(B):
            p = _tree(rng, int(counts[b]) - 1, 16)
            seen = _ancestors(p)
            for j in range(len(p)):
                mask[b, :len(p), j >> 6] |= seen[:, j].astype(np.uint64) << np.uint64(j & 63)
            parents.append(p)
        mask = _dev(mask.view(np.int64))
    s.update(table=_dev(table), cache_len=_dev(lens), mask=mask, parents=parents, lens=lens, counts=counts,
             n=_dev(counts), n_nodes=_dev(counts - 1))
    return s


def _write_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    B, S, Hq, H, D = case["batch"], case["slots"], case["q_heads"], case["kv_heads"], case["dim"]
    P, dt = case["page"], getattr(torch, case["dtype"])
    counts = _slot_counts(case, rng)
    start = _spread(B, max(0, case["start"] // 2), case["start"], rng)
    # pages in front of a sequence's first new row are not needed here: all of them page 0's
    first = start // P
    table = np.zeros((B, int((start + counts - 1).max()) // P + 1), np.int32)
    mine, pages = _table(rng, P, start - first * P + counts, B * (-(-(P - 1 + S) // P)))
    for b in range(B):
        n = int((mine[b] >= 0).sum())
        table[b, first[b]:first[b] + n] = mine[b, :n]

    def normal(*shape):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g)

    # a few dimensions of each head are larger, as keys' are
    size = torch.exp(torch.randn(H, D, device="cuda", generator=g)).to(dt)
    s = dict(q=normal(B, S, Hq, D), k=normal(B, S, H, D).mul_(size), v=normal(B, S, H, D))
    F = case["rot"] // 2
    freq = 10000.0 ** -(np.arange(F) / F)
    if case["axes"] == 1:   # a tree's positions: by depth; a prompt's: one after the other
        step = np.arange(S) if S > 130 else np.ceil(np.arange(S) / max(1, S // 16))
        pos = (start[:, None] + step[None, :])[None]
        axis = None
    else:                   # text, then pictures of 24 columns: time, height, width
        i = np.arange(S)
        t = start[:, None] + (i // 96)[None, :]
        pos = np.stack([t, t + (i // 24 % 4)[None, :], t + (i % 24)[None, :]][:case["axes"]])
        axis = _dev(np.sort(np.arange(F) * case["axes"] // F).astype(np.int32))
    if case["cache"] == "e4m3":
        s["codes"] = _pool(2, pages, P, H, D, dtype=torch.float8_e4m3fn)
        s["scales"] = torch.zeros(2, pages, H, P, dtype=torch.uint8, device="cuda").transpose(2, 3)
        s["back"] = torch.zeros(2, pages, P, H, D, dtype=torch.bfloat16, device="cuda")
        s["full"] = torch.full((pages,), P, dtype=torch.int32, device="cuda")
    else:
        s["pool"] = _pool(2, pages, P, H, D, dtype=dt)
    s.update(table=_dev(table), n=_dev(counts), start=_dev(start), pos=_dev(pos.astype(np.int32)), axis=axis,
             freq=_dev(freq), q_out=torch.zeros_like(s["q"]), pages=pages, counts=counts, starts=start,
             tables=table)
    return s


def _commit_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    B, M, N = case["batch"], case["most"], case["slots"] - 1
    start = _spread(B, max(0, case["start"] // 2), case["start"], rng)
    table, pages = _table(rng, case["page"], start + case["slots"])
    n = _spread(B, M // 4, M, rng)
    # wide trees: an accepted node lies behind all rows that the path will take
    nodes = np.full((B, M), -1, np.int32)
    for b in range(B):
        nodes[b, :n[b]] = np.sort(rng.choice(np.arange(n[b], N), n[b], replace=False))
    pool = _pool(case["planes"], pages, case["page"], case["kv_heads"], case["dim"],
                 dtype=getattr(torch, case["dtype"]))
    pool.transpose(2, 3).normal_(generator=g)
    return dict(pool=pool, table=_dev(table), start=_dev(start), n=_dev(n), nodes=_dev(nodes), starts=start,
                tables=table, n_h=n, nodes_h=nodes)


_INPUTS = dict(attend=_attend_inputs, write=_write_inputs, commit=_commit_inputs)


def prepare(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    s["case"] = case
    if case["kind"] == "attend":
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(s["q"].shape[:3], dtype=torch.float32, device="cuda")
    if own:
        s["ctx"] = _context(s)
    return s


def _context(s):
    """The framework's handle, sized for the case, and quantised pages as its objects."""
    import paper_2608_20375_amd as G
    case = s["case"]
    if case.get("cache") == "e4m3":
        if case["kind"] == "attend":
            s["k"], s["v"] = G.QuantRows(*s["k"]), G.QuantRows(*s["v"])
        else:
            s["cache"] = G.QuantRows(s["codes"], s["scales"])
    depth = case["most"] if case["kind"] == "commit" else 16
    batch = max(case["batch"], s["pages"]) if case["kind"] == "write" else case["batch"]
    return G.Context(batch, depth, 64, 1, max(1, min(1024, case["slots"] - 1)))


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    return (_RUN_OWN if own else _RUN_PLAIN)[s["case"]["kind"]](s)


def _attend_own(s):
    case = s["case"]
    s["ctx"].paged_attention(s["q"], (s["k"], s["v"]), s["table"], s["cache_len"],
                             s["n_nodes"] if case["tree"] else s["n"], s["mask"], with_root=case["tree"],
                             window=case["window"] or None, sinks=case["sinks"], out=s["out"], lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


def _write_own(s):
    case = s["case"]
    pool = s["cache"] if case["cache"] == "e4m3" else s["pool"]
    s["ctx"].paged_write((pool[0], pool[1]), s["table"], s["k"], s["v"], s["n"], s["start"], q=s["q"],
                         q_out=s["q_out"], freq=s["freq"], positions=s["pos"], axis=s["axis"],
                         interleaved=case["interleaved"])
    if case["cache"] == "e4m3":
        pool = s["ctx"].cache_read(s["cache"], s["full"], out=s["back"])
    return dict(q=s["q_out"], pool=pool)


def _commit_own(s):
    return s["ctx"].paged_commit(s["pool"], s["table"], s["start"], s["n"], s["nodes"], with_root=True)


def _rows_at(table, page, b, row):
    """Page and row in it of rows of sequences b."""
    return table[b, torch.div(row, page, rounding_mode="floor")].long(), row % page


def _attend_plain(s):
    case, q = s["case"], s["q"]
    B, S, Hq, D = q.shape
    H, P = case["kv_heads"], case["page"]
    base, n = s["cache_len"].long(), s["n"].long()
    dev = q.device
    slot = torch.arange(S, device=dev)
    # block: slots that a slot sees, and its place: that many behind the cache's last row
    if case["tree"]:
        j = torch.arange(S - 1, device=dev)
        block = torch.zeros(B, S, S, dtype=torch.bool, device=dev)
        block[:, :, 0] = True
        block[:, 1:, 1:] = ((s["mask"][:, :, j >> 6] >> (j & 63)) & 1) == 1
        place = block.sum(-1) - 1
    else:
        block = (slot[None, :] <= slot[:, None]).expand(B, S, S)
        place = slot.expand(B, S)
    # the rows that any slot may see: the first ones, and those from the window's begin on
    most = int(case["length"]) + S
    window, sinks = case["window"], case["sinks"]
    if window and window + sinks + S < most:
        low = (base - window + 1).clamp_min(0)
        first = torch.arange(sinks, device=dev).expand(B, sinks)
        rest = low[:, None] + torch.arange(window - 1 + S, device=dev)
        row = torch.cat([torch.where(first < low[:, None], first, -1), rest], 1)
    else:
        row = torch.arange(most, device=dev).expand(B, most)
    inside = (row >= 0) & (row < (base + n)[:, None])
    page, at = _rows_at(s["table"], P, torch.arange(B, device=dev)[:, None], torch.where(inside, row, 0))
    page = page.clamp_min(0)
    # who sees what
    r = row[:, None, :]
    here = base[:, None, None]
    seen = torch.gather(block, 2, (r - here).clamp(0, S - 1).expand(B, S, -1)) | (r < here)
    if window:
        near = (r > here + place[:, :, None] - window) | (r < sinks)
        seen &= near | (r >= here) if case["tree"] else near
    seen &= inside[:, None, :]

    def side(x):
        if case["cache"] == "e4m3":
            codes = x[0].view(torch.uint8)[page, at].view(torch.float8_e4m3fn)
            return _values(codes, x[1][page, at]).permute(0, 2, 1, 3).contiguous()
        return x[page, at].float().permute(0, 2, 1, 3).contiguous()

    k, v = side(s["k"]), side(s["v"])                                  # [B, H, rows, D]
    qb = q.float().view(B, S, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    score = torch.matmul(qb, k.transpose(2, 3).contiguous()).div_(math.sqrt(D)).view(B, H, S, Hq // H, -1)
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, H, S * (Hq // H), -1), v).view(B, H, S, Hq // H, D) / total
    lse = (top + torch.log(total))[..., 0].permute(0, 2, 1, 3).reshape(B, S, Hq)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, S, Hq, D)
    live = slot[None, :] < n[:, None]
    return dict(out=torch.where(live[..., None, None], o, 0.0).to(q.dtype),
                lse=torch.where(live[..., None], lse, 0.0))


def _rotate(x, cos, sin, rot, interleaved):
    """x [B, S, heads, dim] fp32, cos and sin [B, S, 1, rot / 2]."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    pair = [a * cos - b * sin, b * cos + a * sin]
    turned = torch.stack(pair, -1).flatten(-2) if interleaved else torch.cat(pair, -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _write_plain(s):
    case = s["case"]
    rot, P = case["rot"], case["page"]
    B, S = s["q"].shape[:2]
    dev = s["q"].device
    pos = s["pos"][s["axis"].long()] if s["axis"] is not None else s["pos"][:1]
    angle = pos.double().permute(1, 2, 0) * s["freq"]                  # [B, S, rot / 2]
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    q = _rotate(s["q"].float(), cos, sin, rot, case["interleaved"])
    live = torch.arange(S, device=dev)[None, :] < s["n"][:, None]
    s["q_out"].copy_(torch.where(live[..., None, None], q, s["q_out"].float()))
    b, i = torch.nonzero(live, as_tuple=True)
    page, at = _rows_at(s["table"], P, b, s["start"][b] + i)
    new = torch.stack([_rotate(s["k"].float(), cos, sin, rot, case["interleaved"])[b, i], s["v"][b, i].float()])
    if case["cache"] != "e4m3":
        s["pool"][:, page, at] = new.to(s["pool"].dtype)
        return dict(q=s["q_out"], pool=s["pool"])
    codes, scales = _quantise(new)
    s["codes"].view(torch.uint8)[:, page, at] = codes.view(torch.uint8)
    s["scales"][:, page, at] = scales
    s["back"].copy_(_values(s["codes"], s["scales"]))
    return dict(q=s["q_out"], pool=s["back"])


def _commit_plain(s):
    P = s["case"]["page"]
    i = torch.arange(s["nodes"].shape[1], device=s["nodes"].device)
    b, i = torch.nonzero(i[None, :] < s["n"][:, None], as_tuple=True)
    base = s["start"][b].long() + 1                                    # behind the root
    p0, r0 = _rows_at(s["table"], P, b, base + s["nodes"][b, i])
    p1, r1 = _rows_at(s["table"], P, b, base + i)
    s["pool"][:, p1, r1] = s["pool"][:, p0, r0]
    return s["pool"]


_RUN_OWN = dict(attend=_attend_own, write=_write_own, commit=_commit_own)
_RUN_PLAIN = dict(attend=_attend_plain, write=_write_plain, commit=_commit_plain)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    B, H, D = case["batch"], case["kv_heads"], case["dim"]
    if case["kind"] == "commit":
        n = int(_spread(B, case["most"] // 4, case["most"]).sum())
        return dict(bytes=4 * n * case["planes"] * H * D, flops=0)
    Hq = case["q_heads"]
    row = D + 1 if case["cache"] == "e4m3" else 2 * D                  # a cache row of a head
    slots = _slot_counts(case).astype(np.int64)
    if case["kind"] == "write":
        n = int(slots.sum())
        extra = 0
        if case["cache"] == "e4m3":                                    # the written rows read back
            extra = n * 2 * H * (row + 2 * D)
        return dict(bytes=n * (4 * Hq * D + 2 * H * (2 * D + row) + 4 * case["axes"]) + extra,
                    flops=n * (Hq + H) * case["rot"] * 3)
    # sizes of sequences are drawn in any order: sums of products over their means
    lens = _lengths(case).astype(np.float64)
    w, k = case["window"], case["sinks"]
    tail = (slots + 1) / 2 if not case["tree"] else np.minimum(slots, 9)
    old = lens.mean() if not w else np.minimum(lens, k + np.maximum(0, w - tail.mean())).mean()
    read = lens.sum() if not w else np.minimum(lens, k + w - 1).sum()
    queries = int(slots.sum())
    pairs = float((slots * (old + tail)).sum())
    return dict(bytes=int(queries * Hq * (4 * D + 4) + 2 * H * row * (read + queries)),
                flops=int(4 * D * Hq * pairs))


# ---------------------------------------------------------------------------
# The same results in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    return _EXACT[case["kind"]](case, _INPUTS[case["kind"]](case, seed))


def _decode(codes, scales):
    """The numbers of codes in 64 bits, from the bits: sign, 4 exponent bits (bias 7), 3 of the
    fraction."""
    c = codes.view(torch.uint8).to(torch.int64)
    ex, fr = (c >> 3) & 15, c & 7
    mag = torch.where(ex == 0, fr.double() * 2.0 ** -9, (8 + fr).double() * _pow2_64(ex - 10))
    mag = mag * _pow2_64(scales.to(torch.int64) - 127)[..., None]
    return torch.where(c >= 128, -mag, mag)


def _attend_exact(case, s):
    """A sequence and key head at a time, its rows fetched page by page; a node's visible rows
    from the parents, not the bitset."""
    q = s["q"].double()
    B, S, Hq, D = q.shape
    H, G, P = case["kv_heads"], Hq // case["kv_heads"], case["page"]
    out = torch.zeros(B, S, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.zeros(B, S, Hq, dtype=torch.float64, device=q.device)
    table = s["table"].cpu().numpy()
    for b in range(B):
        base, n = int(s["lens"][b]), int(s["counts"][b])
        pages = torch.from_numpy(table[b, :-(-(base + n) // P)].astype(np.int64)).to(q.device)
        see = np.zeros((n, base + n), bool)
        for i in range(n):
            if case["tree"]:
                path, at = [0], i - 1
                while i and at >= 0:
                    path.append(at + 1)
                    at = int(s["parents"][b][at])
                see[i, base + np.array(path)] = True
                deep = len(path) - 1
            else:
                deep = i
                see[i, base:base + i + 1] = True
            see[i, :base] = True
            if case["window"]:
                lo = max(0, base + deep - case["window"] + 1)
                cut = see[i, :min(lo, base)] if case["tree"] else see[i, :lo]
                cut[case["sinks"]:] = False
        hide = torch.from_numpy(~see).to(q.device)
        for h in range(H):
            kv = []
            for x in (s["k"], s["v"]):
                if case["cache"] == "e4m3":
                    y = _decode(x[0].view(torch.uint8)[pages, :, h], x[1][pages, :, h])
                else:
                    y = x[pages, :, h].double()
                kv.append(y.reshape(-1, D)[:base + n])
            kt = kv[0].T.contiguous()
            for g in range(G):
                a = (q[b, :n, h * G + g] @ kt) * D ** -0.5
                a.masked_fill_(hide, -math.inf)
                z = torch.logsumexp(a, -1)
                lse[b, :n, h * G + g] = z
                out[b, :n, h * G + g] = torch.exp(a - z[:, None]) @ kv[1]
    return dict(out=out, lse=lse)


def _round_e4m3(x):
    """x (64 bits, at most 448 in magnitude) to the nearest e4m3 number, ties to even."""
    _, power = torch.frexp(x)
    step = _pow2_64((power - 1).clamp_min(-6) - 3)
    return torch.round(x / step) * step


def _write_exact(case, s):
    rot, F, P = case["rot"], case["rot"] // 2, case["page"]
    pos, freq = s["pos"].double(), s["freq"].double()
    turn = []                                                          # e^(i angle), [B, S, 1]
    for f in range(F):
        axis = int(s["axis"][f]) if s["axis"] is not None else 0
        turn.append(torch.polar(torch.ones_like(pos[axis]), pos[axis] * freq[f])[..., None])

    def rotated(x):
        y = x.double().clone()
        for f in range(F):
            i, j = (2 * f, 2 * f + 1) if case["interleaved"] else (f, f + F)
            z = torch.complex(x[..., i].double(), x[..., j].double()) * turn[f]
            y[..., i], y[..., j] = z.real, z.imag
        return y

    q, k, v = rotated(s["q"]), rotated(s["k"]), s["v"].double()
    q_out = torch.zeros_like(q)
    H, D = k.shape[2:]
    pool = torch.zeros(2, s["pages"], P, H, D, dtype=torch.float64, device=q.device)
    for b in range(case["batch"]):
        n, first = int(s["counts"][b]), int(s["starts"][b])
        q_out[b, :n] = q[b, :n]
        for i in range(0, n):
            # rows of a page together
            if i and (first + i) % P:
                continue
            r = (first + i) % P
            m = min(P - r, n - i)
            pool[0, s["tables"][b, (first + i) // P], r:r + m] = k[b, i:i + m]
            pool[1, s["tables"][b, (first + i) // P], r:r + m] = v[b, i:i + m]
    if case["cache"] == "e4m3":
        top = pool.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(top / 448.0)).clamp_min(-118)
        e = torch.where(top > 448.0 * _pow2_64(e), e + 1, e)
        e = torch.where(top <= 448.0 * _pow2_64(e - 1), e - 1, e).clamp_min(-118)
        unit = _pow2_64(e)
        pool = _round_e4m3(pool / unit) * unit
    return dict(q=q_out, pool=pool)


def _commit_exact(case, s):
    pool, P = s["pool"].double(), case["page"]
    old = pool.clone()
    for b in range(case["batch"]):
        for i in range(int(s["n_h"][b])):
            x, y = int(s["starts"][b]) + 1 + int(s["nodes_h"][b, i]), int(s["starts"][b]) + 1 + i
            pool[:, s["tables"][b, y // P], y % P] = old[:, s["tables"][b, x // P], x % P]
    return pool


_EXACT = dict(attend=_attend_exact, write=_write_exact, commit=_commit_exact)
