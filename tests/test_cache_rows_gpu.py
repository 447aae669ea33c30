"""Context.cache_write and cache_read: every code, scale and number is exact, and rows that
a call does not name keep their bytes."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import verifier_ref as R  # noqa: E402

pytestmark = pytest.mark.gpu


def context(batch, L=8, N=64):
    import paper_2608_20375_amd as G
    return G.Context(batch, L, 64, 1, N)


def quant_cache(P, B, R_, H, D, fill=0xA5):
    import paper_2608_20375_amd as G
    c = G.QuantRows.empty(P, B, R_, H, D)
    c.codes.fill_(fill)
    c.scales.fill_(fill)
    return c


def special(shape, seed):
    """bf16 numbers with everything in them: ordinary, tiny and huge rows, zeros, infinities,
    NaN, numbers half way between codes, maxima at 448 * 2^e and just past it."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    rows = x.view(-1, shape[-1])
    for i in range(rows.shape[0]):
        k = i % 13
        if k == 1: rows[i] *= 2.0 ** -130
        elif k == 2: rows[i] *= 1e38
        elif k == 3: rows[i] = 0.0
        elif k == 4: rows[i, i % shape[-1]] = float("inf")
        elif k == 5: rows[i, :2] = torch.tensor([float("nan"), -float("inf")])
        elif k == 6: rows[i, 0] = 448.0
        elif k == 7: rows[i, 0] = 450.0
        elif k == 8: rows[i] = torch.arange(shape[-1]) * 17.0 / 16
        elif k == 9: rows[i] = float("nan")
        elif k == 10: rows[i, 3] = 3.3895314e38
        elif k == 11: rows[i] = rows[i].sign() * 2.0 ** (torch.arange(shape[-1]) % 20 - 12.0)
        elif k == 12: rows[i] *= 2.0 ** -118
    return x.to(torch.bfloat16)


def same_codes(got, want):
    """Equal bits; a NaN may have either sign."""
    nan = (want & 0x7F) == 0x7F
    return bool(((got == want) | (nan & ((got & 0x7F) == 0x7F))).all())


@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 112, 128])
@pytest.mark.parametrize("P,B,H,S", [(1, 1, 1, 1), (3, 2, 5, 33), (72, 3, 8, 20), (2, 2, 2, 200)])
def test_prompts(P, B, H, S, D):
    print("prompt", P, B, H, S, D, flush=True)
    ctx = context(B)
    src = special((P, B, S, H, D), S + D)
    n = np.array([S - 3 * b if S > 3 * b else 0 for b in range(B)], np.int32)
    start = np.array([5 * b for b in range(B)], np.int32)
    cache = quant_cache(P, B, S + 12, H, D)
    ctx.cache_write(cache, src.cuda(), torch.from_numpy(n).cuda(), start=torch.from_numpy(start).cuda())
    codes, scales = cache.codes.cpu(), cache.scales.cpu()
    rc, rs = R.quantise(src)
    for b in range(B):
        a, m = int(start[b]), int(n[b])
        assert same_codes(codes[:, b, a:a + m], rc[:, b, :m])
        assert torch.equal(scales[:, b, a:a + m], rs[:, b, :m])
        for part in (codes, scales):
            assert (part[:, b, :a] == 0xA5).all() and (part[:, b, a + m:] == 0xA5).all()
    # and back: exact in both types
    want = R.values(codes, scales)
    for dt in (torch.bfloat16, torch.float32):
        out = torch.full((P, B, S + 2, H, D), 7.0, dtype=dt, device="cuda")
        ctx.cache_read(cache, torch.from_numpy(n).cuda(), start=torch.from_numpy(start).cuda(), out=out)
        out = out.cpu().double()
        for b in range(B):
            a, m = int(start[b]), int(n[b])
            w = want[:, b, a:a + m]
            assert ((out[:, b, :m] == w) | (torch.isnan(out[:, b, :m]) & torch.isnan(w))).all()
            assert (out[:, b, m:] == 7.0).all()
    assert ctx.device_status() == 0
    ctx.close()


def test_every_code_of_every_scale_reads_exactly():
    import paper_2608_20375_amd as G
    ctx = context(1)
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(1, 1, 1, 2, 128).repeat(1, 1, 239, 1, 1)
    scales = torch.arange(9, 248, dtype=torch.int32).to(torch.uint8).view(1, 1, 239, 1).repeat(1, 1, 1, 2)
    want = R.values(codes, scales)
    fits = (want.abs() < 3.4e38) | torch.isnan(want)       # 2^120 times more than 240 is no fp32
    cache = G.QuantRows(codes.cuda(), scales.cuda())
    for dt in (torch.bfloat16, torch.float32):
        out = ctx.cache_read(cache, torch.tensor([239], dtype=torch.int32, device="cuda"), dtype=dt)
        out = out.cpu().double()
        assert (((out == want) | (torch.isnan(out) & torch.isnan(want))) | ~fits).all()
    ctx.close()


@pytest.mark.parametrize("kind", ["e4m3", "bfloat16", "float16"])
@pytest.mark.parametrize("P,B,L,H,D,S", [(1, 1, 1, 1, 16, 2), (72, 4, 8, 8, 128, 65), (5, 3, 33, 3, 80, 40),
                                         (2, 2, 64, 2, 64, 65)])
@pytest.mark.parametrize("root", [False, True])
def test_accepted_paths(kind, P, B, L, H, D, S, root):
    print("paths", kind, P, B, L, H, D, S, root, flush=True)
    rng = np.random.default_rng(L + D)
    ctx = context(B, min(L, 64), 64)
    dt = torch.bfloat16 if kind == "e4m3" else getattr(torch, kind)
    src = special((P, B, S, H, D), L).to(dt)
    most = min(L, S - 1)
    n = rng.integers(0, most + 1, B).astype(np.int32)
    n[0] = most
    nodes = np.full((B, L), -1, np.int32)
    for b in range(B):
        nodes[b, :n[b]] = np.sort(rng.choice(S - 1, n[b], replace=False))
    start = rng.integers(0, 9, B).astype(np.int32)
    rows = L + 12
    if kind == "e4m3":
        cache = quant_cache(P, B, rows, H, D)
        parts = (cache.codes, cache.scales)
        want = list(R.quantise(src))
    else:
        cache = torch.full((P, B, rows, H, D), 7.0, dtype=dt, device="cuda")
        parts, want = (cache,), [src]
    before = [p.cpu().clone() for p in parts]
    ctx.cache_write(cache, src.cuda(), torch.from_numpy(n).cuda(), rows=torch.from_numpy(nodes).cuda(),
                    start=torch.from_numpy(start).cuda(), with_root=root)
    for i, (part, old, w) in enumerate(zip(parts, before, want)):
        ref = old.clone()
        for b in range(B):
            pick = ([0] if root else []) + [int(v) + root for v in nodes[b, :n[b]]]
            a = int(start[b])
            if pick:
                ref[:, b, a:a + len(pick)] = w[:, b, pick]
        bits = torch.int16 if kind != "e4m3" else torch.uint8
        got, ref = part.cpu().view(bits), ref.view(bits)
        assert same_codes(got, ref) if kind == "e4m3" and i == 0 else torch.equal(got, ref)
    assert ctx.device_status() == 0
    ctx.close()


def test_rows_outside_source_or_cache_are_skipped_and_reported():
    ctx = context(3, L=4)
    src = special((2, 3, 10, 2, 32), 1)
    nodes = torch.tensor([[0, 99, 3, 4], [1, 2, -5, 2 ** 31 - 1], [0, 1, 2, 3]], dtype=torch.int32)
    start = torch.tensor([0, 1, 6], dtype=torch.int32)
    n = torch.tensor([4, 4, 2 ** 31 - 1], dtype=torch.int32)      # clamped to the list
    cache = quant_cache(2, 3, 8, 2, 32)
    ctx.cache_write(cache, src.cuda(), n.cuda(), rows=nodes.cuda(), start=start.cuda(), with_root=True)
    rc, _ = R.quantise(src)
    ref = torch.full_like(cache.codes.cpu(), 0xA5)
    ref[:, 0, [0, 1, 3, 4]] = rc[:, 0, [0, 1, 4, 5]]
    ref[:, 1, [1, 2, 3]] = rc[:, 1, [0, 2, 3]]
    ref[:, 2, [6, 7]] = rc[:, 2, [0, 1]]
    assert same_codes(cache.codes.cpu(), ref)
    assert ctx.device_status() == 5 and ctx.device_status() == 0
    # starts below the cache and past it
    cache = quant_cache(2, 3, 8, 2, 32)
    ctx.cache_write(cache, src.cuda(), torch.tensor([3, 2, 1], dtype=torch.int32).cuda(),
                    start=torch.tensor([-1, 2 ** 31 - 2, -2 ** 31], dtype=torch.int32).cuda())
    ref = torch.full_like(ref, 0xA5)
    ref[:, 0, [0, 1]] = rc[:, 0, [1, 2]]
    assert same_codes(cache.codes.cpu(), ref)
    assert ctx.device_status() == 5
    out = torch.full((2, 3, 8, 2, 32), 7.0, device="cuda")
    ctx.cache_read(cache, torch.tensor([2, 9, -4], dtype=torch.int32).cuda(),
                   start=torch.tensor([7, 5, 0], dtype=torch.int32).cuda(), out=out)
    assert (out[:, 0, 1:] == 7).all() and (out[:, 1, 3:] == 7).all() and (out[:, 2] == 7).all()
    assert ctx.device_status() == 5
    ctx.close()


def test_strided_sources_and_caches():
    """Keys and values as slices of a fused projection into planes of a wider cache whose rows
    are behind the heads."""
    import paper_2608_20375_amd as G
    ctx = context(2)
    fused = special((1, 2, 12, 3 * 4, 64), 3).cuda()               # q | k | v heads
    src = fused.view(1, 2, 12, 3, 4, 64)[0, :, :, 1:].permute(2, 0, 1, 3, 4)     # 2 planes
    codes = torch.full((2, 2, 4, 20, 64), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, 2, 4, 20), 0xA5, dtype=torch.uint8, device="cuda")
    cache = G.QuantRows(codes.transpose(2, 3), scales.transpose(2, 3))
    n = torch.tensor([12, 7], dtype=torch.int32, device="cuda")
    start = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    ctx.cache_write(cache, src, n, start=start)
    rc, rs = R.quantise(src.cpu().contiguous())
    ref, res = torch.full((2, 2, 20, 4, 64), 0xA5, dtype=torch.uint8), torch.full((2, 2, 20, 4), 0xA5, dtype=torch.uint8)
    for b, (a, m) in enumerate(((3, 12), (0, 7))):
        ref[:, b, a:a + m], res[:, b, a:a + m] = rc[:, b, :m], rs[:, b, :m]
    assert same_codes(cache.codes.cpu(), ref) and torch.equal(cache.scales.cpu(), res)
    out = torch.zeros(2, 2, 4, 12, 64, dtype=torch.bfloat16, device="cuda").transpose(2, 3)
    ctx.cache_read(cache, n, start=start, out=out)
    want = R.values(ref, res)
    for b, (a, m) in enumerate(((3, 12), (0, 7))):
        w, o = want[:, b, a:a + m], out[:, b, :m].cpu().double()
        assert ((o == w) | (torch.isnan(o) & torch.isnan(w))).all()
    ctx.close()


def test_caches_past_32_bit_offsets():
    import paper_2608_20375_amd as G
    ctx = context(2)
    far = 2 ** 31 + 4096
    buf = torch.empty(far + 32 * 64, dtype=torch.uint8, device="cuda")
    codes = buf.as_strided((1, 2, 16, 2, 64), (0, far, 128, 64, 1))
    codes.fill_(0xA5)
    cache = G.QuantRows(codes, torch.zeros(1, 2, 16, 2, dtype=torch.uint8, device="cuda"))
    src = special((1, 2, 9, 2, 64), 4)
    n = torch.tensor([9, 9], dtype=torch.int32, device="cuda")
    start = torch.tensor([1, 7], dtype=torch.int32, device="cuda")
    ctx.cache_write(cache, src.cuda(), n, start=start)
    rc, _ = R.quantise(src)
    got = cache.codes.cpu()
    assert same_codes(got[:, 0, 1:10], rc[:, 0]) and same_codes(got[:, 1, 7:16], rc[:, 1])
    back = ctx.cache_read(cache, n, start=start)[:, 1, :9].cpu().double()
    want = R.values(got[:, 1, 7:16], cache.scales.cpu()[:, 1, 7:16])
    assert ((back == want) | (torch.isnan(back) & torch.isnan(want))).all()
    ctx.close()


def test_graphs_and_streams():
    ctx = context(2)
    src = torch.randn(4, 2, 9, 2, 64, device="cuda").to(torch.bfloat16)
    cache, n = quant_cache(4, 2, 40, 2, 64), torch.tensor([9, 5], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    out = torch.zeros(4, 2, 9, 2, 64, dtype=torch.bfloat16, device="cuda")
    ctx.cache_write(cache, src, n, start=start)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.cache_write(cache, src, n, start=start)
        ctx.cache_read(cache, n, start=start, out=out)
    for _ in range(3):
        src.copy_(torch.randn(4, 2, 9, 2, 64))
        start += 4
        g.replay()
        torch.cuda.synchronize()
        want = R.values(*R.quantise(src.cpu()))
        assert torch.equal(out[:, 0].cpu().double(), want[:, 0])
        assert torch.equal(out[:, 1, :5].cpu().double(), want[:, 1, :5])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        src.copy_(torch.randn(4, 2, 9, 2, 64))
        ctx.cache_write(cache, src, n, start=start)
        ctx.cache_read(cache, n, start=start, out=out)
    torch.cuda.synchronize()
    assert torch.equal(out[:, 0].cpu().double(), R.values(*R.quantise(src.cpu()))[:, 0])
    ctx.close()
