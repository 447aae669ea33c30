"""Rotated rows appended to pages (paged_write) against fp64 row by row."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paged_ref as R  # noqa: E402
import paper_2608_20375_amd as G  # noqa: E402

pytestmark = pytest.mark.gpu

BF, FP, Q8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def block(rng, B, S, heads, D, dtype, size=1.0):
    x = torch.from_numpy(rng.standard_normal((B, S, heads, D)) * size)
    return x.to(dtype)


def fill(pool, value):
    if isinstance(pool, G.QuantRows):
        pool.codes.fill_(value)
        pool.scales.fill_(value)
    else:
        pool.fill_(value)


def check(B, S, Hq, H, D, rot, page, dtype=BF, cache=None, axes=0, axis=None, interleaved=False, starts=None, counts=None,
          positions=None, freq=None, seed=0, in_place=False, xs=None):
    """One call, all of its outputs and what it must not touch."""
    rng = np.random.default_rng(seed)
    cache = cache or dtype
    F = rot // 2
    freq = 10000.0 ** -(np.arange(F) / max(1, F)) if freq is None else freq
    starts = np.asarray(starts if starts is not None else rng.integers(0, 3 * page + 2, B), np.int32)
    counts = np.asarray(counts if counts is not None else [S - (S // 3) * (b % 2) for b in range(B)], np.int32)
    t, pages = R.table(rng, page, starts + counts)
    q, k, v = xs or (block(rng, B, S, max(Hq, 1), D, dtype), block(rng, B, S, H, D, dtype, 3.0), block(rng, B, S, H, D, dtype))
    if axes and positions is None:
        positions = rng.integers(0, 50000, (axes, B, S)).astype(np.int32)
    ctx = G.Context(B, 4, 64, 1, 8)
    kp, vp = (G.paged_cache(pages + 2, page, H, D, cache) for _ in range(2))
    fill(kp, 7), fill(vp, 7)
    qd = q.cuda() if Hq else None
    out = qd if in_place else (torch.full_like(qd, 7.0) if Hq else None)
    got = ctx.paged_write((kp, vp), dev(t), k.cuda(), v.cuda(), dev(counts), dev(starts), q=qd, q_out=out,
                          freq=dev(freq) if F else None, positions=None if positions is None else dev(positions),
                          axis=None if axis is None else dev(np.asarray(axis, np.int32)), interleaved=interleaved)
    assert ctx.device_status() == 0
    assert got is out
    eps = 2.0 ** -7 if dtype == BF else 2.0 ** -10
    touched = torch.zeros(pages + 2, page, dtype=torch.bool)
    for b in range(B):
        n = int(counts[b])
        pos = np.arange(S)[None] + starts[b] if positions is None else positions[:, b]
        turn = lambda x: R.rotate(x[b, :n].double(), pos[:, :n], freq, axis, interleaved) if F else (
            x[b, :n].double(), torch.zeros(n, x.shape[2], D, dtype=torch.float64))
        r = np.arange(n) + starts[b]
        pg, of = t[b][r // page].astype(np.int64), r % page
        touched[pg, of] = True
        if Hq:
            y, tol = turn(q)
            assert torch.all((out[b, :n].cpu().double() - y).abs() <= tol + eps / 2 * 1.001 * (y.abs() + tol) + 2.0 ** -25)
            rest = out[b, n:].cpu()
            assert torch.equal(rest, q[b, n:] if in_place else torch.full_like(rest, 7.0))
        y, tol = turn(k)
        if cache != Q8:
            g = kp[pg, of].cpu().double()
            assert torch.all((g - y).abs() <= tol + eps / 2 * 1.001 * (y.abs() + tol) + 2.0 ** -25)
            assert torch.equal(vp[pg, of].cpu(), v[b, :n])
            if not F:
                assert torch.equal(kp[pg, of].cpu(), k[b, :n])
        else:
            codes, scales = R.quantise(v[b, :n])
            assert torch.equal(vp.codes[pg, of].cpu(), codes) and torch.equal(vp.scales[pg, of].cpu(), scales)
            s = kp.scales[pg, of].cpu()
            g = R.values(kp.codes[pg, of].cpu(), s)
            top, unit = y.abs().amax(-1), R.pow2(s.to(torch.int64) - 127)
            slack = tol.amax(-1)
            # 2^e is the smallest that holds the largest number, where fp32 tells
            assert torch.all(top - slack <= 448.0 * unit)
            assert torch.all((top + slack > 224.0 * unit) | (s == 9))
            # half a step of the code, or of the smallest ones
            step = torch.maximum(2.0 ** -4 * (y.abs() + tol), 2.0 ** -10 * unit[..., None])
            assert torch.all((g - y).abs() <= step * 1.0001 + tol)
    left = ~touched
    for p in (kp, vp):
        for x in ((p.codes, p.scales) if cache == Q8 else (p,)):
            assert torch.all(x.cpu()[left] == 7)
    ctx.close()


@pytest.mark.parametrize("D,rot", [(16, 16), (32, 16), (48, 48), (64, 0), (64, 64), (80, 48), (80, 80), (96, 32), (112, 112),
                                   (128, 128), (128, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_sizes(D, rot, interleaved):
    check(3, 7, 6, 2, D, rot, 5, interleaved=interleaved, seed=D + rot)


@pytest.mark.parametrize("dtype,cache", [(BF, BF), (FP, FP), (BF, Q8)])
@pytest.mark.parametrize("D", [16, 48, 64, 80, 128])
def test_types(dtype, cache, D):
    check(2, 19, 4, 4, D, D, 16, dtype=dtype, cache=cache, seed=D)
    check(2, 5, 0, 3, D, D // 32 * 16, 7, dtype=dtype, cache=cache, seed=D + 1, interleaved=True)


@pytest.mark.parametrize("B,S,Hq,H,page", [(1, 1, 32, 8, 16), (1, 1, 1, 1, 1), (4, 1, 8, 1, 64), (2, 65, 32, 8, 64), (1, 300, 5, 5, 24),
                                           (3, 33, 64, 16, 1), (64, 3, 4, 2, 100), (1, 2, 1024, 2, 4)])
def test_shapes(B, S, Hq, H, page):
    check(B, S, Hq, H, 64, 64, page, seed=S + page)
    check(B, S, Hq, H, 32, 32, page, cache=Q8, seed=S + page)


@pytest.mark.parametrize("axes", [1, 2, 3, 8])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes(axes, interleaved):
    axis = [f * axes // 32 for f in range(32)]
    check(2, 11, 4, 2, 80, 64, 8, axes=axes, axis=axis, interleaved=interleaved, seed=axes)
    check(2, 11, 4, 2, 64, 64, 8, axes=axes, axis=[f % axes for f in range(32)], interleaved=interleaved, seed=axes)
    check(2, 11, 4, 2, 64, 64, 8, axes=axes, seed=axes)


def test_far_and_negative_positions():
    """The angle keeps its precision at any 32-bit position."""
    pos = np.array([[[0, 1, -1, 2 ** 20 + 1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 123456789]]], np.int32)
    check(1, 8, 2, 1, 64, 64, 4, positions=pos)
    check(1, 8, 2, 1, 128, 128, 4, positions=pos, dtype=FP, freq=np.linspace(0.0, 6.5, 64))
    check(1, 8, 2, 1, 64, 64, 4, starts=[99991])


def test_quarter_turns():
    """Angles at and beside every eighth of a turn."""
    x = np.concatenate([np.arange(-16, 17) * np.pi / 4 + d for d in (0.0, 1e-9, -1e-9)])
    x = np.concatenate([x, np.zeros(-len(x) % 8)])
    for i in range(0, len(x), 64):
        f = x[i:i + 64]
        f = np.concatenate([f, np.zeros(-len(f) % 8)])
        check(1, 1, 1, 1, 128, 2 * len(f), 1, positions=np.ones((1, 1, 1), np.int32), freq=f, counts=[1], starts=[0], dtype=FP)


def test_counts_and_places():
    check(4, 9, 2, 1, 32, 32, 4, counts=[0, 1, 9, 8], starts=[0, 3, 4, 100])
    check(3, 9, 2, 1, 32, 32, 4, counts=[0, 0, 0], starts=[1, 1, 1])


def test_in_place():
    check(3, 7, 4, 2, 80, 48, 5, in_place=True)
    check(3, 7, 4, 2, 64, 64, 5, in_place=True, interleaved=True, dtype=FP)


def test_scale_borders_and_special_values():
    """Largest numbers at and around 448 2^e, zeros, the smallest numbers, infinities and NaN, in rows
    that are not rotated (bit for bit) and, where a turn by nothing keeps them, rotated by 0."""
    D = 32
    rows = []
    for top in (448.0, 450.0, 446.0, 224.0, 1.75, 1.7578125, 0.0, 1e-38, 2.0 ** -133, 3e38, 1e38, 2.0 ** -110):
        r = torch.zeros(D)
        r[3], r[17] = top, -top / 3
        rows.append(r)
    x = torch.stack(rows).to(BF)[None, :, None].repeat(1, 1, 2, 1)
    y = x.clone()
    y[0, 0, 0, 5], y[0, 1, 0, 6], y[0, 2, 1, 7] = float("inf"), float("-inf"), float("nan")
    y[0, 3, 0, :] = float("nan")
    S = x.shape[1]
    ctx = G.Context(1, 4, 64, 1, 8)
    kp, vp = (G.paged_cache(3, 8, 2, D, Q8) for _ in range(2))
    t = dev(np.array([[2, 0]], np.int32))
    ctx.paged_write((kp, vp), t, y.cuda(), y.cuda())
    r = np.arange(S)
    pg, of = np.array([2, 0])[r // 8], r % 8
    codes, scales = R.quantise(y[0])
    for p in (kp, vp):
        assert torch.equal(p.scales[pg, of].cpu(), scales)
        a, b = p.codes[pg, of].cpu(), codes
        nan = (b & 0x7F) == 0x7F
        assert torch.equal((a & 0x7F)[nan], (b & 0x7F)[nan]) and torch.equal(a[~nan], b[~nan])
    ctx.paged_write((kp, vp), t, x.cuda(), x.cuda(), freq=torch.zeros(16, dtype=torch.float64, device="cuda"))
    codes, scales = R.quantise(x[0])
    assert torch.equal(kp.scales[pg, of].cpu(), scales) and torch.equal(kp.codes[pg, of].cpu() & 0x7F, codes & 0x7F)
    assert ctx.device_status() == 0
    ctx.close()


def test_strided_rows_and_pages():
    """Slices of a fused projection, rows before heads in the pages, keys and values side by side in
    one tensor, heads in front of rows, a page table that is a slice."""
    rng = np.random.default_rng(3)
    B, S, Hq, H, D, page = 2, 6, 4, 2, 64, 4
    fused = torch.from_numpy(rng.standard_normal((B, S, Hq + 2 * H, D))).to(BF).cuda()
    q, k, v = fused[:, :, :Hq], fused[:, :, Hq:Hq + H], fused[:, :, Hq + H:]
    starts, counts = np.array([3, 0], np.int32), np.array([6, 5], np.int32)
    t, pages = R.table(rng, page, starts + counts)
    freq = 10000.0 ** -(np.arange(32) / 32)
    ctx = G.Context(3, 4, 64, 1, 8)
    want = None
    for layout in range(3):
        if layout == 0:
            kp, vp = (torch.zeros(pages, page, H, D, dtype=BF, device="cuda") for _ in range(2))
        elif layout == 1:
            both = torch.zeros(pages, page, 2, H, D, dtype=BF, device="cuda")
            kp, vp = both[:, :, 0], both[:, :, 1]
        else:
            both = torch.zeros(pages, 2, H, page, D + 16, dtype=BF, device="cuda")[..., :D]
            kp, vp = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
        out = torch.zeros(B, Hq, S, D, dtype=BF, device="cuda").transpose(1, 2)
        wide = torch.full((3, t.shape[1]), -5, dtype=torch.int32, device="cuda")
        wide[:2] = dev(t)
        ctx.paged_write((kp, vp), wide, k, v, dev(counts), dev(starts), q=q, q_out=out, freq=dev(freq))
        got = (out.contiguous(), kp.contiguous(), vp.contiguous())
        want = want or got
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert ctx.device_status() == 0
    y, tol = R.rotate(q[0].cpu().double(), np.arange(6)[None] + 3, freq)
    assert torch.all((want[0][0].cpu().double() - y).abs() <= tol + 2.0 ** -8 * 1.001 * (y.abs() + tol))
    ctx.close()


def test_rows_without_a_place_are_reported():
    """Cache rows past the table, negative ones, pages that the pool does not have: nothing is
    written for them, the queries are rotated all the same."""
    D, page = 32, 4
    k = torch.ones(4, 6, 1, D, dtype=BF, device="cuda")
    freq = torch.zeros(16, dtype=torch.float64, device="cuda")
    cases = [([0, 0, 0, 0], [[0, 1], [2, -1], [7, 3], [4, 5]], [6, 4, 6, 6], {2: range(4)}),   # page 7 of 6
             ([0, 6, -2, 8], [[0, 1], [2, 3], [4, 5], [1, 1]], [6, 2, 6, 2], {2: (0, 1), 3: (0, 1)})]
    for starts, t, counts, lost in cases:
        ctx = G.Context(4, 4, 64, 1, 8)
        kp, vp = (torch.zeros(6, page, 1, D, dtype=BF, device="cuda") for _ in range(2))
        out = ctx.paged_write((kp, vp), dev(np.array(t, np.int32)), k, k, dev(np.array(counts, np.int32)),
                              dev(np.array(starts, np.int32)), q=k, freq=freq)
        assert ctx.device_status() != 0 and ctx.device_status() == 0
        want = torch.zeros(6, page)
        for b in range(4):
            for i in range(counts[b]):
                if i not in lost.get(b, ()):
                    r = starts[b] + i
                    want[t[b][r // page], r % page] = 1
            assert torch.all(out[b, :counts[b]] == 1) and torch.all(out[b, counts[b]:] == 0)
        for p in (kp, vp):
            assert torch.equal(p[:, :, 0, 0].float().cpu(), want) and torch.equal(p[:, :, 0, D - 1].float().cpu(), want)
        ctx.close()


def test_counts_and_axes_outside_are_reported():
    ctx = G.Context(2, 4, 64, 1, 8)
    k = torch.ones(2, 3, 1, 32, dtype=BF, device="cuda")
    pools = tuple(torch.zeros(4, 4, 1, 32, dtype=BF, device="cuda") for _ in range(2))
    t = dev(np.array([[0, 1], [2, 3]], np.int32))
    ctx.paged_write(pools, t, k, k, dev(np.array([-1, 4], np.int32)))
    assert ctx.device_status() != 0
    assert pools[0][:2].abs().sum() == 0 and torch.all(pools[0][2, :3] == 1) and torch.all(pools[0][2, 3] == 0)
    freq = torch.ones(16, dtype=torch.float64, device="cuda")
    pos = torch.zeros(2, 2, 3, dtype=torch.int32, device="cuda")
    axis = torch.zeros(16, dtype=torch.int32, device="cuda")
    axis[5], axis[6] = 2, -1
    ctx.paged_write(pools, t, k, k, freq=freq, positions=pos, axis=axis)
    assert ctx.device_status() != 0
    assert torch.all(pools[0][0, :3] == 1)         # taken as axis 0: position 0
    ctx.close()


def test_pages_past_32_bit_offsets():
    """A pool of more than 2^32 bytes: the last pages."""
    H, D, page = 8, 128, 1024
    pages = (1 << 32) // (page * H * D * 2) + 64
    kp = torch.zeros(pages, page, H, D, dtype=BF, device="cuda")
    ctx = G.Context(1, 4, 64, 1, 8)
    x = torch.randn(1, 4, H, D, device="cuda").to(BF)
    t = torch.full((1, 3), -1, dtype=torch.int32, device="cuda")
    t[0, 1], t[0, 2] = pages - 1, pages - 2
    vp = torch.zeros_like(kp)
    ctx.paged_write((kp, vp), t, x, x, start=dev(np.array([2 * page - 2], np.int32)))
    assert ctx.device_status() == 0
    for p in (kp, vp):
        assert torch.equal(p[pages - 1, page - 2:], x[0, :2]) and torch.equal(p[pages - 2, :2], x[0, 2:])
        assert int(torch.count_nonzero(p[:pages - 2])) == 0
    ctx.close()


def test_calls_on_side_streams_and_in_graphs():
    """Writes to pages of their own on two streams at once; a captured write follows its inputs' memory."""
    rng = np.random.default_rng(6)
    D, page = 64, 16
    freq = dev(10.0 ** -np.linspace(0, 4, 32))
    runs = []
    for i in range(2):
        ctx = G.Context(2, 4, 64, 1, 8)
        kv = tuple(torch.zeros(6, page, 2, D, dtype=BF, device="cuda") for _ in range(2))
        x = [block(rng, 2, 20, h, D, BF).cuda() for h in (2, 2, 4)]
        t = dev(rng.permutation(6).astype(np.int32).reshape(2, 3))
        start = dev(np.array([3 + i, 20], np.int32))
        runs.append((ctx, kv, x, t, start, torch.zeros_like(x[2]), torch.cuda.Stream()))
    call = lambda r: r[0].paged_write(r[1], r[3], r[2][0], r[2][1], start=r[4], q=r[2][2], q_out=r[5], freq=freq)
    torch.cuda.synchronize()
    for r in runs:
        with torch.cuda.stream(r[6]):
            call(r)
    torch.cuda.synchronize()
    for r in runs:
        got = [x.clone() for x in (*r[1], r[5])]
        for x in (*r[1], r[5]):
            x.zero_()
        call(r)
        assert all(torch.equal(a, b) for a, b in zip(got, (*r[1], r[5]))) and got[0].abs().sum() > 0
    r = runs[0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(r)
    for s in ([0, 5], [28, 1], [9, 9]):
        r[4].copy_(dev(np.array(s, np.int32)))
        r[2][0].copy_(block(rng, 2, 20, 2, D, BF))
        for x in (*r[1], r[5]):
            x.zero_()
        call(r)
        eager = [x.clone() for x in (*r[1], r[5])]
        for x in (*r[1], r[5]):
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (*r[1], r[5])))
    for r in runs:
        assert r[0].device_status() == 0
        r[0].close()


def test_codes_match_the_contiguous_cache():
    """Rows that are not rotated get the codes and scales of cache_write."""
    rng = np.random.default_rng(8)
    k = block(rng, 2, 21, 3, 80, BF, 3.0).cuda()
    ctx = G.Context(2, 4, 64, 1, 8)
    flat = G.QuantRows.empty(1, 2, 24, 3, 80)
    n = dev(np.array([21, 10], np.int32))
    ctx.cache_write(flat, k[None], n)
    kp, vp = (G.paged_cache(6, 8, 3, 80, Q8) for _ in range(2))
    ctx.paged_write((kp, vp), dev(np.array([[5, 0, 3], [1, 2, 4]], np.int32)), k, k, n)
    for b, pages in ((0, (5, 0, 3)), (1, (1, 2, 4))):
        m = int(n[b])
        for p in (kp, vp):
            for x, y in ((p.codes, flat.codes), (p.scales, flat.scales)):
                assert torch.equal(torch.cat([x[i] for i in pages])[:m], y[0, b, :m])
    ctx.close()
