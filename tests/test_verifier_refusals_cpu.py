"""More refusals of the verifier-side operators, on the CPU, by test_verifier_step_cpu's stand-ins for
a context."""
import ctypes as C
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_20375_amd as G  # noqa: E402
from test_verifier_step_cpu import NO_GPU, Fake, attention, context, move, rows  # noqa: E402

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="stands in for a context")


def bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


def quant(*s):
    return G.QuantRows(torch.zeros(s, dtype=torch.uint8), torch.zeros(s[:-1], dtype=torch.uint8))


def block(**kw):
    a = dict(q=bf(2, 8, 4, 64), k=bf(2, 8, 2, 64), v=bf(2, 8, 2, 64), n_nodes=i32(2),
             mask=torch.zeros(2, 32, 1, dtype=torch.int64), cache=(bf(2, 9, 2, 64), bf(2, 9, 2, 64)),
             cache_len=i32(2), shared=(bf(5, 2, 64), bf(5, 2, 64)), with_root=True)
    a.update(kw)
    return a


def test_entry_points_refuse_rows_written_twice():
    L, f = G.lib(), Fake()
    attend = lambda **kw: L.graft_tree_attention(f.h, C.byref(attention(**kw)), None)
    write = lambda **kw: L.graft_cache_write(f.h, C.byref(move(**kw)), None)
    back = dict(src_dtype=3, dst_dtype=1, src=rows(True), dst=rows(), list=0, list_len=0, with_root=0)
    read = lambda **kw: L.graft_cache_read(f.h, C.byref(move(**dict(back, **kw))), None)
    for name in ("batch_stride", "row_stride", "head_stride"):
        for stride in (0, 16, 48):
            assert attend(out=rows(**{name: stride})) == 1, (name, stride)
    assert attend(out=rows(plane_stride=0)) == NO_GPU            # not used
    assert attend(out=rows(batch_stride=0), batch=1) == NO_GPU   # one entry
    for name in ("plane_stride", "batch_stride", "row_stride", "head_stride"):
        for stride in (0, 16, 48):
            assert write(dst=rows(True, **{name: stride})) == 1, (name, stride)
            assert write(dst_dtype=1, dst=rows(**{name: stride})) == 1, (name, stride)
            assert read(dst=rows(**{name: stride})) == 1, (name, stride)
            # what is read may repeat
            assert write(src=rows(**{name: stride})) == NO_GPU, (name, stride)
    assert write(dst=rows(True, plane_stride=0), n_planes=1) == NO_GPU


def test_scale_strides_of_other_types_are_ignored():
    L, f = G.lib(), Fake()
    attend = lambda **kw: L.graft_tree_attention(f.h, C.byref(attention(**kw)), None)
    for stride in (1 << 40, -1):
        far = rows(scale_row_stride=stride, scale_head_stride=stride, scale_batch_stride=stride)
        for name in ("q", "k", "v", "cache_k", "cache_v", "shared_k", "shared_v", "out"):
            assert attend(**{name: far}) == NO_GPU, (name, stride)
    codes = dict(cache_dtype=3, cache_k=rows(True), cache_v=rows(True), shared_k=rows(True), shared_v=rows(True))
    for name in ("cache_k", "cache_v", "shared_k", "shared_v"):
        assert attend(**{**codes, name: rows(True, scale_row_stride=(1 << 22) + 1)}) == 2, name
        assert attend(**{**codes, name: rows(True, scale_row_stride=1 << 22)}) == NO_GPU, name


def test_scales_past_the_exponent_are_refused():
    """scale log2 e would be infinite, and every result NaN."""
    L, f = G.lib(), Fake()
    attend = lambda s: L.graft_tree_attention(f.h, C.byref(attention(scale=s)), None)
    assert attend(1e38) == NO_GPU and attend(1e-38) == NO_GPU
    assert attend(2.4e38) == 2 and attend(3.4e38) == 2


def test_binding_refuses_tensors_written_twice():
    ctx = context()
    for out in (bf(1, 8, 4, 64).expand(2, 8, 4, 64), bf(2, 1, 4, 64).expand(2, 8, 4, 64),
                bf(2, 8, 1, 64).expand(2, 8, 4, 64), bf(2, 8, 4, 1).expand(2, 8, 4, 64),
                bf(4096).as_strided((2, 8, 4, 64), (1024, 128, 64, 1))):
        with pytest.raises(ValueError, match="overlap"):
            ctx.tree_attention(**block(out=out))
    w = dict(dst=quant(3, 2, 20, 2, 64), src=bf(3, 2, 9, 2, 64), n_rows=i32(2), rows=i32(2, 4), start=i32(2))
    codes, scales = w["dst"].codes, w["dst"].scales
    for dst in (G.QuantRows(codes[:1].expand(3, -1, -1, -1, -1), scales),
                G.QuantRows(codes, scales[:, :1].expand(-1, 2, -1, -1)),
                G.QuantRows(codes, scales.flatten().as_strided((3, 2, 20, 2), (80, 40, 1, 1))),
                bf(3, 1, 20, 2, 64).expand(3, 2, 20, 2, 64), bf(3, 2, 1, 2, 64).expand(3, 2, 20, 2, 64)):
        with pytest.raises(ValueError, match="overlap"):
            ctx.cache_write(**{**w, "dst": dst})
    with pytest.raises(ValueError, match="overlap"):
        ctx.cache_read(quant(3, 2, 20, 2, 64), i32(2), out=bf(1, 2, 20, 2, 64).expand(3, 2, 20, 2, 64))
    # views without overlap, and tensors that are read, pass on to the device's check
    with pytest.raises(TypeError, match="CUDA"):
        ctx.tree_attention(**block(out=bf(2, 8, 4, 80)[..., :64]))
    with pytest.raises(TypeError, match="CUDA"):
        ctx.tree_attention(**block(out=bf(2, 4, 8, 64).transpose(1, 2), q=bf(1, 8, 4, 64).expand(2, 8, 4, 64)))
    with pytest.raises(TypeError, match="CUDA"):
        ctx.cache_write(**{**w, "dst": G.QuantRows(quant(3, 2, 2, 20, 64).codes.transpose(2, 3),
                                                   quant(3, 2, 2, 20, 64).scales.transpose(2, 3))})


def test_binding_refuses_extents_past_32_bits():
    """The library's sizes are 32-bit numbers: 2^32 + 9 rows must not become 9, nor 2^32 none."""
    ctx = context()
    for n in (2 ** 31, 2 ** 32, 2 ** 32 + 9):
        far = lambda *lead: bf(*[1] * len(lead), 2, 64).expand(*lead, 2, 64)
        every = lambda *lead: G.QuantRows(torch.zeros(1, dtype=torch.uint8).expand(*lead, 2, 64),
                                          torch.zeros(1, dtype=torch.uint8).expand(*lead, 2))
        for kw in (dict(cache=(far(2, n), far(2, n))), dict(shared=(far(n), far(n))),
                   dict(cache=(every(2, n), every(2, n)), shared=None),
                   dict(cache=(far(2, n), torch.nn.Parameter(far(2, n))), shared=None),
                   dict(q=bf(1).expand(2, n, 4, 64), k=far(2, n), v=far(2, n)),
                   dict(q=bf(1).expand(2, 8, n, 64)),
                   dict(k=bf(1).expand(2, 8, n, 64), v=bf(1).expand(2, 8, n, 64)),
                   ):
            with pytest.raises(ValueError, match="past 2"):
                ctx.tree_attention(**block(**kw))
        w = dict(dst=quant(3, 2, 20, 2, 64), src=bf(3, 2, 9, 2, 64), n_rows=i32(2), rows=i32(2, 4), start=i32(2))
        for kw in (dict(src=far(3, 2, n)), dict(dst=every(3, 2, n)), dict(rows=i32(1, 1).expand(2, n)),
                   dict(n_rows=i32(1).expand(n)), dict(src=far(n, 2, 9), dst=every(n, 2, 20))):
            with pytest.raises(ValueError, match="past 2"):
                ctx.cache_write(**{**w, **kw})
        with pytest.raises(ValueError, match="past 2"):
            ctx.cache_read(every(3, 2, n), i32(2), out=bf(3, 2, 9, 2, 64))
        with pytest.raises(ValueError, match="past 2"):
            ctx.accept_sampled(i32(1).expand(n), i32(2, 32), i32(2, 32), bf(2, 100), bf(2, 8, 100),
                               torch.zeros(2, 4, dtype=torch.float64))


def test_calls_past_a_launch_are_refused():
    """A launch counts its threads in 32 bits: 2^24 - 1 workgroups of 256."""
    L, f = G.lib(), Fake(batch=1 << 24, L=1, N=8)
    attend = lambda **kw: L.graft_tree_attention(f.h, C.byref(attention(**{**big, **kw})), None)
    # single tokens: a workgroup a sequence and key head, sequences in an odd number, then eights
    big = dict(slots=1, with_root=1, q_heads=8, kv_heads=8, shared_len=0, workspace_bytes=1 << 60, out=rows(),
               batch=(1 << 21) - 16)
    assert attend() == NO_GPU and attend(batch=1 << 21) == 2 and attend(batch=1 << 24) == 2
    # four rows of the merge a workgroup; the shared prefix has a pass of its own
    big.update(slots=8, with_root=0, q_heads=8, kv_heads=1, shared_len=5, batch=(1 << 20) - 1)
    assert attend() == NO_GPU and attend(batch=1 << 20) == 2
    t = G.TargetLogits(1, 1 << 20, 100, 0, 0, 0, 0, 0, 1 << 20)
    p = 1 << 20
    walk = lambda batch: L.graft_accept_sampled(f.h, batch, p, p, p, C.byref(t), p, p, p, None, 0, p, 1 << 60, None)
    assert walk((1 << 24) - 1) == NO_GPU and walk(1 << 24) == 2
    m = dict(batch=1, n_planes=1, heads=1, head_dim=128, list=0, list_len=0, with_root=0)
    write = lambda **kw: L.graft_cache_write(f.h, C.byref(move(**{**m, **kw})), None)
    # 16 threads a row, four rows each: 64 rows a workgroup
    assert write(src_rows=1 << 30) == 2 and write(src_rows=(1 << 30) - 64) == NO_GPU
    assert write(src_rows=1 << 20, batch=1 << 10) == 2 and write(src_rows=1 << 20, batch=1 << 9) == NO_GPU
    back = dict(src_dtype=3, dst_dtype=1, src=rows(True), dst=rows())
    read = lambda **kw: L.graft_cache_read(f.h, C.byref(move(**{**m, **back, **kw})), None)
    assert read(dst_rows=1 << 30) == 2 and read(dst_rows=(1 << 30) - 64) == NO_GPU
    assert read(dst_rows=1 << 30, dst_dtype=0) == 2 and read(dst_rows=1 << 28, dst_dtype=0) == NO_GPU
