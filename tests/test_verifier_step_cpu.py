"""Refusals of the verifier-side operators, on the CPU: the binding's checks on tensors, and
the C entry points' on sizes and pointers.  A context is the library's, and needs a GPU; the
entry points' checks read only its sizes, which come first in it, so zeroed memory with sizes in
front stands in for one.  Arguments that pass every check end at the device check, which
finds no GPU."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import paper_2608_20375_amd as G  # noqa: E402

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="stands in for a context")


def context(batch=4, L=3, V=100, N=32):
    ctx = G.Context.__new__(G.Context)
    ctx.dims = G.Dims(batch, L, V, 2, N, 4)
    ctx._h = None
    ctx._device = 0
    return ctx


class Fake:
    def __init__(self, batch=4, L=3, V=100, N=32):
        self.mem = C.create_string_buffer(4096)
        C.memmove(self.mem, C.byref(G.Dims(batch, L, V, 2, N, 4)), C.sizeof(G.Dims))
        self.h = C.c_void_p(C.addressof(self.mem))


def rows(scale=False, **kw):
    r = G.Rows(data=1 << 20, plane_stride=1 << 16, batch_stride=1 << 12, row_stride=256, head_stride=64)
    if scale:
        r.scale = 1 << 20
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def attention(**kw):
    a = G.Attention(batch=2, slots=8, with_root=1, q_heads=4, kv_heads=2, head_dim=64, dtype=1,
                    cache_dtype=1, scale=0.125, q=rows(), k=rows(), v=rows(), n_nodes=1 << 20,
                    mask=1 << 20, cache_k=rows(), cache_v=rows(), cache_rows=10, cache_len=1 << 20,
                    shared_k=rows(), shared_v=rows(), shared_len=5, out=rows(), lse=0,
                    workspace=1 << 20, workspace_bytes=1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


NO_GPU = 4        # GRAFT_ERR_HIP: every check before the device's passed


def test_attention_entry_point():
    L, f = G.lib(), Fake()
    run = lambda a: L.graft_tree_attention(f.h, C.byref(a), None)
    assert run(attention()) == NO_GPU
    assert run(attention(mask=0)) == NO_GPU
    assert run(attention(cache_rows=0, cache_len=0, cache_k=G.Rows(), cache_v=G.Rows())) == NO_GPU
    assert run(attention(shared_len=0, shared_k=G.Rows(), shared_v=G.Rows())) == NO_GPU
    assert run(attention(slots=33)) == NO_GPU
    quant = dict(cache_dtype=3, cache_k=rows(True), cache_v=rows(True), shared_k=rows(True),
                 shared_v=rows(True))
    assert run(attention(**quant)) == NO_GPU
    bad = [dict(batch=0), dict(batch=5), dict(slots=0), dict(slots=34), dict(slots=33, with_root=0),
           dict(q_heads=3), dict(kv_heads=0), dict(q_heads=0), dict(head_dim=0), dict(head_dim=72),
           dict(dtype=0), dict(dtype=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
           dict(scale=float("inf")), dict(cache_rows=-1), dict(shared_len=-1), dict(n_nodes=0),
           dict(cache_len=0), dict(q=rows(data=0)), dict(q=rows(data=(1 << 20) + 8)),
           dict(k=rows(row_stride=4)), dict(v=rows(head_stride=-64)), dict(out=rows(data=0)),
           dict(cache_k=rows(data=0)), dict(shared_v=rows(data=0)), dict(cache_v=rows(batch_stride=2)),
           dict(quant, cache_k=rows()), dict(quant, cache_v=rows(True, row_stride=8)),
           dict(quant, shared_k=rows(True, scale_row_stride=-1))]
    for kw in bad:
        assert run(attention(**kw)) == 1, kw
    for kw in (dict(head_dim=144), dict(q_heads=2048, kv_heads=2), dict(cache_dtype=2),
               dict(cache_dtype=3, dtype=2), dict(cache_rows=2 ** 30 + 1), dict(shared_len=2 ** 30 + 1)):
        assert run(attention(**kw)) == 2, kw
    assert L.graft_tree_attention(None, C.byref(attention()), None) == 1
    assert L.graft_tree_attention(f.h, None, None) == 1
    need = C.c_int64(-1)
    big = attention(cache_rows=1 << 20)
    assert L.graft_tree_attention_workspace(f.h, C.byref(big), C.byref(need)) == 0 and need.value > 0
    big.workspace_bytes = need.value - 1
    assert run(attention(cache_rows=1 << 20, workspace_bytes=need.value - 1)) in (1, NO_GPU)
    assert L.graft_tree_attention_workspace(f.h, C.byref(big), None) == 1
    assert b"" != L.graft_last_error()


def test_sampled_walk_entry_point():
    L, f = G.lib(), Fake()
    p = 1 << 20

    def run(ctx=f.h, batch=2, n=p, tok=p, par=p, acc=p, nodes=p, bonus=p, update=0, ws=p, bytes_=1 << 30,
            **kw):
        t = G.TargetLogits(1, p, 100, p, 3300, 100, 32, 0, p)
        for k, v in kw.items():
            setattr(t, k, v)
        return L.graft_accept_sampled(ctx, batch, n, tok, par, C.byref(t), acc, nodes, bonus, None,
                                      update, ws, bytes_, None)

    assert run() == NO_GPU and run(node=0, node_rows=0) == NO_GPU and run(temperature=p) == NO_GPU
    for kw in (dict(ctx=None), dict(batch=0), dict(batch=5), dict(n=None), dict(tok=None), dict(par=None),
               dict(acc=None), dict(nodes=None), dict(bonus=None), dict(update=1), dict(ws=None),
               dict(ws=p + 8), dict(bytes_=10), dict(dtype=3), dict(dtype=-1), dict(root=0), dict(node=0),
               dict(uniform=0), dict(uniform=p + 4), dict(root=p + 1), dict(dtype=0, node=p + 2),
               dict(node_rows=-1), dict(node_rows=33), dict(root_stride=-1), dict(node_row_stride=99)):
        assert run(**kw) == 1, kw
    need = C.c_int64()
    assert L.graft_accept_sampled_workspace(f.h, 4, C.byref(need)) == 0 and need.value > 0
    assert L.graft_accept_sampled_workspace(f.h, 5, C.byref(need)) == 1
    assert L.graft_accept_sampled_workspace(f.h, 1, None) == 1


def move(**kw):
    m = G.CacheMove(2, 3, 2, 64, 1, 3, rows(), rows(True), 9, 20, 1 << 20, 1 << 20, 1 << 20, 3, 1)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


def test_cache_entry_points():
    L, f = G.lib(), Fake()
    write = lambda m: L.graft_cache_write(f.h, C.byref(m), None)
    read = lambda m: L.graft_cache_read(f.h, C.byref(m), None)
    back = dict(src_dtype=3, dst_dtype=1, src=rows(True), dst=rows(), list=0, list_len=0, with_root=0)
    assert write(move()) == NO_GPU and write(move(start=0)) == NO_GPU
    assert write(move(list=0, list_len=0, with_root=0)) == NO_GPU
    for t in (1, 2):
        assert write(move(src_dtype=t, dst_dtype=t, dst=rows())) == NO_GPU
    assert read(move(**back)) == NO_GPU and read(move(**dict(back, dst_dtype=0))) == NO_GPU
    common = [dict(batch=0), dict(batch=5), dict(n_planes=0), dict(heads=0), dict(head_dim=0),
              dict(head_dim=24), dict(src_rows=0), dict(dst_rows=0), dict(n_rows=0)]
    for kw in common + [dict(list_len=0), dict(list=0), dict(src=rows(data=0)),
                        dict(dst=rows(True, data=24)), dict(dst=rows()), dict(src=rows(row_stride=12))]:
        assert write(move(**kw)) == 1, kw
    for kw in common + [dict(list=1 << 20), dict(list_len=2), dict(with_root=1), dict(src=rows())]:
        assert read(move(**dict(back, **kw))) == 1, kw
    for kw in (dict(src_dtype=2), dict(src_dtype=0), dict(dst_dtype=2), dict(head_dim=144),
               dict(src_dtype=0, dst_dtype=0), dict(n_planes=1 << 27, heads=64)):
        assert write(move(**kw)) == 2, kw
    assert read(move(**dict(back, dst_dtype=2))) == 2 and read(move(**dict(back, src_dtype=1))) == 2
    assert L.graft_cache_write(None, C.byref(move()), None) == 1
    assert L.graft_cache_read(f.h, None, None) == 1


def test_cache_sizes_past_32_bits_are_refused():
    """Row numbers of a workgroup's last rows, and products of the sizes, would wrap."""
    L, f = G.lib(), Fake()
    write = lambda m: L.graft_cache_write(f.h, C.byref(m), None)
    read = lambda m: L.graft_cache_read(f.h, C.byref(m), None)
    small = dict(batch=1, n_planes=1, heads=1, head_dim=16)
    back = dict(small, src_dtype=3, dst_dtype=1, src=rows(True), dst=rows(), list=0, list_len=0, with_root=0)
    top = 2 ** 31 - 1
    for kw in (dict(src_rows=top, list=0, list_len=0, with_root=0), dict(dst_rows=top), dict(list_len=top),
               dict(n_planes=top, heads=top), dict(n_planes=1 << 29), dict(heads=1 << 29)):
        assert write(move(**dict(small, **kw))) == 2, kw
    for kw in (dict(src_rows=top), dict(dst_rows=top), dict(n_planes=top, heads=top)):
        assert read(move(**dict(back, **kw))) == 2, kw
    assert read(move(**dict(back, src_rows=1 << 30, dst_rows=1 << 30))) == NO_GPU


def test_binding_refuses_shapes_and_types_before_any_call():
    ctx = context()
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    quant = lambda *s: G.QuantRows(torch.zeros(s, dtype=torch.uint8), torch.zeros(s[:-1], dtype=torch.uint8))
    good = dict(q=bf(2, 8, 4, 64), k=bf(2, 8, 2, 64), v=bf(2, 8, 2, 64), n_nodes=i32(2),
                mask=torch.zeros(2, 32, 1, dtype=torch.int64), cache=(bf(2, 9, 2, 64), bf(2, 9, 2, 64)),
                cache_len=i32(2), shared=(bf(5, 2, 64), bf(5, 2, 64)), with_root=True)
    with pytest.raises(TypeError, match="CUDA"):
        ctx.tree_attention(**good)
    for kw in (dict(q=bf(2, 8, 256)), dict(k=bf(2, 7, 2, 64)), dict(v=bf(2, 8, 2, 48)), dict(n_nodes=None),
               dict(n_nodes=i32(3)), dict(mask=torch.zeros(2, 31, 1, dtype=torch.int64)),
               dict(cache_len=None), dict(cache_len=i32(1)), dict(cache=bf(2, 9, 2, 64)),
               dict(cache=(bf(1, 9, 2, 64), bf(1, 9, 2, 64))), dict(cache=(bf(2, 9, 2, 64), bf(2, 8, 2, 64))),
               dict(cache=(quant(2, 9, 2, 64), bf(2, 9, 2, 64))),
               dict(cache=(quant(2, 9, 2, 64), quant(2, 9, 2, 64))),
               dict(shared=(bf(5, 1, 64), bf(5, 1, 64))), dict(out=bf(2, 8, 4, 32)),
               dict(lse=torch.zeros(2, 8, 2))):
        with pytest.raises(ValueError):
            ctx.tree_attention(**{**good, **kw})
    for kw in (dict(q=torch.zeros(2, 8, 4, 64)), dict(k=torch.zeros(2, 8, 2, 64)),
               dict(cache=(torch.zeros(2, 9, 2, 64), bf(2, 9, 2, 64)))):
        with pytest.raises(TypeError):
            ctx.tree_attention(**{**good, **kw})

    walk = dict(n_nodes=i32(2), tokens=i32(2, 32), parents=i32(2, 32), root_logits=bf(2, 100),
                node_logits=bf(2, 8, 100), uniform=torch.zeros(2, 4, dtype=torch.float64))
    with pytest.raises(TypeError, match="CUDA"):
        ctx.accept_sampled(**walk)
    for kw in (dict(tokens=i32(2, 31)), dict(parents=i32(1, 32)), dict(root_logits=bf(2, 99)),
               dict(node_logits=bf(2, 8, 99)), dict(node_logits=None), dict(uniform=None),
               dict(uniform=torch.zeros(2, 3, dtype=torch.float64)), dict(temperature=torch.zeros(1)),
               dict(acc_nodes=i32(2, 2)), dict(logp=torch.zeros(2, 3)),
               dict(node_logits=bf(2, 100, 8).transpose(1, 2))):
        with pytest.raises(ValueError):
            ctx.accept_sampled(**{**walk, **kw})
    for kw in (dict(root_logits=bf(2, 100).double(), node_logits=bf(2, 8, 100).double()),
               dict(node_logits=bf(2, 8, 100).half())):
        with pytest.raises(TypeError):
            ctx.accept_sampled(**{**walk, **kw})

    w = dict(dst=quant(3, 2, 20, 2, 64), src=bf(3, 2, 9, 2, 64), n_rows=i32(2), rows=i32(2, 4), start=i32(2))
    with pytest.raises(TypeError, match="CUDA"):
        ctx.cache_write(**w)
    for kw in (dict(dst=quant(2, 2, 20, 2, 64)), dict(dst=quant(3, 1, 20, 2, 64)),
               dict(dst=quant(3, 2, 20, 1, 64)), dict(src=bf(3, 2, 9, 2, 32)), dict(src=bf(3, 2, 9, 128)),
               dict(rows=i32(1, 4)), dict(rows=i32(8)), dict(start=i32(1))):
        with pytest.raises(ValueError):
            ctx.cache_write(**{**w, **kw})
    with pytest.raises(TypeError):
        ctx.cache_read(bf(3, 2, 9, 2, 64), i32(2))
    with pytest.raises(TypeError):
        G.QuantRows(bf(3, 2, 64), torch.zeros(3, 2, dtype=torch.uint8))
    with pytest.raises(ValueError):
        G.QuantRows(torch.zeros(3, 2, 64, dtype=torch.uint8), torch.zeros(3, dtype=torch.uint8))


def test_structs_match_the_header(tmp_path):
    import os
    import subprocess
    here = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    pairs = {"graft_rows": G.Rows, "graft_attention": G.Attention, "graft_target_logits": G.TargetLogits,
             "graft_cache_move": G.CacheMove}
    lines = []
    for name, t in pairs.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in t._fields_]
    src = tmp_path / "p.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "graft.h"\nint main(void) {\n%s\nreturn 0; }\n'
                   % "\n".join(lines))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(here, "include"), "-o", str(tmp_path / "p"), str(src)],
                   check=True)
    got = dict(l.split() for l in subprocess.run([str(tmp_path / "p")], capture_output=True, text=True,
                                                 check=True).stdout.splitlines())
    for k, v in got.items():
        t, _, f = k.partition(".")
        assert (getattr(pairs[t], f).offset if f else C.sizeof(pairs[t])) == int(v), k
