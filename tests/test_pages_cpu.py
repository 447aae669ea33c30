"""Pages on the CPU: pages.h on the host, the refusals of the library and of the binding, and the
structs' layout against the header.  Contexts are test_verifier_step_cpu's stand-ins."""
import ctypes as C
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_20375_amd as G  # noqa: E402
from test_verifier_step_cpu import NO_GPU, Fake, context, rows  # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="stands in for a context")


def test_pages_on_the_host(tmp_path):
    exe = tmp_path / "pages"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2608_20375_amd", "csrc"), "-o", str(exe),
                    os.path.join(HERE, "pages_driver.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


def test_struct_layouts(tmp_path):
    pairs = {"graft_page_table": G.PageTable, "graft_paged_rows": G.PagedRows,
             "graft_paged_attention_desc": G.PagedAttention, "graft_paged_path": G.PagedPath}
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "graft.h"', 'int main(void) {']
    for name, t in pairs.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in t._fields_]
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    for k, v in (line.split() for line in out.splitlines()):
        t, _, f = k.partition(".")
        assert (getattr(pairs[t], f).offset if f else C.sizeof(pairs[t])) == int(v), k


def pages(**kw):
    t = G.PageTable(1 << 20, 8, 8, 40, 16)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def make(cls, **base):
    def f(**kw):
        return cls(**{**base, **kw})
    return f


page = lambda scale=False, **kw: rows(scale, **{**dict(batch_stride=1 << 12, row_stride=128, head_stride=64), **kw})
write = make(G.PagedRows, batch=2, slots=8, q_heads=4, kv_heads=2, head_dim=64, rot_dim=64, interleaved=0, dtype=1, cache_dtype=1,
             q=rows(), q_out=rows(), k=rows(), v=rows(), cache_k=page(), cache_v=page(), pages=pages(), n_rows=0, start=0,
             positions=0, axes=0, axis=0, freq=1 << 20)
attend = make(G.PagedAttention, batch=2, slots=8, with_root=1, q_heads=4, kv_heads=2, head_dim=64, dtype=1, cache_dtype=1, scale=0.125,
              window=0, sinks=0, q=rows(), n_nodes=1 << 20, mask=1 << 20, cache_k=page(), cache_v=page(), pages=pages(),
              cache_len=1 << 20, out=rows(), lse=0, workspace=1 << 20, workspace_bytes=1 << 40)
path = make(G.PagedPath, batch=2, n_planes=3, heads=2, head_dim=64, dtype=1, rows=page(plane_stride=1 << 20), pages=pages(), start=0,
            acc_len=1 << 20, acc_nodes=1 << 20, with_root=1)
TABLES = [(1, dict(table=0)), (1, dict(table_len=0)), (1, dict(pages=0)), (1, dict(page_rows=0)), (1, dict(table_stride=-1)),
          (2, dict(pages=(1 << 30) + 1)), (2, dict(page_rows=(1 << 20) + 1)), (2, dict(table_len=(1 << 26) + 1))]


@no_gpu
def test_write_entry_point():
    L, f = G.lib(), Fake()
    run = lambda a: L.graft_paged_write(f.h, C.byref(a), None)
    q8 = dict(cache_dtype=3, cache_k=page(True), cache_v=page(True))
    for kw in ({}, dict(q_heads=0, q=G.Rows(), q_out=G.Rows()), dict(n_rows=1 << 20, start=1 << 20), dict(rot_dim=0, freq=0), q8,
               dict(positions=1 << 20, axes=3, axis=1 << 20), dict(positions=1 << 20, axes=8), dict(dtype=2, cache_dtype=2),
               dict(rot_dim=16, interleaved=1), dict(slots=1 << 20), dict(axes=99)):
        assert run(write(**kw)) == NO_GPU, kw
    for kw in (dict(batch=0), dict(batch=5), dict(slots=0), dict(q_heads=-1), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=72),
               dict(rot_dim=-16), dict(rot_dim=80), dict(rot_dim=8), dict(dtype=0), dict(dtype=3), dict(freq=0), dict(freq=(1 << 20) + 4),
               dict(positions=1 << 20, axes=0), dict(positions=1 << 20, axes=9), dict(axis=1 << 20), dict(q=rows(data=0)),
               dict(q_out=rows(data=(1 << 20) + 2)), dict(k=rows(row_stride=4)), dict(v=rows(data=0)), dict(q_out=rows(head_stride=32)),
               dict(cache_k=page(row_stride=0)), dict(cache_v=page(batch_stride=16)), dict(cache_k=page(data=0)),
               dict(q8, cache_k=page()), dict(q8, cache_v=page(True, row_stride=8)), dict(q8, cache_v=page(True, scale_row_stride=-1))):
        assert run(write(**kw)) == 1, kw
    for kw in (dict(head_dim=144), dict(q_heads=1025), dict(kv_heads=1025), dict(cache_dtype=2), dict(cache_dtype=3, dtype=2),
               dict(slots=(1 << 24) + 1), dict(cache_k=page(row_stride=1 << 31)),
               dict(q8, cache_k=page(True, scale_row_stride=1 << 30)), dict(slots=1 << 24, q_heads=1024)):
        assert run(write(**kw)) == 2, kw
    for rc, kw in TABLES:
        assert run(write(pages=pages(**kw))) == rc, kw
    assert L.graft_paged_write(None, C.byref(write()), None) == 1 and L.graft_paged_write(f.h, None, None) == 1


@no_gpu
def test_attention_entry_point():
    L, f = G.lib(), Fake()
    run = lambda a: L.graft_paged_attention(f.h, C.byref(a), None)
    q8 = dict(cache_dtype=3, cache_k=page(True), cache_v=page(True))
    for kw in ({}, dict(mask=0), dict(mask=0, n_nodes=0, slots=128, with_root=0), dict(slots=33), q8, dict(window=4, sinks=9),
               dict(mask=0, window=1), dict(dtype=2, cache_dtype=2), dict(scale=1e38), dict(cache_k=page(row_stride=0)),
               dict(pages=pages(table_stride=0))):
        assert run(attend(**kw)) == NO_GPU, kw
    for kw in (dict(batch=0), dict(batch=5), dict(slots=0), dict(slots=34), dict(slots=33, with_root=0), dict(q_heads=3),
               dict(q_heads=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=40), dict(dtype=0), dict(dtype=3), dict(scale=0.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-1.0), dict(window=-1), dict(sinks=-1), dict(window=3),
               dict(cache_len=0), dict(q=rows(data=0)), dict(out=rows(data=0)), dict(out=rows(row_stride=0)), dict(q=rows(batch_stride=4)),
               dict(cache_k=page(data=0)), dict(cache_v=page(data=(1 << 20) + 8)), dict(q8, cache_k=page()),
               dict(mask=0, slots=129), dict(pages=pages(table_len=1, page_rows=7))):
        assert run(attend(**kw)) == 1, kw
    for kw in (dict(head_dim=144), dict(q_heads=2048), dict(cache_dtype=2), dict(cache_dtype=3, dtype=2), dict(scale=2e38),
               dict(cache_v=page(head_stride=1 << 31)), dict(mask=0, slots=(1 << 20) + 1), dict(mask=0, slots=1 << 20, q_heads=1024)):
        assert run(attend(**kw)) == 2, kw
    for rc, kw in TABLES:
        assert run(attend(pages=pages(**kw))) == rc, kw
    need = C.c_int64(-1)
    long = attend(slots=1, pages=pages(table_len=1 << 16))
    assert L.graft_paged_attention_workspace(f.h, C.byref(long), C.byref(need)) == 0 and need.value >= 0
    if need.value:
        long.workspace_bytes = need.value - 1
        assert run(long) in (1, NO_GPU)         # the device is looked at first
    assert L.graft_paged_attention_workspace(f.h, C.byref(long), None) == 1
    assert L.graft_paged_attention_workspace(None, C.byref(long), C.byref(need)) == 1
    assert L.graft_paged_attention(None, C.byref(attend()), None) == 1 and L.graft_paged_attention(f.h, None, None) == 1


@no_gpu
def test_commit_entry_point():
    L, f = G.lib(), Fake()
    run = lambda a: L.graft_paged_commit(f.h, C.byref(a), None)
    q8 = dict(dtype=3, rows=page(True, plane_stride=1 << 20))
    for kw in ({}, q8, dict(start=1 << 20), dict(dtype=2), dict(with_root=0), dict(n_planes=1, rows=page(plane_stride=0))):
        assert run(path(**kw)) == NO_GPU, kw
    for kw in (dict(batch=0), dict(batch=5), dict(n_planes=0), dict(heads=0), dict(head_dim=8), dict(dtype=0), dict(dtype=4),
               dict(acc_len=0), dict(acc_nodes=0), dict(rows=page(data=0)), dict(rows=page(plane_stride=0)),
               dict(rows=page(plane_stride=1 << 20, row_stride=16)), dict(dtype=3), dict(rows=page(plane_stride=1 << 20, head_stride=4))):
        assert run(path(**kw)) == 1, kw
    for kw in (dict(head_dim=144), dict(heads=1025), dict(n_planes=(1 << 20) + 1), dict(n_planes=1 << 20, heads=1024)):
        assert run(path(**kw)) == 2, kw
    for rc, kw in TABLES:
        assert run(path(pages=pages(**kw))) == rc, kw
    assert L.graft_paged_commit(None, C.byref(path()), None) == 1 and L.graft_paged_commit(f.h, None, None) == 1


def bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


def quant(*s):
    return G.QuantRows(torch.zeros(s, dtype=torch.uint8), torch.zeros(s[:-1], dtype=torch.uint8))


f64 = lambda *s: torch.zeros(*s, dtype=torch.float64)


@no_gpu
def test_binding_of_the_write():
    ctx = context()
    good = dict(cache=(bf(9, 4, 2, 64), bf(9, 4, 2, 64)), page_table=i32(2, 5), k=bf(2, 8, 2, 64), v=bf(2, 8, 2, 64), n_rows=i32(2),
                start=i32(2), q=bf(2, 8, 4, 64), q_out=bf(2, 8, 4, 64), freq=f64(32), positions=i32(3, 2, 8), axis=i32(32))
    for kw in ({}, dict(q=None, q_out=None), dict(q_out=None), dict(positions=i32(2, 8)), dict(axis=None), dict(n_rows=None, start=None),
               dict(cache=(quant(9, 4, 2, 64), quant(9, 4, 2, 64))), dict(freq=f64(8), axis=None), dict(page_table=i32(3, 5)),
               dict(freq=None, positions=None, axis=None)):
        with pytest.raises(TypeError, match="CUDA"):
            ctx.paged_write(**{**good, **kw})
    for kw in (dict(k=bf(8, 2, 64)), dict(v=bf(2, 8, 2, 32)), dict(q=bf(2, 7, 4, 64)), dict(q_out=bf(2, 8, 5, 64)), dict(q=None),
               dict(cache=bf(9, 4, 2, 64)), dict(cache=(bf(9, 4, 2, 64), bf(9, 5, 2, 64))), dict(cache=(bf(9, 4, 3, 64), bf(9, 4, 3, 64))),
               dict(cache=(bf(9, 4, 2, 64), quant(9, 4, 2, 64))), dict(page_table=i32(1, 5)), dict(page_table=i32(5)), dict(page_table=None),
               dict(page_table=i32(2, 0)), dict(n_rows=i32(3)), dict(start=i32(1)), dict(freq=f64(33)), dict(freq=f64(0)),
               dict(freq=f64(4, 8)), dict(freq=None), dict(positions=i32(8)), dict(positions=i32(3, 2, 9)), dict(positions=None),
               dict(axis=i32(31)), dict(k=bf(2, 0, 2, 64)),
               dict(cache=(bf(9, 4, 1, 64).expand(9, 4, 2, 64), bf(9, 4, 2, 64))), dict(cache=(bf(9, 4, 2, 64), bf(1, 4, 2, 64).expand(9, 4, 2, 64))),
               dict(q_out=bf(1, 8, 4, 64).expand(2, 8, 4, 64))):
        with pytest.raises(ValueError):
            ctx.paged_write(**{**good, **kw})
    for kw in (dict(k=bf(2, 8, 2, 64).float()), dict(v=bf(2, 8, 2, 64).half()), dict(q=bf(2, 8, 4, 64).half()), dict(freq=f64(32).float()),
               dict(cache=(bf(9, 4, 2, 64).half(), bf(9, 4, 2, 64).half())), dict(page_table=i32(2, 5).long()), dict(cache=(1, 2))):
        with pytest.raises(TypeError):
            ctx.paged_write(**{**good, **kw})


@no_gpu
def test_binding_of_the_attention():
    ctx = context()
    good = dict(q=bf(2, 8, 4, 64), cache=(bf(9, 4, 2, 64), bf(9, 4, 2, 64)), page_table=i32(2, 5), cache_len=i32(2), n_nodes=i32(2),
                mask=torch.zeros(2, 32, 1, dtype=torch.int64), window=9, sinks=1, with_root=True, out=bf(2, 8, 4, 64),
                lse=torch.zeros(2, 8, 4))
    for kw in ({}, dict(n_nodes=None, mask=None), dict(window=None), dict(out=None, lse=None), dict(cache=(quant(9, 4, 2, 64),) * 2),
               dict(q=bf(2, 4, 8, 64).transpose(1, 2)), dict(mask=torch.zeros(3, 32, 1, dtype=torch.int64))):
        with pytest.raises(TypeError, match="CUDA"):
            ctx.paged_attention(**{**good, **kw})
    for kw in (dict(q=bf(8, 4, 64)), dict(cache=(bf(9, 4, 2, 64), bf(8, 4, 2, 64))), dict(cache=(bf(9, 4, 2, 32), bf(9, 4, 2, 32))),
               dict(cache=None), dict(page_table=i32(1, 5)), dict(cache_len=None), dict(cache_len=i32(3)), dict(n_nodes=i32(1)),
               dict(mask=torch.zeros(2, 31, 1, dtype=torch.int64)), dict(window=0), dict(window=-3), dict(window=2 ** 31), dict(sinks=-1),
               dict(sinks=2 ** 31), dict(out=bf(2, 8, 4, 32)), dict(out=bf(1, 8, 4, 64).expand(2, 8, 4, 64)), dict(lse=torch.zeros(2, 8))):
        with pytest.raises(ValueError):
            ctx.paged_attention(**{**good, **kw})
    for kw in (dict(q=bf(2, 8, 4, 64).float()), dict(cache=(bf(9, 4, 2, 64).half(),) * 2), dict(cache_len=i32(2).long()),
               dict(out=bf(2, 8, 4, 64).half()), dict(mask=i32(2, 32, 1)), dict(cache=(3, 4))):
        with pytest.raises(TypeError):
            ctx.paged_attention(**{**good, **kw})


@no_gpu
def test_binding_of_the_commit():
    ctx = context()
    good = dict(cache=bf(3, 9, 4, 2, 64), page_table=i32(2, 5), start=i32(2), acc_len=i32(2), acc_nodes=i32(2, 3))
    for kw in ({}, dict(cache=quant(3, 9, 4, 2, 64)), dict(start=None), dict(with_root=True), dict(acc_nodes=i32(4, 3))):
        with pytest.raises(TypeError, match="CUDA"):
            ctx.paged_commit(**{**good, **kw})
    for kw in (dict(cache=bf(9, 4, 2, 64)), dict(page_table=i32(1, 5)), dict(start=i32(1)), dict(acc_nodes=i32(2, 4)), dict(acc_nodes=None),
               dict(acc_len=None), dict(cache=bf(1, 9, 4, 2, 64).expand(3, 9, 4, 2, 64)), dict(cache=bf(3, 9, 4, 0, 64))):
        with pytest.raises(ValueError):
            ctx.paged_commit(**{**good, **kw})
    for kw in (dict(cache=[1]), dict(acc_len=i32(2).long()), dict(page_table=i32(2, 5).long())):
        with pytest.raises(TypeError):
            ctx.paged_commit(**{**good, **kw})


@no_gpu
def test_binding_refuses_extents_past_32_bits():
    ctx = context()
    n = 2 ** 32 + 2
    for call in (lambda: ctx.paged_write((bf(1).expand(n, 4, 2, 64),) * 2, i32(2, 5), bf(2, 8, 2, 64), bf(2, 8, 2, 64)),
                 lambda: ctx.paged_write((bf(9, 4, 2, 64),) * 2, i32(1).expand(2, n), bf(2, 8, 2, 64), bf(2, 8, 2, 64)),
                 lambda: ctx.paged_write((bf(9, 4, 2, 64),) * 2, i32(2, 5), bf(1).expand(2, n, 2, 64), bf(1).expand(2, n, 2, 64)),
                 lambda: ctx.paged_attention(bf(2, 8, 4, 64), (bf(1).expand(9, n, 2, 64),) * 2, i32(2, 5), i32(2)),
                 lambda: ctx.paged_attention(bf(1).expand(2, n, 4, 64), (bf(9, 4, 2, 64),) * 2, i32(2, 5), i32(2)),
                 lambda: ctx.paged_commit(bf(1).expand(3, n, 4, 2, 64), i32(2, 5), None, i32(2), i32(2, 3)),
                 lambda: ctx.paged_commit(bf(3, 9, 4, 2, 64), i32(2, 5), None, i32(1).expand(n), i32(2, 3))):
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_paged_cache_layout():
    for dtype in (torch.bfloat16, torch.float16):
        p = G.paged_cache(5, 16, 2, 64, dtype, device="cpu")
        assert p.shape == (5, 16, 2, 64) and p.stride() == (2048, 64, 1024, 1) and p.dtype == dtype
        assert G.paged_cache(5, 16, 2, 64, dtype, planes=3, device="cpu").shape == (3, 5, 16, 2, 64)
    p = G.paged_cache(5, 16, 2, 64, torch.float8_e4m3fn, planes=3, device="cpu")
    assert p.shape == (3, 5, 16, 2, 64) and p.scales.stride() == (160, 32, 1, 16)
    with pytest.raises(TypeError):
        G.paged_cache(5, 16, 2, 64, torch.float32, device="cpu")
