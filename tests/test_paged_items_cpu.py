"""The wide walk's row tiles and workgroups on the host, and the binding's packed descriptors against
their structures."""
import ctypes as C
import os
import subprocess

import pytest

pytest.importorskip("torch")

import paper_2608_20375_amd as G

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def test_items(tmp_path):
    exe = tmp_path / "items"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2608_20375_amd", "csrc"), "-o", str(exe),
                    os.path.join(HERE, "items_driver.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


def flat(struct, value, name=""):
    """(name, number) of a structure's fields in order, structures in it taken apart."""
    for field, t in struct._fields_:
        x = getattr(value, field)
        if issubclass(t, C.Structure):
            yield from flat(t, x, name + field + ".")
        else:
            yield name + field, 0 if x is None else x


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("packing,struct", [("_PACK_ROWS", "PagedRows"), ("_PACK_ATTENTION", "PagedAttention"),
                                            ("_PACK_PATH", "PagedPath")])
def test_packed_descriptors(packing, struct, quant):
    """Numbers packed in order arrive in the fields in order; strides and scales that a packing
    leaves out are 0: a block's and a layer's plane stride, and scales where there are none."""
    s, p = getattr(G, struct), getattr(G, packing)[quant]

    def left_out(name):
        rows, _, part = name.partition(".")
        if part.endswith("plane_stride"):
            return struct != "PagedPath" or (part.startswith("scale") and not quant)
        return part.startswith("scale") and (not quant or rows not in ("cache_k", "cache_v", "rows"))

    n = sum(not left_out(name) for name, _ in flat(s, s()))
    got = list(flat(s, s.from_buffer_copy(p.pack(*range(1, n + 1)))))
    want = iter(range(1, n + 1))
    for name, x in got:
        assert x == (0 if left_out(name) else next(want)), name
