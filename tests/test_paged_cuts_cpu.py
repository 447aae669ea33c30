"""How the paged attention's wide walk is cut, on the host: the choice itself, and that calls with many
row tiles are cut at all, by the workspace that they ask for."""
import ctypes as C
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_20375_amd as G  # noqa: E402
from test_pages_cpu import attend, no_gpu, pages  # noqa: E402
from test_verifier_step_cpu import Fake  # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def test_cuts(tmp_path):
    exe = tmp_path / "cuts"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2608_20375_amd", "csrc"), "-o", str(exe),
                    os.path.join(HERE, "cuts_driver.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


@no_gpu
@pytest.mark.parametrize("batch", [1, 55, 56, 63, 64, 65, 200])
@pytest.mark.parametrize("slots,group", [(8, 4), (33, 4), (65, 4), (1, 17)])
def test_long_tables_are_cut_whatever_the_batch(batch, slots, group):
    """A workspace for 512 workgroups' pieces, however many row tiles there are: any sequence may be long."""
    need = C.c_int64()
    a = attend(batch=batch, slots=slots, with_root=0, mask=0, q_heads=8 * group, kv_heads=8, head_dim=128,
               pages=pages(table_len=1024, table_stride=1024, page_rows=64))
    f = Fake(batch=256)
    assert G.lib().graft_paged_attention_workspace(f.h, C.byref(a), C.byref(need)) == 0
    assert need.value == 512 * 128 * (128 * 4 + 8) + 4 * (batch + 1)
