"""How a call of tree_attention is cut, by the workspace that it asks for: parts times rows.  Contexts are
test_verifier_step_cpu's stand-ins."""
import ctypes as C
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_20375_amd as G  # noqa: E402
from test_verifier_step_cpu import Fake, attention, rows  # noqa: E402

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="stands in for a context")


def parts(slots, group, quant, batch=4, heads=32):
    """Parts of a call over a cache that is long enough for any number of them."""
    caches = dict(cache_dtype=3, cache_k=rows(True), cache_v=rows(True)) if quant else {}
    a = attention(batch=batch, slots=slots, q_heads=heads * group, kv_heads=heads, cache_rows=1 << 20, shared_len=0,
                  **caches)
    need = C.c_int64()
    assert G.lib().graft_tree_attention_workspace(Fake().h, C.byref(a), C.byref(need)) == 0
    row = batch * slots * heads * group * (a.head_dim * 4 + 8)     # a part's: numbers, a maximum and a sum a row
    assert need.value % row == 0
    return need.value // row


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("slots,group", [(1, 1), (5, 3), (16, 1), (17, 1), (1, 17), (6, 3), (8, 3), (31, 1), (1, 32), (8, 4),
                                         (16, 2), (32, 1)])
def test_up_to_32_rows_are_one_row_tile(slots, group, quant):
    """The narrow walk reads a cache once for all rows of a key head: 4096 workgroups are shared by
    the sequences and key heads alone, not by tiles of 16 rows as well."""
    assert parts(slots, group, quant) == 4096 // (4 * 32)
    assert parts(slots, group, quant, 3, 30) == -(-4096 // (3 * 30))


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("slots,group,tiles", [(33, 1, 1), (11, 3, 1), (32, 4, 1), (33, 4, 2), (32, 16, 4)])
def test_more_rows_are_tiles_of_128(slots, group, tiles, quant):
    assert parts(slots, group, quant, heads=8) == 1024 // (4 * 8 * tiles)
