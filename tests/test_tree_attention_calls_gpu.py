"""Context.tree_attention: what a call reports and writes, whatever ran before it."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_tree_attention_gpu import call, check, context, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes", [6, 40])
def test_cache_lengths_of_sequences_without_slots_are_reported(nodes):
    """Both walks: a sequence without a node and a root writes nothing, but its length counts."""
    c = make(2, nodes, [9, 12], 0, 2, 2, 64, "bfloat16", False, 0, n=[0, nodes], extra=0)
    ctx = context(c)
    good, zg, _ = call(ctx, c)
    check(c, good, zg)
    assert ctx.device_status() == 0
    for n in (-1, 13, 2 ** 31 - 1):
        lens = torch.tensor([n, 12], dtype=torch.int32, device="cuda")
        out, lse, _ = call(ctx, c, cache_len=lens)
        assert torch.equal(out, good) and torch.equal(lse, zg)
        assert ctx.device_status() == 5 and ctx.device_status() == 0, n
    ctx.close()
