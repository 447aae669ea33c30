"""Page tables that the binding takes and refuses, on the CPU.  Contexts are test_verifier_step_cpu's stand-ins."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_pages_cpu import bf, i32, no_gpu  # noqa: E402
from test_verifier_step_cpu import context  # noqa: E402

pytestmark = no_gpu
POOL = lambda: (bf(9, 4, 2, 64), bf(9, 4, 2, 64))
CALLS = [lambda c, t: c.paged_write(POOL(), t, bf(2, 8, 2, 64), bf(2, 8, 2, 64)),
         lambda c, t: c.paged_attention(bf(2, 8, 4, 64), POOL(), t, i32(2)),
         lambda c, t: c.paged_commit(bf(3, 9, 4, 2, 64), t, None, i32(2), i32(2, 3))]


@pytest.mark.parametrize("call", CALLS)
def test_tables(call):
    """Rows any distance apart: refused for their device alone."""
    ctx = context()
    for t in (i32(2, 5), i32(2, 40)[:, 7:12], i32(6, 5)[::3], i32(5).expand(2, 5), i32(9, 2)[:, :1], i32(3, 9)[:, 2:]):
        with pytest.raises(TypeError, match="must be a CUDA"):
            call(ctx, t)
    for t in (i32(5, 2).t(), i32(2, 10)[:, ::2], i32(1, 5), i32(2, 0), i32(2), None, i32(2, 1).expand(2, 5)):
        with pytest.raises(ValueError):
            call(ctx, t)
    with pytest.raises(TypeError, match="int32"):
        call(ctx, i32(2, 5).long())
