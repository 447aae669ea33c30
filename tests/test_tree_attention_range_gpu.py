"""Context.tree_attention at the ends of its numbers' range: many small probabilities beside a
dominant one, and scores far past what a 32-bit exponent's argument holds."""
import math
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import verifier_ref as R  # noqa: E402
from test_tree_attention_gpu import call, check, context, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("below", [20.0, 24.4, 25.4, 25.9])
@pytest.mark.parametrize("nodes", [0, 40])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_many_small_probabilities(below, nodes, dtype):
    """Ten keys that take nearly all of the probability, with values of 0, among 24000 whose
    probabilities are 2^-below of theirs: the result is those keys' sum, and each of them has to
    keep the relative precision that verifier_ref.attention counts."""
    print("small probabilities", below, nodes, dtype, flush=True)
    c = make(1, nodes, [24000], 0, 1, 1, 64, dtype, False, 1, chain=True, n=[nodes])
    g = torch.Generator().manual_seed(7)
    c["q"].fill_(1.0)
    c["k"].zero_()
    c["v"].zero_()
    keys, values = c["cache"]
    keys.copy_(torch.randn(keys.shape, generator=g) * 0.02)
    values.copy_(torch.randn(values.shape, generator=g) + 8.0)
    keys[:, ::2400] = below * math.log(2.0) / (64 * 0.125)
    values[:, ::2400] = 0.0
    ctx = context(c)
    out, lse, _ = call(ctx, c)
    check(c, out, lse)
    ctx.close()


@pytest.mark.parametrize("kind,power", [(k, p) for k in ("bfloat16", "e4m3") for p in (4, 20, 26, 30, 40, 100)]
                         + [("float16", p) for p in (4, 20, 24, 26, 28, 30)])
@pytest.mark.parametrize("nodes", [0, 40])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(kind, power, nodes, sign):
    """Scores are 1.375^2 2^power times 1, 1/2, 0 and -1 (or about -1, -5/4, -3/2 and -2), one product
    each and so exact in fp32, two keys of different parts having the largest.  Differences from the maximum are exact, so the only errors are the
    roundings of probabilities and results, 2^-23 of an exponent's argument (below 150, or the
    probability is 0) and a few of the sums."""
    print("scores", kind, power, nodes, sign, flush=True)
    quant = kind == "e4m3"
    dtype = "bfloat16" if quant else kind
    c = make(2, nodes, [700, 20], 0, 2, 1, 64, dtype, False, 1, chain=True, n=[nodes, nodes])
    g = torch.Generator().manual_seed(power)
    half = power // 2
    for name in ("q", "k"):
        c[name].zero_()
    c["q"][..., 0] = sign * 1.375 * 2.0 ** half
    rows = c["cache"][0].shape[1]
    factor = torch.tensor([0.5, 0.0, -1.0] if sign > 0 else [1.25, 1.5, 2.0])[torch.randint(0, 3, (2, rows), generator=g)]
    factor[:, 3] = factor[0, 650] = factor[1, 18] = 1.0
    block = 0.0 if sign > 0 else 1.0
    c["k"][..., 0] = block * 1.375 * 2.0 ** (power - half)
    c["cache"][0].zero_()
    c["cache"][0][..., 0, 0] = factor.to(c["dt"]) * (1.375 * 2.0 ** (power - half))
    if quant:
        c["cache"], c["quant"] = [R.quantise(x) for x in c["cache"]], True
        c["val"] = lambda pair: [R.values(*x) for x in pair]
    ctx = context(c)
    out, lse, _ = call(ctx, c, scale=1.0)
    assert ctx.device_status() == 0
    ctx.close()
    keys, values = c["val"](c["cache"])
    query = sign * 1.375 * 2.0 ** half
    out, lse, eps = out.cpu().double(), lse.cpu().double(), torch.finfo(c["dt"]).eps
    for b in range(2):
        n = int(c["lens"][b])
        for i in range(nodes + 1):
            s = query * torch.cat([keys[b, :n, 0, 0], c["k"][b, :i + 1, 0, 0].double()])
            v = torch.cat([values[b, :n, 0], c["v"][b, :i + 1, 0].double()])
            z = torch.logsumexp(s, 0)
            p = torch.exp(s - s.max())
            p /= p.sum()
            want = p @ v
            tol = (eps / 2 + 150 * 2.0 ** -23 + 1024 * 2.0 ** -24) * (p @ v.abs()) + eps / 2 * want.abs()
            for h in range(2):
                assert ((out[b, i, h] - want).abs() <= 1.01 * tol).all(), (b, i, h)
                assert abs(lse[b, i, h] - z) <= 2.0 ** -16 + z.abs() * 2.0 ** -22, (b, i, h)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("nodes", [0, 40])
def test_the_largest_scores(nodes, sign):
    """Scores of 1.25 2^127, all alike, whose product with log2 e is just inside fp32: a row is the
    mean of the values it sees, rounded once with probabilities that are equal and exact."""
    print("largest", nodes, sign, flush=True)
    c = make(2, nodes, [300, 20], 0, 2, 1, 64, "bfloat16", False, 1, chain=True, n=[nodes, nodes])
    c["q"].zero_()
    c["q"][..., 0] = sign * 1.25 * 2.0 ** 63
    for k in (c["k"], c["cache"][0]):
        k.zero_()
        k[..., 0] = 2.0 ** 64
    ctx = context(c)
    out, lse, _ = call(ctx, c, scale=1.0)
    ctx.close()
    out, lse, eps = out.cpu().double(), lse.cpu().double(), torch.finfo(c["dt"]).eps
    for b in range(2):
        for i in range(nodes + 1):
            v = torch.cat([c["cache"][1][b, :int(c["lens"][b]), 0], c["v"][b, :i + 1, 0]]).double()
            want, tol = v.mean(0), 1024 * 2.0 ** -24 * v.abs().mean(0)
            assert ((out[b, i] - want).abs() <= 1.01 * (tol + eps / 2 * want.abs())).all(), (b, i)
            z = sign * 1.25 * 2.0 ** 127
            assert (lse[b, i] - z).abs().max() <= abs(z) * 2.0 ** -22, (b, i)
