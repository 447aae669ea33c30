"""Context.accept_sampled against the walk in 64 bits (verifier_ref.walk): whole numbers
are equal, log-probabilities to fp32's rounding."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import verifier_ref as R  # noqa: E402

pytestmark = pytest.mark.gpu


def make(batch, nodes, L, V, dtype="bfloat16", seed=0, mass=0.8, n=None, T=None, depth=None):
    """Trees and target logits in which a node's children have about `mass` of the
    probability at temperature 1."""
    rng = np.random.default_rng(seed)
    n = np.asarray(n if n is not None else [nodes - i % max(1, nodes // 2) for i in range(batch)],
                   np.int32)
    parents = np.full((batch, nodes), -1, np.int32)
    tokens = np.full((batch, nodes), -1, np.int32)
    z = rng.normal(size=(batch, nodes + 1, V)).astype(np.float32)
    for b in range(batch):
        p, t, _ = R.random_tree(rng, int(n[b]), depth or L, V)
        t = t % V
        parents[b, :n[b]], tokens[b, :n[b]] = p, t
        for i in range(int(n[b])):
            kids = int((p == p[i]).sum())
            z[b, p[i] + 1, t[i]] = np.log(mass / (1 - mass) * V * 1.65 / kids) + 0.1 * rng.normal()
    u = rng.random((batch, L + 1))
    T = np.asarray(T, np.float32) if T is not None else np.ones(batch, np.float32)
    return dict(z=torch.from_numpy(z).to(getattr(torch, dtype)), parents=parents, tokens=tokens, n=n,
                u=u, T=T, L=L, V=V)


def context(c):
    import paper_2608_20375_amd as G
    B, N = c["parents"].shape
    return G.Context(B, c["L"], c["V"], 1, N)


def call(ctx, c, **kw):
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    z = c["z"].cuda()
    a = dict(n_nodes=cu(c["n"]), tokens=cu(c["tokens"]), parents=cu(c["parents"]),
             root_logits=z[:, 0], node_logits=z[:, 1:], uniform=cu(c["u"]), temperature=cu(c["T"]))
    a.update(kw)
    return ctx.accept_sampled(**a)


def check(c, got, rows=None):
    acc, nodes, bonus, logp = (t.cpu().numpy() for t in got)
    z = c["z"].double().numpy()
    for b in range(len(c["n"])):
        zb = z[b] if rows is None else z[b, :rows + 1]
        a, path, x, lp = R.walk(zb, c["parents"][b], c["tokens"][b], int(c["n"][b]), c["L"],
                                c["u"][b], float(c["T"][b]))
        assert (acc[b], bonus[b]) == (a, x), (b, acc[b], a, bonus[b], x)
        assert np.array_equal(nodes[b], path), b
        # fp64 exponentials and sums, one rounding to fp32
        both = np.isinf(lp) & (logp[b] == lp)
        assert (both | (np.abs(np.where(both, 0, logp[b]) - np.where(both, 0, lp))
                        <= 2.0 ** -23 * np.abs(np.where(both, 0, lp)) + 1e-12)).all(), b
    return acc


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("batch,nodes,L,V", [(1, 1, 1, 1), (1, 4, 3, 2), (3, 20, 5, 7), (2, 9, 4, 515),
                                             (5, 30, 6, 8191), (4, 33, 5, 70001), (2, 64, 16, 151936),
                                             (70, 12, 4, 4099)])
def test_shapes(batch, nodes, L, V, dtype):
    print("sampled walk", batch, nodes, L, V, dtype, flush=True)
    if V < nodes:
        nodes = V
    c = make(batch, nodes, L, V, dtype, seed=V + batch)
    ctx = context(c)
    check(c, call(ctx, c))
    assert ctx.device_status() == 0
    ctx.close()


@pytest.mark.parametrize("V", [32000, 4099])
def test_temperatures(V):
    T = [0.0, 0.1, 0.5, 1.0, 1.7, 30.0, float("inf"), 1e-30, 1e30, 0.0]
    c = make(10, 24, 6, V, seed=5, T=T)
    ctx = context(c)
    check(c, call(ctx, c))
    c["T"][:] = 1.0
    check(c, call(ctx, c, temperature=None))
    assert ctx.device_status() == 0
    ctx.close()


def test_bad_temperatures_are_greedy_and_reported():
    c = make(3, 12, 4, 999, seed=6, T=[-1.0, float("nan"), 1.0])
    ctx = context(c)
    got = call(ctx, c)
    c["T"][:2] = 0.0
    check(c, got)
    assert ctx.device_status() == 5 and ctx.device_status() == 0
    ctx.close()


def test_greedy_matches_the_greedy_walk():
    """T = 0 is graft_accept with the rows' largest logits, ties to the lowest token."""
    c = make(6, 40, 8, 5000, seed=7, mass=0.999, T=[0.0] * 6)
    ctx = context(c)
    got = call(ctx, c)
    z = c["z"].float()
    best = torch.from_numpy(np.argmax(z.numpy(), -1).astype(np.int32)).cuda()
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    acc, nodes, bonus = ctx.accept(cu(c["n"]), cu(c["tokens"]), cu(c["parents"]),
                                   target_root=best[:, 0].contiguous(),
                                   target_node=best[:, 1:].contiguous())
    assert torch.equal(got[0], acc) and torch.equal(got[1], nodes) and torch.equal(got[2], bonus)
    assert int(acc.max()) > 0
    ctx.close()


@pytest.mark.parametrize("V", [64, 8200])
def test_ties_masked_and_infinite_logits(V):
    """Equal largest logits at T = 0; rows masked by -inf or bf16's lowest value but for a
    few tokens; NaN; +inf, which share the probability."""
    c = make(8, 6, 3, V, seed=8, T=[0, 0, 1, 1, 1, 1, 0, 1])
    low = torch.finfo(torch.bfloat16).min
    z = c["z"]
    z[0, :] = 1.5
    z[1, :] = -float("inf")
    z[1, :, V // 2:] = low
    z[2, :] = -float("inf")
    z[2, :, V - 1] = low
    z[3, :] = low
    z[3, :, 5], z[3, :, V - 2] = 2.0, 1.0
    z[4, :, ::3] = float("nan")
    z[5, :, 7], z[5, :, V - 3], z[5, :, 0] = float("inf"), float("inf"), float("nan")
    z[6, :, 9], z[6, :, 11] = float("inf"), float("inf")
    z[7, :] = low                                   # the lowest value alone is a number
    ctx = context(c)
    got = call(ctx, c)
    check(c, got)
    assert ctx.device_status() == 0
    ctx.close()


def test_rows_without_a_token_end_the_walk():
    c = make(3, 8, 4, 777, seed=9, mass=0.99)
    c["z"][0, 0] = -float("inf")
    c["z"][1, 0] = float("nan")
    c["z"][2, 1:] = -float("inf")
    ctx = context(c)
    got = call(ctx, c)
    acc = check(c, got)
    assert got[2][:2].tolist() == [-1, -1] and ctx.device_status() == 5
    ctx.close()


@pytest.mark.parametrize("u", [0.0, 5e-324, 1.0 - 2.0 ** -53, 1.0, 2.0, -1.0, float("nan"), float("inf")])
def test_random_numbers_at_and_past_their_ends(u):
    c = make(3, 10, 4, 3001, seed=10)
    c["z"][1, :, :17] = -float("inf")
    c["z"][1, :, -9:] = -float("inf")
    c["u"][:] = u
    ctx = context(c)
    check(c, call(ctx, c))
    ctx.close()


def test_borders_between_tokens():
    """Equal logits: the border after token v is (v + 1) / V exactly; numbers at a border take
    the next token, numbers just below it this one."""
    V, L = 4096, 3
    c = make(6, 1, L, V, n=[0] * 6, dtype="float32")
    c["z"][:] = 0.25
    at = np.array([0, 1, 511, 512, 2047, 4095])
    c["u"][:, 0] = at / V
    ctx = context(c)
    assert call(ctx, c)[2].cpu().numpy().tolist() == at.tolist()
    c["u"][:, 0] = np.nextafter((at + 1) / V, 0)
    assert call(ctx, c)[2].cpu().numpy().tolist() == at.tolist()
    ctx.close()


def test_nodes_without_logits_are_not_followed():
    c = make(4, 30, 6, 900, seed=12, mass=0.97)
    ctx = context(c)
    z = c["z"].cuda()
    for rows in (29, 11, 1):
        check(c, call(ctx, c, root_logits=z[:, 0], node_logits=z[:, 1:1 + rows]), rows)
    check(c, call(ctx, c, node_logits=z[:, 1:1]), 0)
    ctx.close()


def test_strided_and_misaligned_rows():
    """Rows at every alignment inside a wider buffer, the root's elsewhere."""
    c = make(3, 15, 5, 1003, seed=13)
    ctx = context(c)
    for shift in (0, 1, 3, 7):
        wide = torch.full((3, 18, 1003 + 24), 30.0, dtype=torch.bfloat16, device="cuda")
        wide[:, 2:17, shift:shift + 1003] = c["z"][:, 1:].cuda()
        root = torch.full((3, 2000), 30.0, dtype=torch.bfloat16, device="cuda")
        root[:, 5:5 + 1003] = c["z"][:, 0].cuda()
        check(c, call(ctx, c, root_logits=root[:, 5:5 + 1003],
                      node_logits=wide[:, 2:17, shift:shift + 1003]))
    ctx.close()


def test_full_paths_and_the_history():
    """A chain of L nodes taken to its end: L accepted, a bonus after it, and the history."""
    L = 6
    c = make(2, L, L, 500, n=[L, 2], mass=0.9999999, seed=14, depth=L)
    c["u"][:] = 0.5
    ctx = context(c)
    ctx.set_history(torch.zeros(2, 4, dtype=torch.int32, device="cuda"))
    for r in range(3):
        acc = check(c, call(ctx, c, update_history=True))
    assert acc.tolist()[0] == L
    ring, pos = ctx.get_history(2)
    assert ring[:, :3].cpu().tolist() == [[int(a)] * 3 for a in acc] and pos.tolist() == [3, 3]
    ctx.close()


def test_malformed_trees_end():
    """A node listed before its parent, a node that is its own parent and an n_nodes outside
    its range: the walk ends, nothing outside the tree is followed."""
    c = make(3, 5, 8, 50, n=[5, 5, 5], mass=0.9, seed=15)
    c["z"][:, :, :] = -float("inf")
    c["z"][:, :, 3] = 1.0
    c["tokens"][:] = 3
    c["parents"][0] = [2, 2, -1, -1, 2]
    c["parents"][1] = [0, 1, 2, 3, 4]
    c["parents"][2] = [-1, 0, 1, 2, 3]
    ctx = context(c)
    n = torch.tensor([5, 5, 99], dtype=torch.int32, device="cuda")
    acc, nodes, bonus, _ = call(ctx, c, n_nodes=n)
    assert acc.tolist() == [2, 0, 5] and bonus.tolist() == [3, 3, 3]
    assert nodes[0].tolist()[:3] == [2, 4, -1]
    n = torch.tensor([-7, 5, 2], dtype=torch.int32, device="cuda")
    assert call(ctx, c, n_nodes=n)[0].tolist() == [0, 0, 2]
    ctx.close()


def test_the_same_result_on_streams_and_in_graphs():
    c = make(8, 40, 8, 20011, seed=16, T=[1, 0, 1, 0.7, 1, 1, 1, 1])
    ctx = context(c)
    want = [t.clone() for t in call(ctx, c)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call(ctx, c)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    z, u = c["z"].cuda(), cu(c["u"])
    args = (cu(c["n"]), cu(c["tokens"]), cu(c["parents"]), z[:, 0], z[:, 1:], u, cu(c["T"]))
    i32 = dict(dtype=torch.int32, device="cuda")
    graphs = []
    for _ in range(2):
        out = dict(acc_len=torch.empty(8, **i32), acc_nodes=torch.empty(8, 8, **i32),
                   bonus=torch.empty(8, **i32), logp=torch.empty(8, 9, device="cuda"))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.accept_sampled(*args, **out)
        graphs.append((g, out))
    for turn in range(3):
        u.copy_(torch.rand(8, 9, dtype=torch.float64))
        c["u"] = u.cpu().numpy()
        eager = ctx.accept_sampled(*args)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        check(c, eager)
        for _, o in graphs:
            assert torch.equal(o["acc_len"], eager[0]) and torch.equal(o["acc_nodes"], eager[1])
            assert torch.equal(o["bonus"], eager[2]) and torch.equal(o["logp"], eager[3])
    ctx.close()


def test_rows_past_32_bit_offsets():
    """Node rows that start more than 2^31 elements into the buffer."""
    V = 151936
    c = make(1, 2, 2, V, n=[2], seed=17, mass=0.999999, depth=2)
    c["u"][:] = 0.5
    buf = torch.empty(2 ** 31 + 4 * V, dtype=torch.bfloat16, device="cuda")
    far = 2 ** 31 + V
    rows = buf.as_strided((1, 2, V), (0, far, 1))
    rows.copy_(c["z"][:, 1:])
    ctx = context(c)
    acc = check(c, call(ctx, c, node_logits=rows))
    assert acc.tolist() == [2]
    ctx.close()


def test_refusals_with_real_tensors():
    import paper_2608_20375_amd as G
    c = make(2, 6, 3, 100)
    ctx = context(c)
    z = c["z"].cuda()
    with pytest.raises(TypeError):
        call(ctx, c, uniform=torch.zeros(2, 4, device="cuda"))          # fp32 random numbers
    with pytest.raises(TypeError):
        call(ctx, c, root_logits=z[:, 0].float())
    with pytest.raises(ValueError):
        call(ctx, c, node_logits=z[:, 1:].transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError):
        call(ctx, c, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(G.GraftError):
        call(ctx, c, update_history=True)                               # no ring installed
    with pytest.raises(TypeError):
        call(ctx, c, temperature=torch.ones(2))
    ctx.close()
