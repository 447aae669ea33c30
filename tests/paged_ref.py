"""Plain 64-bit forms of the operators on a cache in pages, on the CPU, and their inputs."""
from __future__ import annotations

import math

import numpy as np
import torch

from verifier_ref import pack_mask, pow2, quantise, random_tree, values

U = 2.0 ** -24          # half a step of fp32, relative


def attention(q, k, v, seen, scale, eps):
    """One sequence.  q [n, Hq, D], k and v [rows, H, D] fp64, seen bool [n, rows].  Returns (out,
    lse, tol, lse_tol); the bounds are those of verifier_ref.attention, for scores and
    sums in fp32 and one rounding each of probabilities and results to a type of
    precision eps:
      - a score is a sum of D products: off by (D + 2) 2^-24 sum |q k|, a probability by twice
        scale times that for its own and the maximum's share, and by 2^-20 for exp2;
      - sums over n keys add n 2^-24 relative."""
    n, Hq, D = q.shape
    H = k.shape[1]
    G = Hq // H
    out = torch.zeros(n, Hq, D, dtype=torch.float64)
    tol, lse = out.clone(), torch.full((n, Hq), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros(n, Hq, dtype=torch.float64)
    if n == 0:
        return out, lse, tol, lse_tol
    some = seen.any(1)
    hide = ~seen
    any_ = seen.any(0)                       # rows that nobody sees may hold anything
    k, v = (torch.where(any_[:, None, None], x, 0.0) for x in (k, v))
    for h in range(Hq):
        kk, vv = k[:, h // G], v[:, h // G]
        s = (q[:, h] @ kk.T * scale).masked_fill(hide, -math.inf)
        z = torch.logsumexp(s, 1)
        p = torch.exp(s - torch.where(some, z, 0.0)[:, None])
        o = p @ vv
        size = scale * (q[:, h].abs() @ kk.abs().T).masked_fill(hide, 0.0).amax(1)
        ds = (D + 2) * U * size
        count = seen.sum(1)
        rel = 4 * ds + 2.0 ** -19 + 2 * (count + 64) * U
        out[:, h] = torch.where(some[:, None], o, 0.0)
        tol[:, h] = ((eps / 2 + rel)[:, None] * (p @ vv.abs()) + eps / 2 * o.abs()) * 1.01
        lse[:, h] = z
        lse_tol[:, h] = 2 * ds + (count + 64) * U + 2.0 ** -19 + torch.where(some, z, 0.0).abs() * 2.0 ** -22
    return out, lse, tol, lse_tol


def visible(base, n, window=0, sinks=0, block=None):
    """bool [n, base + n]: the rows that each of a block's n slots sees.  block: bool [n, n] of a
    masked block."""
    chain = block is None
    if chain:
        block = np.tril(np.ones((n, n), bool))
    seen = np.concatenate([np.ones((n, base), bool), block], 1)
    if window:
        place = base + block.sum(1) - 1
        r = np.arange(base + n)
        near = (r[None] > place[:, None] - window) | (r[None] < sinks)
        seen &= near if chain else near | (r[None] >= base)
    return torch.from_numpy(seen)


def tree_block(rng, n, depth=8):
    """Ancestor bits bool [n + 1, n + 1] of a tree of n nodes behind its root, and the nodes' own."""
    seen = random_tree(rng, n, depth)[2]
    block = np.zeros((n + 1, n + 1), bool)
    block[:, 0] = True
    block[1:, 1:] = seen
    return block, seen


def table(rng, page, rows, width=None, pool=None):
    """A page table [B, width] of sequences of rows[b] rows, pages dealt at random, -1 where a
    sequence needs none; and the pool's size."""
    need = [-(-int(n) // page) for n in rows]
    pages = max(1, pool or sum(need))
    order = rng.permutation(pages)
    t = np.full((len(rows), max(1, width or max(need))), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n]
        at += n
    return t, pages


def rows_of(pool, t, page, n):
    """Rows 0 .. n - 1 of a sequence, from a pool [pages, page, ...] and its table row."""
    r = np.arange(n)
    return pool[t[r // page], r % page]


def rotate(x, pos, freq, axis=None, interleaved=False):
    """x [S, heads, D] fp64, pos [axes, S] integers, freq [F] fp64: the rotated rows, and a bound
    of what fp32 makes of them: the angle is formed in fp64 by both, reduced to an argument
    below pi / 4 that fp32 rounds (2^-24), sine and cosine are sums of terms below 1 (three
    roundings count, and 2e-9 is cut), the pair takes three roundings of terms below |x| + |y|:
    10 2^-24 (|x| + |y|)."""
    F = len(freq)
    p = pos[axis] if axis is not None else np.repeat(pos[:1], F, 0)
    a = torch.from_numpy(p.T.astype(np.float64) * freq)[:, None]          # [S, 1, F]
    c, s = torch.cos(a), torch.sin(a)
    i = (slice(0, 2 * F, 2), slice(1, 2 * F, 2)) if interleaved else (slice(0, F), slice(F, 2 * F))
    u, w = x[..., i[0]], x[..., i[1]]
    y, tol = x.clone(), torch.zeros_like(x)
    y[..., i[0]], y[..., i[1]] = u * c - w * s, w * c + u * s
    tol[..., i[0]] = tol[..., i[1]] = 10 * U * (u.abs() + w.abs())
    return y, tol


__all__ = ["attention", "visible", "tree_block", "table", "rows_of", "rotate", "pack_mask", "quantise", "values",
           "pow2", "U"]
