"""Plain 64-bit forms of the verifier-side operators (tree attention, the sampled
walk, quantised rows) in numpy and torch on the CPU, for the tests."""
from __future__ import annotations

import math

import numpy as np
import torch


def pow2(e):
    """2^e exactly, integer tensor e in -1022..1023, fp64."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def quantise(x):
    """(codes uint8, scales uint8) of a bfloat16 CPU tensor's rows along its last axis."""
    d = x.double()
    fin = torch.isfinite(d)
    top = torch.where(fin, d.abs(), 0.0).amax(-1)
    part, power = torch.frexp(top)
    e = torch.where(part <= 0.875, power - 9, power - 8)
    e = torch.where(top == 0, -118, e).clamp_min(-118)
    most = torch.where(e == 120, 240.0, 448.0).unsqueeze(-1).double()
    y = d / pow2(e).unsqueeze(-1)
    y = torch.where(torch.isnan(y), y, torch.minimum(torch.maximum(y, -most), most))
    codes = y.float().to(torch.float8_e4m3fn).view(torch.uint8)
    codes = torch.where(torch.isnan(d), codes | 0x7F, codes)
    return codes, (e + 127).to(torch.uint8)


def values(codes, scales):
    """The fp64 numbers of codes and scales (CPU)."""
    c = codes.view(torch.uint8).view(torch.float8_e4m3fn).double()
    return c * pow2(scales.to(torch.int64) - 127).unsqueeze(-1)


def random_tree(rng, n, depth, vocab=50000):
    """Canonical parents, tokens and the ancestor bits (bool [n, n]) of a random tree."""
    if n == 0:
        return np.zeros(0, np.int32), np.zeros(0, np.int32), np.zeros((0, 0), bool)
    depth = min(depth, n)
    at = np.sort(np.concatenate([np.arange(depth), rng.integers(0, depth, n - depth)]))
    parents, tokens = np.full(n, -1, np.int32), np.zeros(n, np.int32)
    toks = rng.permutation(max(vocab, n))[:n]
    for d in range(depth):
        level = np.flatnonzero(at == d)
        if d:
            above = np.flatnonzero(at == d - 1)
            parents[level] = np.sort(rng.choice(above, len(level)))
        order = np.lexsort((toks[level], parents[level]))
        tokens[level] = toks[level][order]
        parents[level] = parents[level][order]
    seen = np.zeros((n, n), bool)
    for i in range(n):
        if parents[i] >= 0:
            seen[i] = seen[parents[i]]
        seen[i, i] = True
    return parents, tokens, seen


def pack_mask(seen, n_max):
    """Bitset words [n_max, words] int64 of a bool [n, n]."""
    n = len(seen)
    m = np.zeros((n_max, (n_max + 63) // 64), np.uint64)
    for j in range(n):
        m[:n, j >> 6] |= seen[:, j].astype(np.uint64) << np.uint64(j & 63)
    return m.view(np.int64)


def attention(q, k, v, seen, prefix_k, prefix_v, scale, eps):
    """One sequence in 64 bits.  q [S, Hq, D], k and v [S, H, D] fp64, seen bool [S, S],
    prefix [P, H, D].  Returns (out, lse, tol, lse_tol): tol bounds the error of a kernel that
    forms scores and sums in fp32 and rounds probabilities and results to a type of
    precision eps (a rounding is off by eps / 2 of the value):
      - a score is a sum of D products: off by (D + 2) 2^-24 sum |q k|, so a probability by
        twice scale times that (its own and the maximum's share), and by 2^-20 for exp2;
      - sums over n keys add n 2^-24 relative;
      - probabilities rounded once, results rounded once."""
    S, Hq, D = q.shape
    H = k.shape[1]
    out = torch.zeros(S, Hq, D, dtype=torch.float64)
    tol = torch.zeros(S, Hq, D, dtype=torch.float64)
    lse = torch.full((S, Hq), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros(S, Hq, dtype=torch.float64)
    u = 2.0 ** -24
    for h in range(Hq):
        g = h // (Hq // H)
        for i in range(S):
            rows = torch.from_numpy(np.flatnonzero(seen[i]))
            kk = torch.cat([prefix_k[:, g], k[rows, g]])
            vv = torch.cat([prefix_v[:, g], v[rows, g]])
            n = len(kk)
            if n == 0:
                continue
            s = kk @ q[i, h] * scale
            z = torch.logsumexp(s, 0)
            p = torch.exp(s - z)
            out[i, h] = p @ vv
            lse[i, h] = z
            ds = scale * (D + 2) * u * (kk.abs() @ q[i, h].abs()).max()
            rel = 4 * ds + 2.0 ** -19 + 2 * (n + 64) * u
            tol[i, h] = (eps / 2 + rel) * (p @ vv.abs()) * 1.01 + eps / 2 * out[i, h].abs() * 1.01
            lse_tol[i, h] = 2 * ds + (n + 64) * u + 2.0 ** -19 + z.abs() * 2.0 ** -22
    return out, lse, tol, lse_tol


def walk(logits, parents, tokens, n, L, uniform, T):
    """One sequence's sampled walk.  logits [1 + rows, V] fp64 numpy (NaN, infinities allowed).
    Returns acc_len, nodes, bonus, logp."""
    V = logits.shape[1]
    n = min(n, logits.shape[0] - 1)
    at, nodes = -1, np.full(L, -1, np.int32)
    logp = np.zeros(L + 1)
    for d in range(L + 1):
        z = logits[at + 1].copy()
        z[np.isnan(z)] = -np.inf
        top = z.max()
        if top == -np.inf:
            logp[d] = -np.inf
            return d, nodes, -1, logp
        if not T > 0:
            x, lp = int(np.argmax(z)), 0.0
        else:
            with np.errstate(all="ignore"):
                e = np.exp((z - top) / T)
            e[z == -np.inf] = 0.0
            if top == np.inf:
                e[:] = 0.0
            e[z == top] = 1.0
            c = np.cumsum(e)
            hit = np.flatnonzero((c > uniform[d] * c[-1]) & (e > 0))
            x = int(hit[0]) if len(hit) else int(np.flatnonzero(e > 0)[-1])
            lp = math.log(e[x]) - math.log(c[-1])
        logp[d] = lp
        child = [i for i in range(at + 1, n) if parents[i] == at and tokens[i] == x]
        if d == L or not child:
            return d, nodes, x, logp
        at = nodes[d] = child[0]
