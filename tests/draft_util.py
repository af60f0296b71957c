"""Inputs and 64-bit references for the tests of the entry points on drafted tokens."""
from __future__ import annotations

import torch

from paged_util import rows_of


def random_parents(n, g):
    """Parents of a random tree of n tokens: an earlier token, or -1."""
    return [int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(n)]


def seen_by(parents):
    """[n, n] truth values: token i sees itself and its ancestors; and every token's depth."""
    n = len(parents)
    seen, depth = torch.zeros(n, n, dtype=torch.bool), [0] * n
    for i, a in enumerate(parents):
        if a >= 0:
            seen[i] = seen[a]
            depth[i] = depth[a] + 1
        seen[i, i] = True
    return seen, depth


def pack(seen, words):
    """[n, words] int32 of a [n, m] truth matrix, bit by bit."""
    out = torch.zeros(seen.shape[0], words, dtype=torch.int32)
    for i, row in enumerate(seen.tolist()):
        for w in range(words):
            x = sum(1 << e for e in range(32) if 32 * w + e < len(row) and row[32 * w + e])
            out[i, w] = x - (1 << 32) if x >= 1 << 31 else x
    return out


def tree_reference(q, k, v, ks, vs, table, lens, offsets, seens, scale):
    """(O, lse, A) in 64 bits: q [T, Hq, d]; seens[b] [n, n] says which drafts the drafts of sequence b see.  A = sum_j p_j |v_j|."""
    T, Hq, _ = q.shape
    Hkv, dv = k.shape[1], v.shape[3]
    O, A = torch.zeros(T, Hq, dv, dtype=torch.float64), torch.zeros(T, Hq, dv, dtype=torch.float64)
    L = torch.zeros(Hq, T, dtype=torch.float64)
    qd = q.cpu().double()
    for b, n in enumerate(lens):
        here = slice(offsets[b], offsets[b + 1])
        m = offsets[b + 1] - offsets[b]
        if m == 0:
            continue
        kd, vd = rows_of(k, ks, table, b, n), rows_of(v, vs, table, b, n)
        vis = torch.ones(m, n, dtype=torch.bool)
        draft = torch.arange(n) - (n - m)
        vis[:, draft >= 0] = seens[b][:, draft[draft >= 0]]
        for h in range(Hq):
            z = (qd[here, h] @ kd[h // (Hq // Hkv)].T) * scale
            z = z.masked_fill(~vis, -float("inf"))
            lse = torch.logsumexp(z, 1) if n else torch.full((m,), -float("inf"), dtype=torch.float64)
            p = torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[:, None])
            vh = vd[h // (Hq // Hkv)]
            # (a masked value may be anything finite)
            O[here, h], A[here, h] = p @ vh, p @ vh.abs()
            L[h, here] = lse
    return O, L, A
