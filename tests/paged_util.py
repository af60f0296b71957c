"""Inputs and 64-bit references for the tests of the paged-cache and differential-attention entry points."""
from __future__ import annotations

import math

import numpy as np
import torch

E4M3_MAX = 448.0
BF16_HALF = 2.0 ** -8       # half a step of bf16, relative to the value
E4M3_HALF = 2.0 ** -4
# fp32 arithmetic of a score: its error is below d * 2^-24 * sum |q k| * scale, about 192 * 2^-24 * 12 for the unit Gaussian
# inputs used here; the exponential turns it into a relative error of a probability, the sums and the division add a few 2^-24.
FP32_SLACK = 3e-4


def pool(lens, page, Hkv, dqk, dv, e4m3, heads_first, seed, device="cuda", spare=3, poison=True, shift=0.0):
    """A page pool in shuffled order.  Slots that belong to no key hold NaN (and infinities), block table entries that no key needs
    hold numbers that are no pages.  Returns (k, v, table, lens tensor, k_scale, v_scale); k and v have the logical shape."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g)
    table = torch.full((len(lens), max(max(need), 1) + 1), 2 ** 31 - 1, dtype=torch.int32)
    table[:, -1] = -7
    used = torch.zeros(pages, page, dtype=torch.bool)
    at = 0
    for b, n in enumerate(need):
        mine = order[at:at + n]
        table[b, :n] = mine.to(torch.int32)
        for j in range(n):
            used[mine[j], :min(page, lens[b] - j * page)] = True
        at += n
    out = []
    for d in (dqk, dv):
        shape = (pages, Hkv, page, d) if heads_first else (pages, page, Hkv, d)
        x = torch.randn(shape, generator=g) + shift
        x = (x * 20).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn) if e4m3 else x.to(torch.bfloat16)
        y = x if heads_first else x.permute(0, 2, 1, 3)
        if poison:
            bad = ~used[:, None, :, None].expand(pages, Hkv, page, d)
            if e4m3:
                y.view(torch.uint8)[bad] = 0x7F
            else:
                y[bad] = float("nan")
                y[:, :, :, ::7][bad[:, :, :, ::7]] = float("inf")
        out.append(y)
    ks = vs = None
    if e4m3:
        ks, vs = (0.9 + 0.2 * torch.rand(Hkv, generator=g)) / 20, (0.9 + 0.2 * torch.rand(Hkv, generator=g)) / 20
    move = lambda t: None if t is None else t.to(device)  # noqa: E731
    # (.to keeps the memory order of a permuted dense tensor)
    return move(out[0]), move(out[1]), move(table), torch.tensor(lens, dtype=torch.int32, device=device), move(ks), move(vs)


def rows_of(cache, scale, table, b, n):
    """The first n rows [Hkv, n, d] of sequence b in float64 on the CPU."""
    Hkv, page, d = cache.shape[1:]
    if n == 0:
        return torch.zeros(Hkv, 0, d, dtype=torch.float64)
    ids = table[b, :-(-n // page)].long().cpu()
    x = cache.cpu()
    x = torch.cat([(x[i].float() if x.dtype == torch.float8_e4m3fn else x[i]).double() for i in ids.tolist()], dim=1)[:, :n]
    return x if scale is None else x * scale.cpu().double()[:, None, None]


def softmax64(q, k, scale, last):
    """q [n, d], k [m, d] float64; row i sees keys j <= last[i].  Probabilities [n, m] (zero rows where nothing is seen), lse."""
    if k.shape[0] == 0:
        return torch.zeros(q.shape[0], 0, dtype=torch.float64), torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    z = (q @ k.T) * scale
    z = z.masked_fill(torch.arange(k.shape[0])[None] > last[:, None], -math.inf)
    lse = torch.logsumexp(z, 1)
    p = torch.where(torch.isinf(lse)[:, None], torch.zeros_like(z), torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[:, None]))
    return p, lse


def paged_reference(q, k, v, ks, vs, table, lens, Sq, scale):
    """(O, lse, A): A = sum_j p_j |v_j|, which the error of the rounded probabilities is measured by.  q [B*Sq, Hq, d] bf16."""
    T, Hq, dqk = q.shape
    Hkv, dv = k.shape[1], v.shape[3]
    O, A = torch.zeros(T, Hq, dv, dtype=torch.float64), torch.zeros(T, Hq, dv, dtype=torch.float64)
    L = torch.zeros(Hq, T, dtype=torch.float64)
    qd = q.cpu().double()
    for b, n in enumerate(lens):
        kd, vd = rows_of(k, ks, table, b, n), rows_of(v, vs, table, b, n)
        last = torch.arange(n - Sq, n)
        here = slice(b * Sq, (b + 1) * Sq)
        for h in range(Hq):
            p, lse = softmax64(qd[here, h], kd[h // (Hq // Hkv)], scale, last)
            O[here, h], A[here, h] = p @ vd[h // (Hq // Hkv)], p @ vd[h // (Hq // Hkv)].abs()
            L[h, here] = lse
    return O, L, A


def assert_attention(o, lse, O, L, A, what=""):
    """bf16 O and fp32 lse against the 64-bit ones: one rounding of O, one of every probability, fp32 arithmetic."""
    o = o.cpu().double()
    assert torch.isfinite(o).all(), what + " non-finite O"
    tol = BF16_HALF * O.abs() + (BF16_HALF + FP32_SLACK) * A + 1e-30
    worst = ((o - O).abs() / tol).max().item() if o.numel() else 0.0
    assert worst <= 1.0, "%s O is %.2f times its tolerance off" % (what, worst)
    if lse is not None:
        lse = lse.cpu().double()
        assert torch.equal(torch.isneginf(lse), torch.isneginf(L)), what + " rows without keys"
        fin = torch.isfinite(L)
        assert torch.isfinite(lse[fin]).all(), what
        if fin.any():
            off = ((lse - L)[fin].abs() / (FP32_SLACK + 1e-6 * L[fin].abs())).max().item()
            assert off <= 1.0, "%s lse is %.2f times its tolerance off" % (what, off)
    return worst


def diff_rows(q, k, v, lam, scale, last):
    """Y and its error measure for one head: q [n, 128], k [m, 128], v [m, dv] float64."""
    p1, _ = softmax64(q[:, :64], k[:, :64], scale, last)
    p2, _ = softmax64(q[:, 64:], k[:, 64:], scale, last)
    return (p1 - lam * p2) @ v, (p1 + abs(lam) * p2) @ v.abs()


def diff_norm(Y, A, weight, eps, out_scale):
    """O and the tolerance of its bf16 value, from Y and the measure A of the probabilities' rounding.

    dY <= (2^-8 + fp32) A.  With r = sqrt(mean Y^2 + eps), |d(Y / r)| <= (dY + |Y| / r * rms(dY)) / r."""
    dY = (BF16_HALF + FP32_SLACK) * A
    if weight is None:
        O = out_scale * Y
        return O, abs(out_scale) * dY + BF16_HALF * O.abs() + 1e-30
    r = torch.sqrt((Y * Y).mean(-1, keepdim=True) + eps)
    O = out_scale * weight * Y / r
    first = (dY + Y.abs() / r * torch.sqrt((dY * dY).mean(-1, keepdim=True))) / r
    return O, (out_scale * weight).abs() * (first * 1.01 + 1e-6 * Y.abs() / r) + BF16_HALF * O.abs() + 1e-30


def assert_close(o, O, tol, what=""):
    o = o.cpu().double()
    assert torch.isfinite(o).all(), what + " non-finite"
    worst = ((o - O).abs() / tol).max().item() if o.numel() else 0.0
    assert worst <= 1.0, "%s is %.2f times its tolerance off" % (what, worst)
    return worst


def ok(handle):
    from paper_2609_21264_b200 import binding
    torch.cuda.synchronize()
    st, detail = binding.fa_last_status(handle)
    assert st == binding.FA_OK, "device status %d (site 0x%x)" % (st, detail)


def rope_table(n, dim, device="cuda", base=10000.0):
    half = dim // 2
    angle = np.arange(n)[:, None] * base ** (-np.arange(half) / half)
    return torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).to(device)


def turned(x, rows, dim, offset, span, interleaved):
    """x [n, H, d] float64 with every span's pairs turned by the rows [n, dim] of the table, and the sum of the products' sizes."""
    y, size = x.clone(), x.abs()
    if rows is None:
        return y, size
    half = dim // 2
    for first in range(offset, x.shape[2], span):
        for i in range(half):
            a, b = (first + 2 * i, first + 2 * i + 1) if interleaved else (first + i, first + half + i)
            c, s = rows[:, i, None], rows[:, half + i, None]
            y[:, :, a], y[:, :, b] = x[:, :, a] * c - x[:, :, b] * s, x[:, :, b] * c + x[:, :, a] * s
            size[:, :, a] = size[:, :, b] = x[:, :, a].abs() + x[:, :, b].abs()
    return y, size
