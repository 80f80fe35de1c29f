"""Full caches and the position rotation, written out in 64 bits on the CPU, with bounds of what a
32-bit computation may be off by.

Rounding: a result in type t is off by at most half a step, eps(t) / 2 of its size.  In fp32 a sum of n
terms is off by at most n 2^-24 of the sum of their sizes, whatever its order."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24                                             # half a step of fp32
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}       # half a step, of the result


def inv_freqs(r, base=10000.0):
    return (base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float()


def turn(x, positions, freqs, r, pairs, inverse=False):
    """x [T, heads, d] turned by positions [T] (64 bits), and the bound of its error when stored in x's
    type: the angle's fraction of a turn is rounded to fp32 (2 pi 2^-25 radians at most), its cosine and
    sine to 2^-23, two products and a sum: 5 2^-24 of |x| + |y|, within 2^-21 of it in all."""
    y = x.double().clone()
    if r:
        a = positions.double()[:, None] * freqs.double()
        c, s = a.cos()[:, None], (-a.sin() if inverse else a.sin())[:, None]
        first, second = (slice(0, r // 2), slice(r // 2, r)) if pairs == "halves" else (slice(0, r, 2), slice(1, r, 2))
        u, v = x[..., first].double(), x[..., second].double()
        y[..., first], y[..., second] = u * c - v * s, u * s + v * c
        size = torch.zeros_like(y)
        size[..., first] = size[..., second] = u.abs() + v.abs()
    else:
        size = torch.zeros_like(y)
    off = size * 2.0 ** -21 + (HALF[x.dtype] * (y.abs() + size * 2.0 ** -21) if r else 0.0)
    off[..., r:] = 0.0   # copied
    return y, off


def attend(q, K, V, n, wide=False):
    """Queries q [m, hq, d] at the positions n .. n + m - 1 over keys and values K, V [hkv, n + m, d]:
    (out, lse, bound of out, bound of lse).  Scores: products summed over d in fp32, scaled, and the
    scale's own rounding: (d + 4) U of the sum of |q_i k_i| / sqrt(d); exp2 of a difference of two such
    (its argument rounded, the result within 2^-22): so each probability, before it is divided, within
    a relative e = 2 max((d + 4) U sum|q k| / sqrt(d)) + 2^-20; P as two bf16 terms 2^-16 (wide tiles: as
    one, 2^-8); sums over n keys n U of the sum of |p v|; numerator and denominator alike, hence twice."""
    m, hq, d = q.shape
    G = hq // K.shape[0]
    dt = q.dtype
    out, lse = torch.zeros(m, hq, d, dtype=torch.float64), torch.zeros(m, hq, dtype=torch.float64)
    eo, el = torch.zeros_like(out), torch.zeros_like(lse)
    for h in range(hq):
        k, v = K[h // G, :n + m].double(), V[h // G, :n + m].double()
        x = q[:, h].double()
        seen = torch.arange(n + m) <= n + torch.arange(m)[:, None]
        s = torch.where(seen, x @ k.t() / math.sqrt(d), -math.inf)
        size = torch.where(seen, x.abs() @ k.abs().t() / math.sqrt(d), 0.0).amax(1)
        lse[:, h] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[:, h, None])
        out[:, h] = p @ torch.where(seen.any(0)[:, None], v, 0.0)
        e = 2 * (d + 4) * U * size + 2.0 ** -20 + (n + m) * U
        a = p @ v.abs()
        eo[:, h] = 2 * e[:, None] * a
        if dt == torch.bfloat16:
            eo[:, h] += 2.0 ** (-8 if wide else -16) * (1 + e[:, None]) * a
        eo[:, h] += HALF[dt] * (out[:, h].abs() + eo[:, h])
        el[:, h] = e + 4 * U * (lse[:, h].abs() + 10)
    return out, lse, eo, el


def close(got, want, off, what):
    got = got.detach().cpu().double()
    bad = ~((got - want).abs() <= off)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} too far off, first at {i}: got {got[i].item()!r}, "
                             f"want {want[i].item()!r} within {off[i].item():.3e}")


def fill_tables(full, need, gen, spare=0):
    """Pages for rows that need so many, in no order; unused entries -1."""
    order = torch.randperm(full.cfg.num_pages - spare, generator=gen).int() + spare
    table = torch.full((full.cfg.batch, full.cfg.max_pages), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    full.page_table.copy_(table)
    return table


def rows_of(pool, table, b, tokens, page):
    """Row b's first tokens of a pool [pages, hkv, page, d] as [hkv, tokens, d]."""
    if tokens == 0:
        return pool[0, :, :0]
    pages = table[b, :-(-tokens // page)].long()
    x = pool[pages]
    return x.transpose(0, 1).reshape(pool.shape[1], -1, pool.shape[3])[:, :tokens]
