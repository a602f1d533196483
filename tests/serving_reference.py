"""Plain implementations in 64 bits (numpy) of page planning, norm with rotation, and attention over the quantized cache."""
import math

import numpy as np

import mx_reference as mx


def plan(lens, fresh, page, table, free, count, total):
    """-> table, lens, q_starts, starts, slots, positions, left, missing."""
    table, width = np.array(table, dtype=np.int64), table.shape[1]
    count = min(max(count, 0), len(free))
    slots, positions, after, taken = [-1] * total, [0] * total, [], 0
    q_starts, starts, t = [0], [0], 0
    for s, (h, m) in enumerate(zip(lens, fresh)):
        h, m = max(int(h), 0), max(int(m), 0)
        for p in range(min(-(-h // page), width), min(-(-(h + m) // page), width)):
            table[s, p] = free[count - 1 - taken] if taken < count else -1
            taken += 1
        for at in range(h, h + m):
            if t < total:
                held = table[s, at // page] if at // page < width else -1
                slots[t], positions[t] = (held * page + at % page if held >= 0 else -1), at
            t += 1
        after.append(h + m)
        q_starts.append(t)
        starts.append(starts[-1] + h + m)
    return table, after, q_starts, starts, slots, positions, max(count - taken, 0), max(taken - count, 0)


def norm_rotate(x, weight, positions, freqs, eps, pairs):
    """x [tokens, heads, dim] in 64 bits."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x * weight.astype(np.float64) / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    half = len(freqs)
    t = positions.astype(np.float64)[:, None] * freqs.astype(np.float64)[None]
    c, s = np.cos(t)[:, None], np.sin(t)[:, None]
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def rows_of(codes, scales, dim, i8):
    """Values [..., dim] of cache rows."""
    if i8:
        return codes.astype(np.float64) * scales.astype(np.float64)[..., None]
    lead = codes.shape[:-1]
    return mx.values(codes.reshape(-1, codes.shape[-1]), scales.reshape(-1, scales.shape[-1]), dim).reshape(*lead, dim)


def attend(q, k, v, lens, q_starts, table, page, scale, window=0, cap=0.0, slopes=None, bits=11):
    """q [rows, q_heads, dim]; k, v [pages, page, heads, dim] values.  -> out, lse (NaN in rows of no sequence), and a bound on
    what rounding may do to out and to lse of a kernel whose weights have `bits` bits."""
    rows, q_heads, dim = q.shape
    heads = k.shape[2]
    group = q_heads // heads
    out, lse = np.full((rows, q_heads, dim), np.nan), np.full((rows, q_heads), np.nan)
    off, off_lse = np.zeros((rows, q_heads, dim)), np.zeros((rows, q_heads))
    for s in range(len(lens)):
        lo = min(max(q_starts[s], 0), rows)
        n = min(max(q_starts[s + 1], lo), rows) - lo
        for i in range(n):
            p = lens[s] - n + i
            j = np.arange(max(0, p - window + 1) if window else 0, max(0, min(p + 1, table.shape[1] * page)))
            ids = table[s, j // page] if len(j) else np.zeros(0, dtype=np.int64)
            ok = (ids >= 0) & (ids < k.shape[0])
            j, ids = j[ok], ids[ok]
            kk, vv = k[ids, j % page], v[ids, j % page]                      # [tokens, heads, dim]
            for h in range(q_heads):
                if not len(j):
                    out[lo + i, h], lse[lo + i, h] = 0.0, -np.inf
                    continue
                qq, kh, vh = q[lo + i, h], kk[:, h // group], vv[:, h // group]
                if not np.isfinite(qq).all():
                    out[lo + i, h], lse[lo + i, h] = np.nan, np.nan
                    continue
                x = scale * (kh @ qq)
                if cap:
                    x = cap * np.tanh(x / cap)
                if slopes is not None:
                    x = x + slopes[h] * (j - p)
                if np.isnan(x).any() or np.isnan(vh).any():
                    out[lo + i, h], lse[lo + i, h] = np.nan, (np.nan if np.isnan(x).any() else x.max() + math.log(np.exp(x - x.max()).sum()))
                    continue
                e = np.exp(x - x.max())
                w = e / e.sum()
                out[lo + i, h], lse[lo + i, h] = w @ vh, x.max() + math.log(e.sum())
                # scores: dim products and sums in binary32, queries of 22 bits at least, a few roundings of x itself; then exp to 2^-22 and a
                # sum of len terms; weights to half a step of `bits` bits; sums over len terms
                dx = 2.0 ** -24 * ((dim + 8) * abs(scale) * (np.abs(kh) @ np.abs(qq)).max() + 12 * (np.abs(x).max() + cap + (abs(slopes[h]) * (p - j[0]) if slopes is not None else 0))) + \
                    2.0 ** -22 * abs(scale) * np.abs(qq).max() * np.abs(kh).sum(-1).max()
                dp = dx + 2.0 ** -21 + len(j) * 2.0 ** -24
                off[lo + i, h] = (2 * dp + 2.0 ** -bits + (len(j) + 16) * 2.0 ** -24) * (w @ np.abs(vh)) + 2.0 ** -30 * np.abs(vh).max()
                off_lse[lo + i, h] = dp + 2.0 ** -23 * (np.abs(lse[lo + i, h]) + 1)
    return out, lse, off, off_lse
