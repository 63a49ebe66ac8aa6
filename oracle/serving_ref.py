"""The serving cache's two operations in 64 bits, token by token, from their definitions (numpy; nothing of the GPU path).

A cache is given as values: [l][P][bt][heads][d] float64 arrays.  Both functions are slow and plain on purpose.
"""
import math

import numpy as np

TOP = {"i8": 127.0, "e4m3": 448.0}


def rotate(x, pos, table, pairs):
    """x [..., d] turned by row `pos` of table [positions][rot] (cosines, then sines)."""
    x = np.array(x, dtype=np.float64)
    half = table.shape[1] // 2
    for i in range(half):
        lo, hi = (2 * i, 2 * i + 1) if pairs else (i, i + half)
        c, s = float(table[pos, i]), float(table[pos, half + i])
        a, b = x[..., lo].copy(), x[..., hi].copy()
        x[..., lo], x[..., hi] = a * c - b * s, b * c + a * s
    return x


def tokens(starts, lens):
    """(request, packed row, logical position) of every new token, in order."""
    for b in range(len(lens)):
        n = int(starts[b + 1] - starts[b])
        for i in range(n):
            yield b, int(starts[b]) + i, int(lens[b]) - n + i


def slots(starts, lens, table, bt):
    """The same with the token's page and its row there."""
    for b, t, p in tokens(starts, lens):
        yield b, t, p, int(table[b][p // bt]), p % bt


def page_scales(x, starts, lens, table, bt, kind, old):
    """Scales [P][heads] of one layer after x [T][heads][d] (rotated) was appended, from those before."""
    new = np.array(old, dtype=np.float64)
    seen = {}
    for b, t, p, page, row in slots(starts, lens, table, bt):
        first = seen.setdefault(page, row)
        most = np.abs(x[t]).max(-1)
        most = np.where(most < 2.0 ** -100, 0.0, most / TOP[kind])
        if first == row:
            new[page] = most if row == 0 else np.maximum(old[page], most)
        else:
            new[page] = np.maximum(new[page], most)
    return new


def attention(q, k, v, starts, lens, table, bt, scale, causal=True, sink=0, window=0):
    """q [T][q_heads][d]; k, v [P][bt][heads][d] of one layer.  -> out [T][q_heads][d], lse [T][q_heads], the weighted mean of |v| and
    the largest sum of |q||k| of a score (both per out row: what rounding errors scale with), the sum of |v| over what a row sees."""
    T, q_heads, d = q.shape
    group = q_heads // k.shape[2]
    out, lse = np.zeros((T, q_heads, d)), np.full((T, q_heads), -math.inf)
    size, worth, total = np.zeros((T, q_heads, d)), np.zeros((T, q_heads)), np.zeros((T, q_heads, d))
    for b, t, p in tokens(starts, lens):
        n = int(lens[b])
        j = np.arange(n)
        see = np.ones(n, dtype=bool)
        if causal:
            see &= j <= p
        if window:
            see &= (j > p - window) | (j < sink)
        j = j[see]
        if not len(j):
            continue
        pages, rows = np.asarray(table[b])[j // bt], j % bt
        for u in range(q_heads):
            kk, vv = k[pages, rows, u // group], v[pages, rows, u // group]
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                s = kk @ q[t, u] * scale
                m = s.max()
                w = np.exp(s - m)
                out[t, u] = (w[:, None] * vv).sum(0) / w.sum()
                lse[t, u] = m + math.log(w.sum()) if np.isfinite(m) else math.nan
                size[t, u] = (w[:, None] * np.abs(vv)).sum(0) / w.sum()
                worth[t, u] = (np.abs(kk) @ np.abs(q[t, u])).max() * abs(scale)
                total[t, u] = np.abs(vv).sum(0)
    return out, lse, size, worth, total
