"""Attention over selected pages, and who holds which page, from their definitions (numpy and plain lists; nothing of the GPU path).  Slow and plain on purpose."""
import math

import numpy as np

from . import serving_ref

BAD, NO_PAGES = 2, 3


def bounds(x, k_scale, starts, lens, table, bt, codes, scale):
    """x [P][bt][heads][d] float64: values, or codes, of one layer; k_scale [P][heads] or None.  -> (codes [P][heads][2][d], scale [P][heads] in 64 bits) after the
    call, from those before it."""
    codes, scale = np.array(codes), np.array(scale, dtype=np.float64)
    for b in range(len(lens)):
        n, length = int(starts[b + 1] - starts[b]), int(lens[b])
        if n == 0:
            continue
        for j in range((length - n) // bt, (length - 1) // bt + 1):
            page = int(table[b][j])
            rows = x[page, :min(bt, length - j * bt)]
            for h in range(x.shape[2]):
                y = rows[:, h]
                if not np.isfinite(y).all():
                    codes[page, h], scale[page, h] = 0, math.nan
                    continue
                a = np.abs(y).max()
                if a < 2.0 ** -100:
                    codes[page, h], scale[page, h] = 0, 0
                else:  # 127 y / a is a whole number or 2^-19 of itself away from one: 64 bits find its floor and ceiling
                    codes[page, h, 0], codes[page, h, 1] = np.floor(127 * y.min(0) / a), np.ceil(127 * y.max(0) / a)
                    scale[page, h] = a / 127
                if k_scale is not None:
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = scale[page, h] * float(k_scale[page, h])
                    scale[page, h] = s if abs(s) < 2.0 ** 128 else math.nan
    return codes, scale


def scores(q, codes, scale):
    """q [group][d], codes [n][2][d], scale [n]: the scores, numbers of 32 bits."""
    best = np.full(len(codes), -np.inf, dtype=np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        for row in np.asarray(q, dtype=np.float64):
            a = np.abs(row).max()
            fine = np.isfinite(row).all() and a >= 2.0 ** -100
            c = np.rint(127 * row / a) if fine else np.zeros_like(row)
            dots = np.maximum(c * codes[:, 0], c * codes[:, 1]).sum(-1)
            best = np.maximum(best, dots.astype(np.float32) * np.float32(a if fine else 0))
        s = best * scale.astype(np.float32)
    return np.where(np.isfinite(scale) & ~np.isnan(s), s, np.float32(np.inf))


def select(q, codes, scale, starts, lens, table, bt, count, first, last, heads, out):
    """q [T][q_heads][d]; codes [P][heads][2][d], scale [P][heads].  out [T][heads][count] with the rows of the requests' tokens filled in."""
    out = np.array(out)
    pages = len(codes)
    for b, t, p in serving_ref.tokens(starts, lens):
        n = p // bt + 1 if p >= 0 else 0
        at = np.asarray(table[b][:n], dtype=np.int64)
        there = [j for j in range(n) if 0 <= at[j] < pages]
        for h in range(heads):
            group = q.shape[1] // heads
            always = [j for j in there if j < first or j >= n - last]
            rest = [j for j in there if j not in set(always)]
            if rest:
                s = scores(q[t, h * group:(h + 1) * group], codes[at[rest], h], scale[at[rest], h])
                rest = [rest[i] for i in np.lexsort((np.arange(len(rest)), -s))]
            chosen = sorted(always + rest[:max(0, count - len(always))])
            out[t, h] = -1
            out[t, h, :len(chosen)] = chosen
    return out


def attention(q, k, v, starts, lens, table, bt, scale, lists):
    """serving_ref.attention with the tokens on each token's and head's listed pages: the same results, in the same order."""
    T, q_heads, d = q.shape
    heads = k.shape[2]
    group = q_heads // heads
    out, lse = np.zeros((T, q_heads, d)), np.full((T, q_heads), -math.inf)
    size, worth, total = np.zeros((T, q_heads, d)), np.zeros((T, q_heads)), np.zeros((T, q_heads, d))
    for b, t, p in serving_ref.tokens(starts, lens):
        for h in range(heads):
            mine = [int(x) for x in lists[t, h] if x >= 0]
            j = np.array([x * bt + r for x in mine for r in range(bt) if x * bt + r <= p], dtype=np.int64)
            if not len(j):
                continue
            pages, rows = np.asarray(table[b])[j // bt], j % bt
            kk, vv = k[pages, rows, h], v[pages, rows, h]
            for u in range(h * group, (h + 1) * group):
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


def fork(table, lens, refs, bt, parents=None, grow=None):
    """-> (table, lens, refs, status, pairs of pages to copy).  table: lists of equal length."""
    n, columns, pages = len(lens), len(table[0]), len(refs)
    room = min(columns * bt, 2 ** 31 - 128)
    parents, grow = list(range(n)) if parents is None else list(parents), [0] * n if grow is None else list(grow)
    refs, status = list(refs), [0] * n
    for row, length in zip(table, lens):
        if 0 < length <= room:
            for p in row[:-(-length // bt)]:
                if 0 <= p < pages:
                    refs[p] -= 1
    kept, wanted = [[] for _ in range(n)], [None] * n
    for b, a in enumerate(parents):
        length = lens[a] if 0 <= a < n else 0
        if a >= n or grow[b] < 0 or length < 0 or length + grow[b] > room or (a >= 0 and any(not 0 <= p < pages for p in table[a][:-(-length // bt)])):
            status[b] = BAD
            continue
        full = length // bt
        first = not any(parents[i] == a and grow[i] >= 0 and length + grow[i] <= room for i in range(b))
        kept[b] = list(table[a][:full + (1 if length % bt and first else 0)]) if a >= 0 else []
        wanted[b] = (length + grow[b], table[a][full] if length % bt and not first else -1)
        for p in kept[b]:
            refs[p] += 1
    free = [p for p in range(pages) if refs[p] == 0]
    used, out, lens_out, pairs = 0, [], [0] * n, []
    for b in range(n):
        row = []
        if wanted[b] is not None:
            need = -(-wanted[b][0] // bt) - len(kept[b])
            used += need
            if need and used > len(free):
                status[b] = NO_PAGES
                for p in kept[b]:
                    refs[p] -= 1
            else:
                fresh = free[used - need:used]
                for p in fresh:
                    refs[p] = 1
                if wanted[b][1] >= 0:
                    pairs.append((wanted[b][1], fresh[0]))
                row, lens_out[b] = kept[b] + fresh, wanted[b][0]
        out.append(row + [-1] * (columns - len(row)))
    return out, lens_out, refs, status, pairs


def compact(table, lens, refs, bt):
    """-> (table, refs, moved, status, pairs of pages to copy)."""
    columns, pages = len(table[0]), len(refs)
    room = min(columns * bt, 2 ** 31 - 128)
    used = [p for p in range(pages) if refs[p] > 0]
    holes = [p for p in range(len(used)) if refs[p] <= 0]
    moved, after, pairs = [-1] * pages, [0] * pages, []
    for p in used:
        to = p
        if p >= len(used):
            to = holes.pop(0)
            pairs.append((p, to))
        moved[p], after[to] = to, refs[p]
    out, status = [], []
    for row, length in zip(table, lens):
        bad = not 0 <= length <= room
        held = 0 if bad else -(-length // bt)
        new = [moved[p] if 0 <= p < pages else -1 for p in row[:held]]
        status.append(BAD if bad or -1 in new else 0)
        out.append(new + [-1] * (columns - held))
    return out, after, moved, status, pairs
