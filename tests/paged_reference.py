"""Plain 64-bit implementations of the paged cache's operators, for the tests.

Written from the definitions in include/occ.h, in numpy and Python integers, sharing nothing with the library."""
import math

import numpy as np


def tables(cached, fresh, table, ring, free, page, pages, rows):
    """occ_kv_tables, one request after the other; table and ring are copied."""
    table, ring = [list(r) for r in table], list(ring)
    head, count = free
    size, width = len(ring), len(table[0]) if table else 0
    lens, starts, slots, positions = [], [0], [-1] * rows, [0] * rows
    tokens = asked = taken = 0
    back = []
    for i, (c, f) in enumerate(zip(cached, fresh)):
        if f < 0:
            have = min(-(-max(c, 0) // page), width)
            back += table[i][:have]
            lens.append(0)
            starts.append(min(tokens, rows))
            continue
        start, end = tokens, tokens + f
        tokens = end
        starts.append(min(end, rows))
        if c < 0 or c + f > width * page or end > rows:
            lens.append(-1)
            continue
        have, want = -(-c // page), -(-(c + f) // page)
        asked += want - have
        if want > have and asked > count:
            lens.append(-1)
            continue
        lens.append(c + f)
        if want > have:
            for j in range(have, want):
                table[i][j] = ring[(head + asked - want + j) % size]
            taken = asked
        for u in range(f):
            p = c + u
            i_page = table[i][p // page]
            slots[start + u] = i_page * page + p % page if 0 <= i_page < pages else -1
            positions[start + u] = p
    for j, p in enumerate(back):
        if count + j < size:
            ring[(head + count + j) % size] = p
    return table, ring, lens, starts, slots, positions, [(head + taken) % size, min(count - taken + len(back), size - taken)]


def rope(x, positions, turns, interleaved, scale, inverse):
    """Turned heads of x (rows, heads, D) in 64 bits; the angles' remainders in whole numbers."""
    y = np.array(x, dtype=np.float64)
    pairs = len(turns)
    for r, pos in enumerate(positions):
        for i, t in enumerate(turns):
            part = (int(pos) * int(t)) % (1 << 64)
            if part >= 1 << 63:
                part -= 1 << 64
            a = 2 * math.pi * (part / 2.0 ** 64) * (-1 if inverse else 1)
            c, s = scale * math.cos(a), scale * math.sin(a)
            j0, j1 = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
            x0, x1 = np.array(x[r, :, j0], dtype=np.float64), np.array(x[r, :, j1], dtype=np.float64)
            y[r, :, j0], y[r, :, j1] = x0 * c - x1 * s, x1 * c + x0 * s
    return y


def attention(q, k_cache, v_cache, table, starts, lens, scale, causal, window):
    """(out, lse, mag, logit, seen): mag: sum p |v| / sum p; logit: the largest sum |q| |k| scale of a row; seen: keys
    of a row, -1 for rows of no request."""
    rows, Hq, D = q.shape
    pages, page, Hkv, _ = k_cache.shape
    out = np.full((rows, Hq, D), np.nan)
    lse, mag = np.full((rows, Hq), np.nan), np.zeros((rows, Hq, D))
    logit, seen = np.zeros((rows, Hq)), np.full(rows, -1)
    group = Hq // Hkv
    for i, n in enumerate(lens):
        a = min(max(starts[i], 0), rows)
        b = min(max(starts[i + 1], a), rows)
        n = min(max(n, 0), len(table[i]) * page)
        ids = np.array([table[i][j // page] for j in range(n)], dtype=np.int64)
        offs = np.arange(n) % page
        good = (ids >= 0) & (ids < pages)
        safe = np.where(good, ids, 0)
        keys, values = k_cache[safe, offs], v_cache[safe, offs]   # (n, Hkv, D)
        for r in range(a, b):
            pos = n - (b - a) + (r - a)
            j = np.arange(n)
            see = good & ((j <= pos) if causal else True) & ((j > pos - window) if window else True)
            seen[r] = see.sum()
            out[r], lse[r] = 0.0, -np.inf
            if not see.any():
                continue
            for h in range(Hq):
                k, v = keys[see, h // group], values[see, h // group]
                x = (k @ q[r, h]) * scale
                m = x.max()
                p = np.exp(x - m)
                with np.errstate(invalid="ignore"):
                    out[r, h] = (p[:, None] * v).sum(0) / p.sum()
                    mag[r, h] = (p[:, None] * np.abs(v)).sum(0) / p.sum()
                lse[r, h] = m + math.log(p.sum())
                logit[r, h] = (np.abs(k) @ np.abs(q[r, h])).max() * scale
    return out, lse, mag, logit, seen
