"""fp64 oracle of serving many requests over one pool of cache pages: the bookkeeping of a step, attention over pages, low-rank adapters.
Plain Python and numpy from the definitions, one request and one token at a time; shares nothing with the library."""
from __future__ import annotations

import numpy as np


def pages_assign(free, count, table, page_rows, lengths, change, max_tokens):
    """Lists and a [batch][cols] table, changed in place.  -> (count, lengths, granted, starts, slots, positions, owners)"""
    cols, n_pages = len(table[0]), len(free)
    need = lambda rows: -(-rows // page_rows)
    lens = [min(max(n, 0), cols * page_rows) for n in lengths]
    count = min(max(count, 0), n_pages)
    granted = [0] * len(lens)
    for b, (n, c) in enumerate(zip(lens, change)):           # pages that are no longer needed
        if c < 0:
            granted[b] = max(c, -n)
            for col in range(need(n + granted[b]), need(n)):
                if count < n_pages:
                    free[count] = table[b][col]
                    count += 1
                table[b][col] = -1
    slots, positions, owners, starts = [], [], [], [0]
    wanted, there = 0, count
    for b, (n, c) in enumerate(zip(lens, change)):           # pages for new rows
        c = max(c, 0)
        end = starts[-1] + c
        ok = c > 0 and n + c <= cols * page_rows and end <= max_tokens
        if ok:
            take = need(n + c) - need(n)
            wanted += take
            ok = take == 0 or wanted <= there
            if ok:
                granted[b] = c
                for col in range(need(n), need(n + c)):
                    count -= 1
                    table[b][col] = free[count]
        for j in range(min(end, max_tokens) - min(starts[-1], max_tokens)):
            row = n + j
            page = table[b][row // page_rows] if ok else -1
            slots.append(page * page_rows + row % page_rows if 0 <= page < n_pages else -1)
            positions.append(row)
            owners.append(b)
        starts.append(end)
    pad = max_tokens - len(slots)
    return (count, [n + g for n, g in zip(lens, granted)], granted, [min(s, max_tokens) for s in starts], slots + [-1] * pad,
            positions + [0] * pad, owners + [-1] * pad)


def rows_of(pages, table, length, page_rows):
    """The rows of one request: pages [n_pages, heads, rows, dh] -> [heads, length, dh]"""
    if length == 0:
        return np.zeros((pages.shape[1], 0, pages.shape[3]))
    return np.stack([pages[table[r // page_rows], :, r % page_rows] for r in range(length)], 1)


def attention(q, k, v, table, lengths, scale):
    """q [B,Hq,dh]; k, v [n_pages,Hkv,P,dh].  -> (out [B,Hq,dh], sum_j P |v|, what rounding errors are measured in)"""
    B, Hq, dh = q.shape
    Hkv, P = k.shape[1:3]
    out, mag = np.zeros((B, Hq, dh)), np.zeros((B, Hq, dh))
    for b in range(B):
        n = lengths[b]
        if n <= 0:
            continue
        kr, vr = rows_of(k, table[b], n, P), rows_of(v, table[b], n, P)
        for h in range(Hq):
            g = h // (Hq // Hkv)
            s = (kr[g] @ np.asarray(q[b, h], np.float64)) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[b, h], mag[b, h] = p @ vr[g], p @ np.abs(vr[g])
    return out, mag


def adapters(x, base, a, b, scale, ids, part_end, rank):
    """-> (y, sums of magnitudes of the two products: of the first pushed through |b|, of the second)"""
    x, y = np.asarray(x, np.float64), np.array(base, np.float64)
    first, second = np.zeros_like(y), np.zeros_like(y)
    for m, i in enumerate(ids):
        if not 0 <= i < a.shape[0]:
            continue
        lo = 0
        for p, hi in enumerate(part_end):
            ap, bp = np.asarray(a[i, p * rank:(p + 1) * rank], np.float64), np.asarray(b[i, lo:hi], np.float64)
            t = ap @ x[m]
            y[m, lo:hi] += scale[i] * (bp @ t)
            first[m, lo:hi] = abs(scale[i]) * (np.abs(bp) @ (np.abs(ap) @ np.abs(x[m])))
            second[m, lo:hi] = abs(scale[i]) * (np.abs(bp) @ np.abs(t))
            lo = hi
    return y, first, second
