"""Oracle of windowed serving: attention with a sliding window and sinks, and the
page and row movements of the cache. Plain numpy in fp64 / integers, one query,
page or row at a time. Test infrastructure, like the rest of this package."""
from __future__ import annotations

import numpy as np

PAGE = 64
NO_PAGES, SHARED_PAGE, BAD_INDEX = 0x40, 0x80, 0x100
BAD_KV_LEN, BAD_PAGE = 0x4, 0x8


def depths(parent, n):
    d = []
    for i in range(n):
        d.append(0 if parent[i] < 0 else d[parent[i]] + 1)
    return d


def visible(t, L, window, sinks, parent=None):
    """The slots query t sees, in increasing order."""
    if parent is None:
        p, new = L + t, [(L + a, L + a) for a in range(t + 1)]
    else:
        d = depths(parent, t + 1)
        p, new, a = L + d[t], [], t
        while a >= 0:
            new.append((L + a, L + d[a]))
            a = parent[a]
    sees = lambda pos: p - pos < window or pos < sinks  # noqa: E731
    return [s for s in range(L) if sees(s)] + sorted(s for s, pos in new if sees(pos))


def window_rows(q, rows_of, L, scale, window, sinks, g_of, parent=None, sel=()):
    """For each (t, h) of sel: (out [D], sum_j a_j |V_j| [D], lse) of one sequence.
    q: [T, Hq, D] fp64; rows_of(slots, g) -> (K [n, D], V [n, D]) fp64."""
    res = []
    for t, h in sel:
        K, V = rows_of(visible(t, L, window, sinks, parent), g_of(h))
        x = scale * (K @ q[t, h])
        m = x.max()
        w = np.exp(x - m)
        z = w.sum()
        res.append(((w / z) @ V, (w / z) @ np.abs(V), m + np.log(z)))
    return res


def reserve(table, ref, kv_len, n_new):
    """kv_reserve on copies: (table, refcount, flags)."""
    table, ref, flags = table.copy(), ref.copy(), 0
    P = table.shape[1]
    start = ref.copy()
    free = [p for p in range(len(ref)) if ref[p] == 0]
    at = 0
    for b in range(table.shape[0]):
        L, n = int(kv_len[b]), int(n_new[b])
        if L < 0 or n < 0 or L + n > P * PAGE:
            flags |= BAD_KV_LEN
            continue
        if n == 0:
            continue
        span = range(L // PAGE, -(-(L + n) // PAGE))
        need, bad = [], 0
        for e in span:
            pg = table[b, e]
            if pg == -1:
                need.append(e)
            elif pg < 0 or pg >= len(ref):
                bad |= BAD_PAGE
            elif start[pg] != 1:
                bad |= SHARED_PAGE
        if bad:
            flags |= bad
            continue
        if not need:
            continue
        if at + len(need) > len(free):
            flags |= NO_PAGES
            at = len(free) + 1
            continue
        for e in need:
            table[b, e] = free[at]
            ref[free[at]] = 1
            at += 1
    return table, ref, flags


def release(table, ref, begin, end):
    table, ref, flags = table.copy(), ref.copy(), 0
    P = table.shape[1]
    for b in range(table.shape[0]):
        if begin[b] < 0 or end[b] > P * PAGE:
            flags |= BAD_KV_LEN
            continue
        for e in range(P):
            if e * PAGE < begin[b] or (e + 1) * PAGE > end[b] or table[b, e] == -1:
                continue
            if table[b, e] < 0 or table[b, e] >= len(ref):
                flags |= BAD_PAGE
                continue
            if ref[table[b, e]] > 0:
                ref[table[b, e]] -= 1
            else:
                flags |= BAD_PAGE
            table[b, e] = -1
    return table, ref, flags


def fork(table, ref, parent, kv_len, pools):
    """pools: arrays [layers, pages, 64, ...] changed in place.
    Returns (table, refcount, new lengths, flags)."""
    B, P = table.shape
    kv_len = np.asarray(kv_len)
    same = (table.copy(), ref.copy(), kv_len.copy())
    if any(q < -1 or q >= B for q in parent):
        return (*same, BAD_INDEX)
    if any(q >= 0 and not 0 <= kv_len[q] <= P * PAGE for q in parent):
        return (*same, BAD_KV_LEN)
    if ((table < -1) | (table >= len(ref))).any():
        return (*same, BAD_PAGE)
    new = np.full_like(table, -1)
    copies, taken = [], set()
    for i in range(B):
        q = int(parent[i])
        if q < 0:
            continue
        full, tail = divmod(int(kv_len[q]), PAGE)
        if tail and table[q, full] < 0:
            return (*same, BAD_PAGE)
        if q not in taken:
            taken.add(q)
            new[i] = table[q]
        else:
            new[i, :full] = table[q, :full]
            if tail:
                copies.append((i, full, int(table[q, full]), tail))
    # the holders of each page change by what the table says
    after = ref.copy()
    for p in table[table >= 0]:
        after[p] -= 1
    for p in new[new >= 0]:
        after[p] += 1
    free = [p for p in range(len(after)) if after[p] == 0]
    if len(free) < len(copies):
        return (*same, NO_PAGES)
    for (i, e, src, tail), dst in zip(copies, free):
        new[i, e] = dst
        after[dst] = 1
        for x in pools:
            x[:, dst, :tail] = x[:, src, :tail]
    return new, after, np.array([0 if q < 0 else kv_len[q] for q in parent], dtype=kv_len.dtype), 0


def prune_moves(keep, v0, n_vis, L):
    """(destination, source) slots of one sequence."""
    r = len(keep)
    return [(v0 + i, int(s)) for i, s in enumerate(keep)] + [(s - (n_vis - r), s) for s in range(v0 + n_vis, L)]
