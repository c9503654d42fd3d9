"""CPU oracle of the calls with several new tokens per sequence (test infrastructure only).

Written out from the definitions in include/hardkv.h: page bookkeeping and the draft rule in exact
integers, attention in float64, one head or one sequence at a time.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16
ONE = 1 << 40


def row_end(mask_row, n_pages: int) -> int:
    """One past the highest valid slot of the newest page (its first slot if none is valid)."""
    if n_pages == 0:
        return 0
    return (n_pages - 1) * PAGE + (int(mask_row[n_pages - 1]) & 0xFFFF).bit_length()


def reserve(table, mask, n_pages, free_ids, free_top, lens, Hkv: int):
    """Slots for lens[s % len(lens)] tokens at the end of every row of sequence s, in place on copies.
    Returns (granted, table, mask, n_pages, free_top, slots) with slots[h] = the pool rows of head h's
    new tokens; on refusal everything as it was."""
    t, m, n = (np.array(x, dtype=np.int64) for x in (table, mask, n_pages))
    H, width = t.shape
    need, ends = [], []
    for h in range(H):
        k = lens[(h // Hkv) % len(lens)]
        ends.append(row_end(m[h], int(n[h])))
        need.append(max(0, -(-(ends[h] + k) // PAGE) - int(n[h])))
    total = sum(need)
    if total > free_top or any(int(n[h]) + need[h] > width for h in range(H)):
        return False, t, m, n, free_top, None
    pops = [int(x) for x in np.asarray(free_ids)[free_top - total:free_top]]
    slots = []
    for h in range(H):
        for _ in range(need[h]):
            t[h, n[h]] = pops.pop(0)
            m[h, n[h]] = 0
            n[h] += 1
        mine = []
        for j in range(ends[h], ends[h] + lens[(h // Hkv) % len(lens)]):
            m[h, j // PAGE] |= 1 << (j % PAGE)
            mine.append(int(t[h, j // PAGE]) * PAGE + j % PAGE)
        slots.append(mine)
    return True, t, m, n, free_top - total, slots


def trim(table, mask, n_pages, free_ids, free_top, drops, Hkv: int):
    """The last drops[s % len(drops)] slots of every row taken back; (table, mask, n_pages, free_ids,
    free_top)."""
    t, m, n = (np.array(x, dtype=np.int64) for x in (table, mask, n_pages))
    free = np.array(free_ids, dtype=np.int64)
    top = int(free_top)
    for h in range(t.shape[0]):
        d = int(drops[(h // Hkv) % len(drops)])
        if d <= 0:
            continue
        end = max(0, row_end(m[h], int(n[h])) - d)
        keep = -(-end // PAGE)
        for p in range(keep, int(n[h])):
            free[top] = t[h, p]
            top += 1
            t[h, p], m[h, p] = -1, 0
        if end % PAGE:
            m[h, keep - 1] &= (1 << (end % PAGE)) - 1
        n[h] = keep
    return t, m, n, free, top


def chunk_attn_head(q, keys, vals, valid, end: int, sm_scale: float):
    """Causal attention of one KV head's chunk: q [len, G, D], the row's slots keys, vals [S, D], valid
    [S], end as row_end.  Returns o [len, G, D], lse [len, G], and what error bounds are made of: the
    largest sm_scale * sum_d |q_d k_d| seen [len, G] and sum_j p_j |v_j| [len, G, D]."""
    q = np.asarray(q, np.float64)
    n, G, D = q.shape
    o, absv = np.zeros((n, G, D)), np.zeros((n, G, D))
    lse, zabs = np.full((n, G), -math.inf), np.zeros((n, G))
    for i in range(n):
        see = np.nonzero(np.asarray(valid, bool)[:max(0, end - n + i + 1)])[0]
        if not len(see):
            continue
        k, v = np.asarray(keys, np.float64)[see], np.asarray(vals, np.float64)[see]
        z = sm_scale * (q[i] @ k.T)
        m = z.max(1, keepdims=True)
        e = np.exp(z - m)
        lse[i] = (m + np.log(e.sum(1, keepdims=True)))[:, 0]
        p = e / e.sum(1, keepdims=True)
        o[i], absv[i] = p @ v, p @ np.abs(v)
        zabs[i] = sm_scale * (np.abs(q[i]) @ np.abs(k).T).max(1)
    return o, lse, zabs, absv


def whole(x) -> int:
    """floor(2^40 clamp(x, 0, 1)) of a probability, NaN as 0."""
    x = float(x)
    return 0 if x != x else int(math.floor(min(max(x, 0.0), 1.0) * ONE))


def draw24(u) -> int:
    u = float(u)
    return 0 if u != u else min(max(int(math.floor(u * (1 << 24))), 0), (1 << 24) - 1)


def verify(tokens, p, q, u):
    """One sequence's chunk: tokens [len] (the last token that stands, then the drafts), p [len, V],
    q [len, V] or None, u [len].  Returns (n_accept, next_token, n_drop)."""
    n = len(tokens)
    if n == 0:
        return 0, -1, 0
    V = len(p[0])
    kept = 0
    for i in range(1, n):
        x = int(tokens[i])
        if not 0 <= x < V:
            break
        Q = ONE if q is None else whole(q[i][x])
        if not draw24(u[i]) * Q < whole(p[i - 1][x]) << 24:
            break
        kept += 1
    full = [whole(x) for x in p[kept]]
    w = full
    if kept < n - 1:
        gone = int(tokens[kept + 1])
        less = [(ONE if v == gone else 0) for v in range(V)] if q is None else [whole(x) for x in q[kept + 1]]
        w = [max(0, a - b) for a, b in zip(full, less)]
        if sum(w) == 0:
            w = full
    total = sum(w)
    if total == 0:
        return kept, -1, n - 1 - kept
    goal, run = draw24(u[0]) * total >> 24, 0
    for v, x in enumerate(w):
        run += x
        if run > goal:
            return kept, v, n - 1 - kept
    raise AssertionError("unreachable: the goal is below the total")
