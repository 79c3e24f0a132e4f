"""Plain fp64 / integer CPU statements of the paged-cache operators (include/meda.h, "paged caches"), one
function per entry point, written as loops over sequences and heads.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def n_pages_of(rows: int, page_size: int) -> int:
    return -(-rows // page_size)


def page_tables(lens, new_lens, free_pages, top, table, page_size, capacity):
    """Returns (table, free_pages, top, cu_new, slots, ok) after the change of lengths; on failure the inputs."""
    n, width = table.shape
    lens = [0] * n if lens is None else [int(x) for x in lens]
    new_lens = [int(x) for x in new_lens]
    free0, table0 = free_pages.copy(), table.copy()
    bad = table, free_pages, top, np.zeros(n + 1, np.int64), np.full(capacity, -1, np.int64), False
    if any(x < 0 or x > width * page_size for x in lens + new_lens) or not 0 <= top <= len(free_pages):
        return bad
    given = [int(table0[i, p]) for i in range(n)
             for p in range(n_pages_of(new_lens[i], page_size), n_pages_of(lens[i], page_size))]
    wanted = sum(max(0, n_pages_of(b, page_size) - n_pages_of(a, page_size)) for a, b in zip(lens, new_lens))
    fresh = sum(max(0, b - a) for a, b in zip(lens, new_lens))
    if wanted > len(given) + len(free_pages) - top or fresh > capacity or len(given) - wanted > top:
        return bad
    source = given + [int(x) for x in free0[top:]]
    table, free_pages = table.copy(), free_pages.copy()
    taken = 0
    cu, slots = [0], []
    for i in range(n):
        for p in range(n_pages_of(lens[i], page_size), n_pages_of(new_lens[i], page_size)):
            table[i, p] = source[taken]
            taken += 1
        for r in range(lens[i], new_lens[i]):
            slots.append(int(table[i, r // page_size]) * page_size + r % page_size)
        cu.append(len(slots))
    left = given[taken:]
    for j, page in enumerate(left):
        free_pages[top - 1 - j] = page
    top += max(0, taken - len(given)) - len(left)
    slots = np.array(slots + [-1] * (capacity - len(slots)), np.int64)
    return table, free_pages, top, np.array(cu, np.int64), slots, True


def page_bounds(k_rows):
    """k_rows [rows][D] -> (min, max) over the rows; a NaN wins."""
    return np.min(k_rows, axis=0), np.max(k_rows, axis=0)


def axes(sections, order):
    t, h, w = sections
    half = t + h + w
    if order == 0:
        return [0] * t + [1] * h + [2] * w
    out = [0] * half
    for i in range(half):
        if i % 3 == 1 and i < 3 * h:
            out[i] = 1
        if i % 3 == 2 and i < 3 * w:
            out[i] = 2
    return out


def rope(x, positions, sections, order, pairing, theta):
    """x [tokens][heads][D] fp64, positions [3][tokens] integers."""
    half = sum(sections)
    ax = axes(sections, order)
    y = x.copy()
    for i in range(half):
        angle = positions[ax[i]].astype(np.float64) * theta ** (-i / half)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        a, b = (i, i + half) if pairing == 0 else (2 * i, 2 * i + 1)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def page_scores(q_heads, bounds):
    """q_heads [G][D], bounds [pages][2][D] -> fp32 scores of one KV head's pages."""
    with np.errstate(invalid="ignore", over="ignore"):
        per = np.where(q_heads[:, None] >= 0, q_heads[:, None] * bounds[None, :, 1], q_heads[:, None] * bounds[None, :, 0])
        s = per.sum(-1)
        s = np.where(np.isnan(s).any(0), np.nan, s.max(0))
        return s.astype(np.float32)


def select_pages(scores, keep, n_first, n_last):
    n = len(scores)
    if n <= keep:
        return np.arange(n)
    s = scores.astype(np.float64)
    rank = np.where(np.isnan(s), np.inf, s)
    cls = np.where(np.isnan(s), 1, 0)                      # NaN above +inf, forced pages above both
    idx = np.arange(n)
    forced = (idx < n_first) | (idx >= n - n_last)
    rank[forced], cls[forced] = np.inf, 2
    order = np.lexsort((idx, -rank, -cls))
    return np.sort(order[:keep])


def attention(q_heads, k_rows, v_rows):
    """q_heads [G][D], k_rows / v_rows [rows][D] fp64 -> (out [G][D], lse [G], helper dict for error bounds)."""
    g, d = q_heads.shape
    if len(k_rows) == 0:
        return np.zeros((g, d)), np.full(g, -np.inf), dict(spread=np.zeros((g, d)), mag=np.zeros(g))
    s = q_heads @ k_rows.T / np.sqrt(d)
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    z = e.sum(-1, keepdims=True)
    p = e / z
    mag = (np.abs(q_heads) @ np.abs(k_rows).T / np.sqrt(d)).max(-1)
    return p @ v_rows, (m + np.log(z))[:, 0], dict(spread=p @ np.abs(v_rows), mag=mag)
