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


# ---- quantised pages: every 64 dimensions of a row share a step and a lowest value

GROUP = 64


def _bf16(x, up):
    """fp32 -> the next bf16 value not below (up) or not above it, as fp32."""
    bits = np.ascontiguousarray(x, np.float32).view(np.uint32)
    cut = bits & np.uint32(0xffff0000)
    away = (cut != bits) & ((bits >> 31 == 0) == up)
    return (cut + np.where(away, np.uint32(0x10000), np.uint32(0))).view(np.float32)


def quantise(x, bits):
    """fp32 rows [..., d] -> (codes uint8 [..., d / 64, 64], step, low fp32 [..., d / 64]); every operation an fp32 one.  A group with a
    NaN or an element of magnitude 2^126 or more has step = low = NaN (and codes of 0 here)."""
    x = np.asarray(x, np.float32)
    x = x.reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    with np.errstate(invalid="ignore", over="ignore"):
        fine = (np.abs(x) < np.float32(2.0 ** 126)).all(-1)        # False for NaN
        safe = np.where(fine[..., None], x, np.float32(0))
        low = _bf16(safe.min(-1), False) + np.float32(0)           # a zero counts as +0
        step = _bf16((safe.max(-1) - low) * (np.float32(1) / np.float32((1 << bits) - 1)), True)
        step = np.maximum(step, np.float32(2.0 ** -126))
        code = np.rint((safe - low[..., None]) * (np.float32(1) / step)[..., None])
    nan = np.float32(np.nan)
    return code.astype(np.uint8), np.where(fine, step, nan), np.where(fine, low, nan)


def held(code, step, low):
    """What the codes stand for, fp64 [..., d]."""
    v = low[..., None].astype(np.float64) + step[..., None].astype(np.float64) * code
    return v.reshape(v.shape[:-2] + (v.shape[-2] * GROUP,))


def pack_page(code, step, low, bits):
    """Codes [..., rows, groups, 64] and their steps and lowest values -> the bytes of a page [..., rows * row_bytes], written bit by bit."""
    *lead, rows, groups, _ = code.shape
    d = groups * GROUP
    n = rows * d * bits // 8
    out = np.zeros(lead + [n + rows * 4 * groups], np.uint8)
    for r in range(rows):
        for g in range(groups):
            for x in range(GROUP):
                bit = (((x // 8) * groups + g) * 8 + x % 8) * bits
                out[..., r * d * bits // 8 + bit // 8] |= code[..., r, g, x] << (bit % 8)
    half = np.stack([step, low], -2).astype(np.float32)              # [..., rows, 2, groups]
    half = np.ascontiguousarray(half.view(np.uint32) >> 16, np.uint16)
    out[..., n:] = half.reshape(lead + [rows * 2 * groups]).view(np.uint8)
    return out


def unpack_page(page, rows, d, bits):
    """The inverse: (codes, step, low)."""
    groups, n = d // GROUP, rows * d * bits // 8
    lead = page.shape[:-1]
    code = np.zeros(lead + (rows, groups, GROUP), np.uint8)
    data = page[..., :n].reshape(lead + (rows, d * bits // 8))
    for g in range(groups):
        for x in range(GROUP):
            bit = (((x // 8) * groups + g) * 8 + x % 8) * bits
            code[..., g, x] = data[..., bit // 8] >> (bit % 8) & ((1 << bits) - 1)
    half = np.ascontiguousarray(page[..., n:]).view(np.uint16).reshape(lead + (rows, 2, groups)).astype(np.uint32) << 16
    half = half.view(np.float32)
    return code, half[..., 0, :], half[..., 1, :]


def rope_fp32(x, positions, sections, order, pairing, theta):
    """rope() as the quantised pages define it: x fp32 [tokens][heads][D]; the angle in 64-bit fixed point, cosine and sine rounded to
    fp32, two products and their sum rounded one by one.  The result is still to be rounded to the cache's type."""
    half = sum(sections)
    ax = axes(sections, order)
    x = np.asarray(x, np.float32)
    y = x.copy()
    for i in range(half):
        freq = int(theta ** (-i / half) / 6.283185307179586476925 * 18446744073709551616.0)
        turn = [(int(p) * freq + (1 << 63)) % (1 << 64) - (1 << 63) for p in positions[ax[i]]]
        angle = np.array(turn, np.float64) * (np.pi * 2.0 ** -63)
        c, s = np.cos(angle).astype(np.float32)[:, None], np.sin(angle).astype(np.float32)[:, None]
        a, b = (i, i + half) if pairing == 0 else (2 * i, 2 * i + 1)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y
