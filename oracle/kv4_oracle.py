"""Plain float64 statement of the paged 4-bit cache and the operators on it
(include/buddy.h): numpy, one entry, head and sequence at a time."""
from __future__ import annotations

import numpy as np

GROUP = 32
MAX_SCALE = 896.0


def page_plan(length, n_new, page, table, free, head):
    """(table, kv_len, row_start, slot, pos, head) after the call's new tokens."""
    table = np.array(table)
    slot, pos, starts = [], [], [0]
    for i, (n, m) in enumerate(zip(length, n_new)):
        for at in range(-(-n // page), -(-(n + m) // page)):
            table[i, at] = free[head]
            head += 1
        for p in range(n, n + m):
            slot.append(int(table[i, p // page]) * page + p % page)
            pos.append(p)
        starts.append(starts[-1] + m)
    return table, np.asarray(length) + np.asarray(n_new), np.array(starts), np.array(slot, np.int64), np.array(pos), head


def norm_rope(x, gain, pos, theta, eps):
    """x [tokens, heads, hd]: norm of each head (gain not None) and rotate-half RoPE."""
    x = np.asarray(x, np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    h = x.shape[-1] // 2
    a = np.asarray(pos, np.float64)[:, None, None] * float(theta) ** (-np.arange(h) / h)
    lo, hi = x[..., :h], x[..., h:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)


def norm_rope_axes(x, gain, pos, axis, theta, eps):
    """The same with several position axes: pos [axes, tokens], axis[j] that of frequency j."""
    out, h = np.empty(np.shape(x)), np.shape(x)[-1] // 2
    for a, p in enumerate(np.asarray(pos)):
        turned = norm_rope(x, gain, p, theta, eps)
        for j in range(h):
            if axis[j] == a:
                out[..., [j, j + h]] = turned[..., [j, j + h]]
    return out


def scale_of(amax):
    """The stored scale of a group with this largest magnitude."""
    if np.isnan(amax):
        return np.nan
    s = amax / 7.0
    if s == 0.0:
        return 0.0
    if np.isinf(s):
        return MAX_SCALE
    step = 2.0 ** (np.floor(np.log2(s)) - 6)             # the last of 7 significant bits
    s = min(np.round(s / step) * step, MAX_SCALE)
    return float(np.float16(s))


def quantise(x):
    """x [..., hd] -> (codes int [..., hd] in 1..15, scales [..., hd / 32])."""
    x = np.asarray(x, np.float64)
    grp = x.reshape(-1, GROUP)
    codes, scales = np.full(grp.shape, 8), np.zeros(len(grp))
    for i, v in enumerate(grp):
        s = scales[i] = scale_of(np.nan if np.isnan(v).any() else np.abs(v).max())
        if s > 0:
            codes[i] = np.clip(np.round(v / s), -7, 7) + 8
    return codes.reshape(x.shape), scales.reshape(*x.shape[:-1], x.shape[-1] // GROUP)


def values(codes, scales):
    return (codes - 8) * np.repeat(scales, GROUP, -1)


def pack(codes):
    """codes [..., hd] -> bytes [..., hd / 2]."""
    w = np.zeros(codes.shape[:-1] + (codes.shape[-1] // 8,), np.uint32)
    for e in range(8):
        nib = e // 2 if e % 2 == 0 else 4 + e // 2
        w |= codes[..., e::8].astype(np.uint32) << np.uint32(4 * nib)
    return np.ascontiguousarray(w.astype("<u4")).view(np.uint8)


def unpack(b):
    w = np.ascontiguousarray(b).view("<u4")
    out = np.zeros(w.shape[:-1] + (w.shape[-1] * 8,), np.int64)
    for e in range(8):
        nib = e // 2 if e % 2 == 0 else 4 + e // 2
        out[..., e::8] = (w >> np.uint32(4 * nib)) & 15
    return out


def blocks(codes, scales):
    """codes [pages, heads, page, hd] and their scales -> page bytes [pages, heads, block]."""
    n, g, page, hd = codes.shape
    sc = np.ascontiguousarray(scales.astype("<f2")).view(np.uint8).reshape(n, g, -1)
    return np.concatenate([pack(codes).reshape(n, g, -1), sc], -1)


def entries(pages, page, hd):
    """Page bytes [pages, heads, block] -> values [pages, heads, page, hd]."""
    n, g, _ = pages.shape
    cut = page * hd // 2
    codes = unpack(pages[..., :cut].reshape(n, g, page, hd // 2))
    scales = np.ascontiguousarray(pages[..., cut:]).view("<f2").reshape(n, g, page, hd // GROUP)
    return values(codes, scales.astype(np.float64))


def attention(q, k, v, n_new, scale):
    """One sequence: q [n_new, nq, hd]; k, v [heads, positions, hd]."""
    q = np.asarray(q, np.float64)
    out = np.zeros_like(q)
    group, n = q.shape[1] // k.shape[0], k.shape[1]
    for j in range(n_new):
        seen = n - n_new + j + 1
        if seen <= 0:
            continue
        for h in range(q.shape[1]):
            s = k[h // group, :seen] @ q[j, h] * scale
            p = np.exp(s - s.max())
            out[j, h] = p @ v[h // group, :seen] / p.sum()
    return out


def page_bounds(keys, page, n):
    """keys [pages, heads, page, hd] of one sequence of n positions: [pages, heads, 2, hd]."""
    out = np.empty(keys.shape[:2] + (2, keys.shape[-1]))
    for j, blk in enumerate(keys):
        held = blk[:, :n - j * page]
        out[j, :, 0], out[j, :, 1] = held.min(1), held.max(1)
    return out


def _eights(x):
    """fp32 sum over the last axis: halves onto each other inside eight neighbours, then so over the eights."""
    x = x.reshape(*x.shape[:-1], -1, 8)
    for _ in range(2):
        while x.shape[-1] > 1:
            h = x.shape[-1] // 2
            x = x[..., :h] + x[..., h:]
        x = x[..., 0]
    return x


def page_scores(q, bounds):
    """q [nq, hd] and bounds [pages, heads, 2, hd], fp32: [heads, pages], every product and sum rounded."""
    q, bounds = np.asarray(q, np.float32), np.asarray(bounds, np.float32)
    out = np.empty((bounds.shape[1], bounds.shape[0]), np.float32)
    group = len(q) // bounds.shape[1]
    with np.errstate(all="ignore"):
        for g in range(bounds.shape[1]):
            mine = q[g * group:(g + 1) * group]
            a, b = np.maximum(mine[0], 0), np.minimum(mine[0], 0)
            for x in mine[1:]:
                a, b = a + np.maximum(x, 0), b + np.minimum(x, 0)
            out[g] = _eights(a * bounds[:, g, 1]) + _eights(b * bounds[:, g, 0])
    return out


def select(score, budget, first, last):
    """Positions of the selected pages of score [pages], ascending; None for a page that is not there."""
    n = len(score)
    if n <= budget:
        return list(range(n))
    always = list(range(first)) + list(range(n - last, n))
    rank = {j: (0, 0) if score[j] is None else (2, 0) if np.isnan(score[j]) else (1, score[j]) for j in range(first, n - last)}
    best = sorted(rank, key=lambda j: (-rank[j][0], -rank[j][1], j))[:budget - first - last]
    return sorted(always + best)
