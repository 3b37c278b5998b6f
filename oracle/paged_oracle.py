"""fp64 oracle of the paged cache: where positions lie, the bounds of a page's keys, which pages a score selects, and
attention over positions or pages.  Test infrastructure only; shares nothing with the CUDA path.
"""
from __future__ import annotations

import math

import numpy as np


def place(table, page: int, pos: int):
    """(page number, row) of a position of one sequence."""
    return int(table[pos // page]), pos % page


def rows(pool, table, page: int, n: int):
    """float64 [Hkv, n, 128]: the first n positions of one sequence, from a pool [pages, Hkv, page, 128]."""
    pages = pool[np.asarray(table[: -(-n // page)], dtype=np.int64)]           # [P, Hkv, page, 128]
    return np.asarray(pages, dtype=np.float64).transpose(1, 0, 2, 3).reshape(pool.shape[1], -1, pool.shape[3])[:, :n]


def bounds_after(old_lo, old_hi, new, joins: bool):
    """Bounds of a page and head behind an append of keys `new` [rows, 128] (NaN does not count)."""
    lo = np.where(np.isnan(new), np.inf, new).min(0)
    hi = np.where(np.isnan(new), -np.inf, new).max(0)
    return (np.minimum(lo, old_lo), np.maximum(hi, old_hi)) if joins else (lo, hi)


def scores(q, k_min, k_max):
    """q [G, 128]; k_min, k_max [P, 128].  The largest product of a query of the group with a key inside a page's bounds."""
    big = 2.0 ** 128
    lo, hi, q = (np.clip(np.asarray(x, dtype=np.float64), -big, big) for x in (k_min, k_max, q))
    best = np.full(len(lo), -np.inf)
    for h in q:
        best = np.maximum(best, np.where(h < 0, h * lo, h * hi).sum(-1))
    return best


def select(score, top: int, first: int, last: int):
    """The pages taken of len(score), ascending: the first and the last ones before all others, then by score, then the lower."""
    n = len(score)
    forced = [i < first or i >= n - last for i in range(n)]
    order = sorted(range(n), key=lambda i: (not forced[i], 0.0 if forced[i] else -score[i], i))
    return sorted(order[: min(top, n)])


def attend(q, k, v, at=None, scale=None):
    """q [Hq, 128], k and v [Hkv, n, 128]; at[g]: positions that KV head g attends (all of them where None).
    Returns out [Hq, 128] and sum_j p_j |v_j| [Hq, 128]; zeros where nothing is attended."""
    hq, hkv = len(q), len(k)
    scale = 1.0 / math.sqrt(q.shape[1]) if scale is None else scale
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(hq):
        g = h // (hq // hkv)
        sel = np.arange(k.shape[1]) if at is None else np.asarray(at[g], dtype=np.int64)
        if len(sel) == 0:
            continue
        s = k[g, sel] @ q[h] * scale
        p = np.exp(s - s.max())
        p /= p.sum()
        out[h], size[h] = p @ v[g, sel], p @ np.abs(v[g, sel])
    return out, size
