"""Paged cache and chunk attention in plain fp64 numpy, one token and one head at a time: the definitions of
include/fly_cache.h as they are written there."""
from __future__ import annotations

import math

import numpy as np


def e4m3_grid() -> np.ndarray:
    """The 127 magnitudes of e4m3 in order: eight steps to the smallest normal 2^-6, then eight per power of two up to 448."""
    return np.array([m / 8 * 2.0 ** -6 for m in range(8)] +
                    [(1 + m / 8) * 2.0 ** x for x in range(-6, 9) for m in range(8) if not (x == 8 and m == 7)])


GRID = e4m3_grid()


def to_code(y: float) -> float:
    """The e4m3 value nearest to y (|y| <= 448); of two as near, the one whose place in the grid is even."""
    a = abs(y)
    j = int(np.searchsorted(GRID, a))
    if j == 0:
        return 0.0
    lo, hi = GRID[j - 1], GRID[j] if j < len(GRID) else math.inf
    pick = j - 1 if a - lo < hi - a else j if a - lo > hi - a else (j if j % 2 == 0 else j - 1)
    return math.copysign(float(GRID[pick]), y)


def quantise_row(x) -> tuple[np.ndarray, int]:
    """Codes (as their values) and scale byte of one row of bf16 values."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return np.zeros_like(x), 255
    s = 7
    while np.abs(x).max() > 448 * 2.0 ** (s - 127):
        s += 1
    most = 240.0 if s == 247 else 448.0        # (256 * 2^120 is no bf16 number)
    return np.clip([to_code(v / 2.0 ** (s - 127)) for v in x], -most, most), s


def row_values(codes, s: int) -> np.ndarray:
    return np.full(len(codes), np.nan) if s == 255 else np.asarray(codes, dtype=np.float64) * 2.0 ** (s - 127)


def place(table_row, pos: int, page_size: int, num_pages: int):
    """(page, slot) of a position, or None."""
    if pos < 0 or pos >= len(table_row) * page_size:
        return None
    page = int(table_row[pos // page_size])
    return (page, pos % page_size) if 0 <= page < num_pages else None


def held_length(L: int, table_row, page_size: int) -> int:
    return L if 0 <= L <= len(table_row) * page_size else -1


def held_count(counts, b: int, n: int) -> int:
    if counts is None:
        return n
    return int(counts[b]) if 0 <= counts[b] <= n else 0


def visible(P: int, window: int, sinks: int):
    """Positions that the row at position P sees."""
    return [p for p in range(P + 1) if window == 0 or p > P - window or p < sinks]


def attend_row(q, keys, values, scale: float):
    """out and lse of one query over the rows that it sees."""
    if len(keys) == 0:
        return np.zeros_like(q), -math.inf
    s = scale * (keys @ q)
    top = s.max()
    if top == -math.inf:
        return np.zeros_like(q), -math.inf
    p = np.exp(s - top)
    return (p @ values) / p.sum(), top + math.log(p.sum())
