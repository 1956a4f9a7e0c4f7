"""A cache in pages, in fp64 numpy, written from the formulas: rows through a table, bounds of a page's keys, scores of pages, their selection,
attention over any set of rows."""
from __future__ import annotations

import math

import numpy as np


def places(table_row, page: int, n_pages: int, rows: int):
    """(page, row within it, whether there is one) of rows 0 .. rows - 1 of a sequence."""
    j = np.arange(rows)
    number = np.where(j // page < len(table_row), np.asarray(table_row)[np.minimum(j // page, len(table_row) - 1)], -1)
    return number, j % page, (number >= 0) & (number < n_pages)


def in_order(bits: np.ndarray) -> np.ndarray:
    """bf16 bits as whole numbers in the order -NaN < -infinity .. -0 < +0 .. +infinity < NaN."""
    x = bits.astype(np.int64)
    return np.where(x & 0x8000, -(x & 0x7FFF) - 1, x)


def bounds(bits: np.ndarray):
    """Least and largest of key rows [rows, D] (bf16 bits) in every dim, as bits."""
    at_least, at_most = in_order(bits).argmin(axis=0), in_order(bits).argmax(axis=0)
    d = np.arange(bits.shape[1])
    return bits[at_least, d], bits[at_most, d]


def attention(q, K, V, seen, pos: int, scale: float, cap: float = 0.0, slope: float = 0.0):
    """One query row over the rows `seen` (numbers, any order) of K, V (f64): (out, lse, scores, sizes of their terms); no row: (0, -inf, ..)."""
    if not len(seen):
        return np.zeros(q.shape[-1]), -math.inf, np.zeros(0), np.zeros(0)
    k = K[seen]
    s = scale * (k @ q)
    size = abs(scale) * (np.abs(k) @ np.abs(q)) + abs(slope) * np.abs(pos - seen)
    if cap > 0:
        s = cap * np.tanh(s / cap)
    s = s - slope * np.abs(pos - seen)
    m = s.max()
    p = np.exp(s - m)
    return (p / p.sum()) @ V[seen], m + math.log(p.sum()), s, size


def page_scores(q, k_min, k_max, scale: float, agg: str):
    """q [G, D], bounds [pages, D] (f64, finite): (scores, sizes of their terms) [pages]."""
    x = scale * np.maximum(q[:, None] * k_min, q[:, None] * k_max).sum(axis=-1)
    size = abs(scale) * np.maximum(np.abs(q[:, None] * k_min), np.abs(q[:, None] * k_max)).sum(axis=-1).max(axis=0)
    return (x.max(axis=0) if agg == "max" else x.mean(axis=0) if agg == "mean" else x[0]), size


def select(scores, last: int, k: int, keep_first: int, keep_last: int):
    """Pages of a token whose own page is `last`, out of scores [pages of the row]: k numbers, -1 behind them."""
    n = max(0, min(last + 1, len(scores)))
    j = np.arange(n)
    x = np.asarray(scores[:n], dtype=np.float64).copy()
    x[np.isnan(x) | (j < keep_first) | (j > last - keep_last)] = math.inf
    best = sorted(sorted(j.tolist(), key=lambda y: (-x[y], y))[:k])
    return np.array(best + [-1] * (k - len(best)), dtype=np.int64)


__all__ = ["places", "in_order", "bounds", "attention", "page_scores", "select"]
