"""Attention over a shared prefix and a cache that evicts by attention weight, in float64."""
from __future__ import annotations

import numpy as np


def row_weights(q: np.ndarray, k: np.ndarray, see: np.ndarray, lse: np.ndarray, scale: float):
    """(sum over the queries that see a key of exp(q . k * scale - lse), largest sum |q k| * scale) per key; queries
    with lse -inf add nothing, keys that a query does not see do not reach it."""
    w, size = np.zeros(len(k)), np.zeros(len(k))
    for i in range(len(q)):
        idx = np.nonzero(see[i])[0]
        if len(idx) == 0 or lse[i] == -np.inf:
            continue
        w[idx] += np.exp((k[idx] @ q[i]) * scale - lse[i])
        size[idx] = np.maximum(size[idx], np.abs(k[idx]) @ np.abs(q[i]) * scale)
    return w, size


def rows_that_stay(weights, pos, n: int, n_seen: int, n_keep: int, n_first: int, n_recent: int):
    """For every row of the smaller cache the row that it is taken from, by the rule as it is stated: rows leave one
    by one, unprotected before protected, NaN before numbers, the lighter before the heavier, the lower before the higher."""
    def goes_before(i):
        safe = pos[i] < n_first or pos[i] >= n_seen - n_recent
        w = weights[i]
        return (safe, 0.0 if safe or w != w else 1.0, 0.0 if safe or w != w else float(w), i)
    m = min(n, n_keep)
    stay = set(sorted(range(n), key=goes_before)[n - m:])
    late = [i for i in sorted(stay) if i >= m]
    return [i if i in stay else late.pop(0) for i in range(m)]
