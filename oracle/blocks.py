"""The prompt's block selection and its attention over selected blocks, in float64."""
from __future__ import annotations

import numpy as np


def tile_blocks(q_tile: np.ndarray, reps: np.ndarray, p0: int, p1: int, block: int, n_first: int, n_recent: int,
                n_top: int):
    """The blocks of a tile whose queries q_tile [rows][d] are tokens p0..p1."""
    hi = p1 // block
    lo = max(0, p0 // block - n_recent)
    forced = [b for b in range(hi + 1) if b < n_first or b >= lo]
    rest = [b for b in range(hi + 1) if not (b < n_first or b >= lo)]
    qs = q_tile.astype(np.float64).sum(axis=0)
    score = {b: float(np.sum(qs * reps[b].astype(np.float64))) for b in rest}
    rank = sorted(rest, key=lambda b: (-score[b] if score[b] == score[b] else np.inf, b))
    return sorted(forced + rank[:n_top])


def masked_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, see: np.ndarray, scale: float):
    """softmax(q k^T * scale) v over the keys that see [rows][keys] allows: (out, lse, weight-mean of |v|, largest
    sum |q k| * scale); a row that sees nothing is 0 with lse -inf.  Keys that a row does not see do not reach it."""
    out = np.zeros((q.shape[0], v.shape[1]))
    lse = np.full(q.shape[0], -np.inf)
    mass = np.zeros_like(out)
    size = np.zeros(q.shape[0])
    for i in range(q.shape[0]):
        idx = np.nonzero(see[i])[0]
        if len(idx) == 0:
            continue
        x = (k[idx] @ q[i]) * scale
        top = x.max()
        if top == -np.inf:
            continue
        e = np.exp(x - top)
        p = e / e.sum()
        out[i] = p @ v[idx]
        mass[i] = p @ np.abs(v[idx])
        lse[i] = top + np.log(e.sum())
        size[i] = (np.abs(k[idx]) @ np.abs(q[i])).max() * scale
    return out, lse, mass, size
