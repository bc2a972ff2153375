"""CPU oracle for the paged key-value cache: rotation, append, attention of one new token.  TEST
INFRASTRUCTURE ONLY (same rules as verify_oracle.py).  float64, one sequence and one head at a time."""
from __future__ import annotations

from typing import Sequence

import numpy as np


def rotate(x: np.ndarray, pos: int, theta: float) -> np.ndarray:
    """RoPE with rotate-half pairs (verify_oracle.py's reading Q6), x [..., d] at position pos."""
    d = x.shape[-1]
    angle = pos * theta ** (-2.0 * np.arange(d // 2) / d)
    a, b = x[..., :d // 2], x[..., d // 2:]
    return np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], axis=-1)


def visible(length: int, window: int, n_sink: int) -> np.ndarray:
    j = np.arange(length)
    return j if window == 0 else j[(j < n_sink) | (j >= length - window)]


def attend(q: np.ndarray, k_pool: np.ndarray, v_pool: np.ndarray, table: Sequence[int], length: int, scale: float,
           window: int = 0, n_sink: int = 0):
    """q [heads, d], pools [pages, kv heads, page size, d] -> (out [heads, d], lse [heads], largest sum |q k| scale).
    Rows of pages outside the pool are not visible."""
    n_pages, n_kv, size, d = k_pool.shape
    rows = [(table[j // size], j % size) for j in visible(length, window, n_sink)]
    rows = [(p, r) for p, r in rows if 0 <= p < n_pages]
    out, lse, reach = np.zeros(q.shape), np.full(q.shape[0], -np.inf), 0.0
    if not rows:
        return out, lse, reach
    p, r = np.array(rows).T
    for h in range(q.shape[0]):
        hk = h // (q.shape[0] // n_kv)
        k, v = k_pool[p, hk, r], v_pool[p, hk, r]
        s = scale * (k @ q[h])
        reach = max(reach, float(abs(scale) * np.max(np.abs(k) @ np.abs(q[h]))))
        w = np.exp(s - s.max())
        out[h], lse[h] = w @ v / w.sum(), s.max() + np.log(w.sum())
    return out, lse, reach
