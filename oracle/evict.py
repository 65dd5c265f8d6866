"""Attention weights added up per cache row, and eviction by them, in 64 bits with numpy -- TEST INFRASTRUCTURE, not part of the product.

Written with explicit loops from the definitions: the weight that row j of a cache receives is the sum, over the tokens that attend
and the query heads of its KV head, of the softmax weights (positions and causality as in ``attention.py``); eviction keeps the first
`sink` rows, the last `recent` rows and the heaviest of those between.  Imports nothing from the CUDA package.
"""
from __future__ import annotations

import numpy as np

from .attention import rope


def weights(q, k_cache, length: int, rope_base: float, scale: float | None = None) -> np.ndarray:
    """Weights [rows] that the tokens q [G, n, d] at cache rows length - n .. length - 1 give to rows [0, length), summed over all."""
    q, K = np.asarray(q, dtype=np.float64), np.asarray(k_cache, dtype=np.float64)[:length]
    G, n, d = q.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    K = np.stack([rope(K[j], j, rope_base) for j in range(length)])
    total = np.zeros(length)
    for i in range(n):
        last = length - n + i
        for g in range(G):
            s = scale * (K[: last + 1] @ rope(q[g, i], last, rope_base))
            e = np.exp(s - s.max())
            total[: last + 1] += e / e.sum()
    return total


def keep(mass, length: int, kept: int, sink: int, recent: int) -> list[int]:
    """Rows that stay, ascending."""
    middle = list(range(sink, length - recent))
    # heaviest first; NaN before everything; of equal ones the lower row first
    middle.sort(key=lambda j: (0, 0.0, j) if np.isnan(mass[j]) else (1, -float(mass[j]), j))
    return list(range(sink)) + sorted(middle[: kept - recent]) + list(range(length - recent, length))
