"""Oracle for rotary positions with several axes, in float64.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

Pair i of a head (i < half = sum of the sections) is turned by
w_i = positions[axis(i)] * theta^(-i / half):  a' = a cos w - b sin w,
b' = b cos w + a sin w.  "sectioned": axis 0 has the first sections[0]
frequencies, axis 1 the next ones and so on; "interleaved": frequency i
belongs to axis i mod A if i < A * sections[that axis], to axis 0 otherwise.
"halves" pairs values (i, half + i), "adjacent" (2i, 2i + 1).  Values past
2 * half are copied.
"""
from __future__ import annotations

from typing import List, Sequence

import numpy as np


def axes_of(sections: Sequence[int], order: str) -> List[int]:
    half, A = sum(sections), len(sections)
    if order == "interleaved":
        return [i % A if i < A * sections[i % A] else 0 for i in range(half)]
    return [a for a, n in enumerate(sections) for _ in range(n)]


def rotate(x: np.ndarray, positions: np.ndarray, sections: Sequence[int], theta: float, order: str = "sectioned",
           pairing: str = "halves", inverse: bool = False) -> np.ndarray:
    """x [rows][heads][d], positions int [axes][rows] -> float64 [rows][heads][d]."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    half = sum(sections)
    for i, a in enumerate(axes_of(sections, order)):
        w = positions[a].astype(np.float64) * theta ** (-i / half)
        c, s = np.cos(w)[:, None], np.sin(w)[:, None] * (-1.0 if inverse else 1.0)
        u, v = (i, half + i) if pairing == "halves" else (2 * i, 2 * i + 1)
        y[..., u] = x[..., u] * c - x[..., v] * s
        y[..., v] = x[..., v] * c + x[..., u] * s
    return y
