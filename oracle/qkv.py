"""Plain CPU oracle for the norm and rotation of q and k heads.

TEST INFRASTRUCTURE ONLY (see ``oracle.paged_kv``).

A head's row ``x`` of ``d`` values, in fp64::

    y = x / sqrt(mean(x^2) + eps) * weight                 (no weight: y = x)
    pair i < rot/2 of y is (a, b): dims (i, i + rot/2), or (2i, 2i + 1) interleaved
    (a, b) -> (a c - b s, b c + a s)

with ``c, s = table[p, i], table[p, i + rot/2]`` and ``p`` the token's position on the
pair's axis. A position outside the table gives NaN.
"""
from __future__ import annotations

import numpy as np


def rope_table(length: int, rot: int, base: float = 10000.0) -> np.ndarray:
    """float32 [length, rot]: cosines of the rot / 2 pairs, then sines."""
    a = np.arange(length)[:, None] * base ** (-np.arange(0, rot, 2) / rot)[None, :]
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def norm_rope(x, *, weight=None, eps=0.0, table=None, positions=None, sections=None,
              interleaved=False):
    """``x`` [T, heads, d] -> (its values in fp64, the size of the terms each value sums)."""
    y = np.asarray(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    size = np.abs(y)
    if table is None:
        return y, size
    table = np.asarray(table, dtype=np.float64)
    rot = table.shape[1]
    positions = np.atleast_2d(np.asarray(positions))
    sections = (rot // 2,) if sections is None else sections
    y, size = y.copy(), size.copy()
    i = 0
    for axis, pairs in enumerate(sections):
        for _ in range(pairs):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
            p = positions[axis]
            inside = (p >= 0) & (p < len(table))
            at = np.where(inside, p, 0)
            c = np.where(inside, table[at, i], np.nan)[:, None]
            s = np.where(inside, table[at, i + rot // 2], np.nan)[:, None]
            u, v = y[..., a].copy(), y[..., b].copy()
            y[..., a], y[..., b] = u * c - v * s, v * c + u * s
            size[..., a] = np.abs(u * c) + np.abs(v * s)
            size[..., b] = np.abs(v * c) + np.abs(u * s)
            i += 1
    assert i == rot // 2, "sections must cover the pairs"
    return y, size
