"""Head norms with the position rotation, float64.

    x' = x * w / sqrt(mean(x^2) + eps)                 (w given; else x' = x)
    (y0, y1) = x' pair turned by positions[axis of the pair][t] * inv_freq[pair]

Pairs are elements (i, i + rot/2), or (2i, 2i + 1) when adjacent; elements past
rot are x'.  With three axes, sections give the pairs of each axis in order;
strided, pair i belongs to axis 1 if i % 3 == 1 and i < 3 * sections[1], to
axis 2 if i % 3 == 2 and i < 3 * sections[2], else to axis 0.

Test infrastructure only; shares no code with the HIP path.
"""
from __future__ import annotations

import numpy as np


def pair_axes(half: int, sections=None, strided: bool = False) -> np.ndarray:
    if sections is None or len(sections) == 1:
        return np.zeros(half, dtype=np.int64)
    if not strided:
        return np.concatenate([np.full(n, a, dtype=np.int64) for a, n in enumerate(sections)])
    axes = np.zeros(half, dtype=np.int64)
    axes[1:3 * sections[1]:3] = 1
    axes[2:3 * sections[2]:3] = 2
    return axes


def head_norm(x: np.ndarray, weight, eps: float) -> np.ndarray:
    if weight is None:
        return np.array(x, dtype=np.float64)
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * weight


def rotate(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray, sections=None, adjacent=False,
           strided=False) -> np.ndarray:
    """x [T, heads, d], positions [axes, T], inv_freq [rot/2] (all exact float64 / int64)."""
    half = len(inv_freq)
    axes = pair_axes(half, sections, strided)
    y = np.array(x, dtype=np.float64)
    for i in range(half):
        a = positions[axes[i]].astype(np.float64) * inv_freq[i]
        p, q = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        y[..., p] = x[..., p] * c - x[..., q] * s
        y[..., q] = x[..., q] * c + x[..., p] * s
    return y
