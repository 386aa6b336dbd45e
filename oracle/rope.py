"""Norm and rotation of queries and keys in plain numpy and binary64.

TEST INFRASTRUCTURE ONLY; shares nothing with the library.
"""
from __future__ import annotations

import numpy as np


def norm(x, weight=None, eps=1e-6, offset=0.0):
    if weight is None:
        return np.asarray(x, dtype=np.float64)
    x = np.asarray(x, dtype=np.float64)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps))) * (
        np.asarray(weight, dtype=np.float64) + float(np.float32(offset)))


def rotate(x, positions, inv_freq, sections=None, interleaved=False):
    """x [T, H, D]; positions [T] or [axes, T]; turns the first 2 len(inv_freq) dims."""
    y = np.array(x, dtype=np.float64)
    F = len(inv_freq)
    axis = np.zeros(F, dtype=np.int64) if sections is None else np.repeat(np.arange(len(sections)), sections)
    pos = np.asarray(positions, dtype=np.float64).reshape(-1, y.shape[0])
    for f in range(F):
        a = pos[axis[f]] * float(inv_freq[f])
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        i, j = (2 * f, 2 * f + 1) if interleaved else (f, f + F)
        u, v = y[..., i].copy(), y[..., j].copy()
        y[..., i], y[..., j] = u * c - v * s, v * c + u * s
    return y
