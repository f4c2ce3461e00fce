"""CPU oracle of the position rotation of include/bq4.h (test infrastructure only): plain numpy in extended precision.

Pins: tests/test_rotary_host.py (exact quarter turns, complex products, composition of turns, planted mistakes)."""
from __future__ import annotations

import numpy as np


def turn(x: np.ndarray, positions: np.ndarray, frequencies: np.ndarray, axis_of_pair: np.ndarray, interleaved: bool) -> np.ndarray:
    """x [rows, heads, dim] (float64), positions [axes, rows] -> the same with the pairs of the first 2 len(frequencies) elements turned."""
    y = np.array(x, np.float64)
    pairs = len(frequencies)
    for i in range(pairs):
        a = positions[axis_of_pair[i]].astype(np.longdouble) * np.longdouble(frequencies[i])
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        u, v = x[:, :, p].astype(np.longdouble), x[:, :, q].astype(np.longdouble)
        y[:, :, p] = u * c - v * s
        y[:, :, q] = v * c + u * s
    return y
