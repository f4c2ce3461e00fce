"""CPU oracle of the 4-bit key/value cache: store, causal attention, accumulated weights, eviction (test infrastructure only).

Plain numpy statements of the definitions in include/bq4.h, in 64 bits apart from the codec itself (bq4_oracle).  A cache is
held here as values: per sequence two arrays [slots, heads, dim] in float64, without pages.  Nothing here is imported by the
library or its binding.  Pins: tests/test_kvcache_host.py (torch's double softmax, hand-worked evictions, planted mistakes).
"""
from __future__ import annotations

import numpy as np

from . import bq4_oracle as o4
from .mmd_oracle import narrow, widen


def store(bits: np.ndarray, dt: int, block: int, cb: np.ndarray):
    """Rows [..., dim] of 16-bit patterns -> (packed [..., dim / 2], scale bits [..., dim / block], values in float64)."""
    shape = bits.shape
    flat = np.ascontiguousarray(bits).reshape(-1)
    packed, scale = o4.quantize_s16(flat, dt, block, cb)
    vals = cb[o4.unpack(packed, flat.size)].astype(np.float64) * np.repeat(widen(scale, o4.BF16).astype(np.float64), block)
    return packed.reshape(shape[:-1] + (shape[-1] // 2,)), scale.reshape(shape[:-1] + (shape[-1] // block,)), vals.reshape(shape)


def read(values: np.ndarray, dt: int) -> np.ndarray:
    """The 16-bit patterns a read of stored values gives (the product of a 24-bit value and an 8-bit scale, rounded to fp32 first)."""
    return narrow(values.astype(np.float32), dt)


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, sm_scale: float):
    """q [n, Hq, dim], k, v [len, H, dim] of one sequence whose last n slots are the rows' own -> dict of float64 arrays:
    out [n, Hq, dim]; weights [H, len]; and for tolerances mass = sum p |v| [n, Hq, dim], spread = max over seen slots of
    sm sum |q k| [n, Hq]."""
    n, hq, dim = q.shape
    length, h, _ = k.shape
    g = hq // h
    out, mass, spread = np.zeros((n, hq, dim)), np.zeros((n, hq, dim)), np.zeros((n, hq))
    weights, heavy = np.zeros((h, length)), np.zeros((h, length))
    for i in range(n):
        seen = length - n + i + 1
        if seen <= 0:
            continue
        for j in range(hq):
            x = (k[:seen, j // g] @ q[i, j]) * sm_scale
            e = np.exp(x - x.max())
            p = e / e.sum()
            out[i, j] = p @ v[:seen, j // g]
            mass[i, j] = p @ np.abs(v[:seen, j // g])
            spread[i, j] = (np.abs(k[:seen, j // g]) @ np.abs(q[i, j])).max() * abs(sm_scale)
            weights[j // g, :seen] += p
            heavy[j // g, :seen] += p * spread[i, j]
    return {"out": out, "weights": weights, "mass": mass, "spread": spread, "heavy": heavy}


def evict_places(w: np.ndarray, length: int, budget: int, sinks: int, recent: int) -> np.ndarray:
    """For one head: place[j] = the old slot whose row ends up in slot j, j < min(length, budget)."""
    if length <= budget:
        return np.arange(length)
    middle = list(range(sinks, length - recent))
    key = {j: (-np.inf if np.isnan(w[j]) else float(w[j]), ) for j in middle}
    # heaviest first, NaN after every number, the lower slot first among equals
    ranked = sorted(middle, key=lambda j: (bool(np.isnan(w[j])), -key[j][0], j))
    stays = set(ranked[:budget - sinks - recent])
    place = list(range(budget))
    late = sorted(j for j in stays if j >= budget - recent)
    for j in range(sinks, budget - recent):
        if j not in stays:
            place[j] = late.pop(0)
    assert not late
    for i in range(recent):
        place[budget - recent + i] = length - recent + i
    return np.array(place)
