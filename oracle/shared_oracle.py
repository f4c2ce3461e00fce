"""CPU oracle of the attention behind a shared prefix (test infrastructure only): plain numpy in 64 bits, one sequence at a time.

Pins: tests/test_shared_host.py (torch's double softmax over the joined slots, planted mistakes)."""
from __future__ import annotations

import numpy as np


def attend(q, kp, vp, k, v, sm_scale: float):
    """q [n, Hq, dim]; kp, vp [prefix, H, dim]; k, v [len, H, dim], the rows' own slots the last n of them -> dict of float64 arrays as
    kvcache_oracle.attend gives them; weights and heavy of the own slots [H, len]."""
    n, hq, dim = q.shape
    length, h, _ = k.shape
    g = hq // h
    out, mass, spread = np.zeros((n, hq, dim)), np.zeros((n, hq, dim)), np.zeros((n, hq))
    weights, heavy = np.zeros((h, length)), np.zeros((h, length))
    for i in range(n):
        own = max(length - n + i + 1, 0)
        keys, values = np.concatenate([kp, k[:own]]), np.concatenate([vp, v[:own]])
        if len(keys) == 0:
            continue
        for j in range(hq):
            x = (keys[:, j // g] @ q[i, j]) * sm_scale
            e = np.exp(x - x.max())
            p = e / e.sum()
            out[i, j] = p @ values[:, j // g]
            mass[i, j] = p @ np.abs(values[:, j // g])
            spread[i, j] = (np.abs(keys[:, j // g]) @ np.abs(q[i, j])).max() * abs(sm_scale)
            weights[j // g, :own] += p[len(kp):]
            heavy[j // g, :own] += p[len(kp):] * spread[i, j]
    return {"out": out, "weights": weights, "mass": mass, "spread": spread, "heavy": heavy}
