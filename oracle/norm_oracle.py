"""CPU oracle of the root-mean-square norm fused with the row operation (test infrastructure only).

numpy restatement of mmd_norm_rowquant in include/mmd.h: the steps that decide a code (the residual's sum, h gamma, 127 t / a)
with the roundings stated there, the factor 1 / rms in 64 bits.  Nothing here is imported by the library or its binding.
Pins: tests/test_kvcache_host.py.
"""
from __future__ import annotations

import numpy as np

from .mmd_oracle import narrow, side_columns, widen


def norm_rowquant(xbits, resbits, gbits, eps: float, dt: int, idx):
    """-> dict: h (bits), q int8, scale float64, side float64 [R, side columns], normed float64 [R, K]."""
    x, gamma = widen(xbits, dt), widen(gbits, dt)
    hbits = np.ascontiguousarray(xbits) if resbits is None else narrow((x + widen(resbits, dt)).astype(np.float32), dt)
    h = widen(hbits, dt)
    R, K = h.shape
    idx = np.asarray(idx, np.int64)
    regular = np.ones(K, bool)
    regular[idx] = False
    t = (h * gamma[None, :]).astype(np.float32)
    a = np.abs(t[:, regular]).max(axis=1).astype(np.float32) if regular.any() else np.zeros(R, np.float32)
    d = np.where(a != 0, a, np.float32(1)).astype(np.float32)
    q = np.rint(((t * np.float32(127)).astype(np.float32) / d[:, None]).astype(np.float32)).astype(np.int8)
    q[:, ~regular] = 0
    rms = 1.0 / np.sqrt((h.astype(np.float64) ** 2).mean(axis=1) + eps)
    side = np.zeros((R, side_columns(len(idx))))
    side[:, :len(idx)] = t[:, idx].astype(np.float64) * rms[:, None]
    return {"h": hbits, "q": q, "scale": a.astype(np.float64) / 127.0 * rms, "side": side, "normed": t.astype(np.float64) * rms[:, None]}
