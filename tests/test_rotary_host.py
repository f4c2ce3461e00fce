"""The store with positions without a GPU: refusals before any device is touched, and pins of its oracle."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import rotary_oracle as ro
from paper_2407_19775_b200.binding import BqError

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_handle_refusals(bq):
    from paper_2407_19775_b200 import kvcache
    L, out = kvcache._lib(), ctypes.c_void_p()
    f = np.ones(128)
    of = np.zeros(128, np.int32)

    def make(dim=128, f=f, of=None, axes=1, to=ctypes.byref(out)):
        return L.bqkv_make_rotary(dim, None if f is None else f.ctypes.data, None if of is None else of.ctypes.data, axes, 0, to)

    assert make(to=None) == 1 and make(f=None) == 1 and make(axes=2) == 1
    assert make(dim=0) == 4 and make(dim=3) == 4 and make(dim=258) == 4 and make(axes=0, of=of) == 4 and make(axes=256, of=of) == 4
    for bad in (np.nan, np.inf, 65537.0, -65537.0):
        g = f.copy()
        g[63] = bad
        assert make(f=g) == 4
        g[63], g[64] = 1.0, bad                                      # behind the pairs that turn: not looked at
        assert make(f=g) == 0 and L.bqkv_free_rotary(out) == 0
    for bad in (-1, 2):
        o = of.copy()
        o[5] = bad
        assert make(of=o, axes=2) == 4
    assert out.value is None or make() == 0
    assert L.bqkv_free_rotary(None) == 0
    for kw in (dict(dim=7), dict(dim=8, base=0.0), dict(dim=8, base=float("nan")), dict(dim=8, frequencies=[1.0] * 3), dict(dim=8, sections=[1, 2]),
               dict(dim=8, sections=[5, -1]), dict(dim=8, axes=[0, 1, 0]), dict(dim=8, axes=[0, 1, 0, -1]), dict(dim=8, sections=[4], axes=[0] * 4), dict(dim=512)):
        with pytest.raises(BqError):
            bq.Rotary(**kw)
    r = bq.Rotary(16, sections=[2, 3, 3])
    assert r.axes == 3 and np.allclose(r.frequencies, 10000.0 ** (-np.arange(8) / 8))
    assert bq.Rotary(16, axes=[0, 1, 2, 0, 1, 2, 0, 1]).axes == 3 and bq.Rotary(16).axes == 1


def test_call_refusals_need_no_device(bq):
    from paper_2407_19775_b200 import kvcache
    L, cb = kvcache._lib(), bq.Codebook4()
    one, rot, rot3 = ctypes.c_void_p(1 << 20), bq.Rotary(128), bq.Rotary(128, sections=[16, 24, 24])
    at = lambda n: ctypes.c_void_p(n)                                # noqa: E731

    def cache(**change):
        f = dict(k_codes=256, v_codes=256, k_scale=256, v_scale=256, table=256, lens=256, n_pages=8, kv_heads=2, page=16, head_dim=128, block=64, n_seq=2,
                 max_pages=4, table_stride=4)
        f.update(change)
        return ctypes.byref(kvcache._Cache(*f.values()))

    def call(c=None, cb=cb.handle, rot=rot.handle, q=one, k=at(1 << 22), v=at(1 << 23), dt=1, qs=512, ks=256, vs=256, heads=4, pos=None, ps=0, starts=None, n=2,
             out=at(1 << 24), os_=512):
        return L.bqkv_append_rotary(cache() if c is None else c, cb, rot, q, k, v, dt, qs, ks, vs, heads, pos, ps, starts, n, out, os_, None)

    assert call(dt=0) == 2 and call(c=cache(block=12)) == 3 and call(c=cache(lens=None)) == 1 and call(c=cache(head_dim=132)) == 4
    assert call(cb=None) == 5 and call(rot=None) == 1 and call(c=cache(head_dim=64, block=64)) == 4      # more turned elements than a row has
    assert call(n=3) == 4 and call(n=-1) == 4 and call(heads=-1) == 4 and call(heads=65536) == 4
    assert call(k=None) == 1 and call(v=None) == 1 and call(q=None) == 1 and call(out=None) == 1
    assert call(qs=511) == 4 and call(ks=255) == 4 and call(vs=255) == 4 and call(os_=511) == 4
    assert call(q=at(1025)) == 4 and call(k=at(1025)) == 4 and call(v=at(1025)) == 4 and call(out=at(1025)) == 4
    assert call(pos=at(1026)) == 4 and call(rot=rot3.handle, pos=at(1024), ps=1) == 4
    assert call(n=0, starts=one, k=None, q=None) == 0
    # outputs over inputs: q_out is q with q's stride, or meets nothing
    base = 1 << 20
    assert call(out=at(base), os_=600) == 4 and call(out=at(base + 2)) == 4 and call(out=at(base + 2 * 512)) == 4 and call(out=at(base - 2 * 512)) == 4
    assert call(out=at(1 << 22)) == 4 and call(out=at((1 << 23) + 512)) == 4
    assert call(qs=1024, ks=1024, q=at(base), k=at(base + 1024), out=at(base + 1024), os_=1024) == 4     # over k, in a fused projection
    assert call(qs=1024, ks=1024, q=at(base), k=at(base + 1022), out=at(base), os_=1024) == 4            # in place, but k begins inside q


def test_rows_that_interleave_are_told_from_rows_that_meet():
    """rows_meet's rule, restated, against sets of bytes."""
    def meet(x, xs, xn, y, ys, yn, n):
        d, x1, y1 = y - x, xs * (n - 1) + xn, ys * (n - 1) + yn
        if d >= x1 or -d >= y1:
            return False
        if xs != ys or n == 1:
            return True
        off = d % xs
        i = (d - off) // xs
        if off < xn and -(n - 1) <= i <= n - 1:
            return True
        return off + yn > xs and -(n - 1) <= i + 1 <= n - 1

    rng = np.random.default_rng(0)
    for _ in range(4000):
        n, xs = int(rng.integers(1, 5)), int(rng.integers(2, 12))
        xn, yn, y = int(rng.integers(1, xs + 1)), int(rng.integers(1, xs + 1)), int(rng.integers(-40, 60))
        rows = lambda a, w: {a + i * xs + j for i in range(n) for j in range(w)}      # noqa: E731
        assert meet(0, xs, xn, y, xs, yn, n) == bool(rows(0, xn) & rows(y, yn))


def _pin(m) -> bool:
    rng = np.random.default_rng(1)
    x = rng.normal(size=(6, 2, 12))
    f = np.array([np.pi / 2, 1.0, 1e-3, 0.25])                       # four pairs: eight of the twelve elements turn
    pos = np.array([[0, 1, 2, 3, -1, 1000003], [5, 0, -7, 1, 2, 3]])
    of = np.array([0, 1, 0, 1])
    ok = True
    for inter in (False, True):
        y = m.turn(x, pos, f, of, inter)
        at = lambda t: (t[..., :8].reshape(6, 2, 4, 2) if inter else t[..., :8].reshape(6, 2, 2, 4).transpose(0, 1, 3, 2))      # noqa: E731
        z, w = at(x)[..., 0] + 1j * at(x)[..., 1], at(y)[..., 0] + 1j * at(y)[..., 1]
        ok &= np.allclose(w, z * np.exp(1j * (pos[of] * f[:, None]).T)[:, None], atol=1e-9) and np.array_equal(y[..., 8:], x[..., 8:])
        ok &= np.allclose(w[1, :, 0], 1j * z[1, :, 0]) and np.allclose(w[2, :, 0], -z[2, :, 0])      # quarter and half turns
        ok &= np.allclose(m.turn(m.turn(x, pos, f, of, inter), -pos, f, of, inter), x, atol=1e-12)
    return bool(ok)


def test_oracle_and_planted_mistakes():
    import types
    text = open(os.path.join(ROOT, "oracle", "rotary_oracle.py")).read()
    assert _pin(ro)
    for old, new in (("u * c - v * s", "u * c + v * s"), ("v * c + u * s", "v * c - u * s"), ("i + pairs", "i + pairs + 1"), ("axis_of_pair[i]", "0"),
                     ("2 * i, 2 * i + 1", "i, i + 1"), ("np.array(x, np.float64)", "np.zeros_like(x)")):
        m = types.ModuleType("planted")
        assert text.count(old) == 1
        exec(compile(text.replace(old, new), "planted", "exec"), m.__dict__)
        assert not _pin(m), old
