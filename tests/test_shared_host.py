"""Attention behind a shared prefix without a GPU: refusals before any device is touched, and pins of its oracle."""
import ctypes
import math
import os

import numpy as np
import torch

from oracle import shared_oracle as so

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_refusals_need_no_device(bq):
    from paper_2407_19775_b200 import kvcache
    L, cb = kvcache._lib(), bq.Codebook4()
    at = lambda n: ctypes.c_void_p(n)                                # noqa: E731

    def cache(**change):
        f = dict(k_codes=256, v_codes=256, k_scale=256, v_scale=256, table=256, lens=256, n_pages=8, kv_heads=2, page=16, head_dim=128, block=64, n_seq=2,
                 max_pages=4, table_stride=4)
        f.update(change)
        return ctypes.byref(kvcache._Cache(*f.values()))

    def call(c=None, p=None, cb=cb.handle, members=None, q=at(1 << 20), dt=1, qs=512, starts=None, n=2, heads=4, new=1, sm=0.1, w=None, ws_=64, out=at(1 << 22), ws=at(1 << 24),
             size=1 << 30, path=0):
        return L.bqkv_attend_shared(cache() if c is None else c, cache(n_seq=1) if p is None else p, cb, members, q, dt, qs, starts, n, heads, new, 0, 0, 0, sm, w, ws_, out, ws,
                                    size, path, None)

    for change, code in ((dict(head_dim=0), 4), (dict(block=12), 3), (dict(kv_heads=0), 4), (dict(page=0), 4), (dict(n_seq=0), 4), (dict(table_stride=3), 4), (dict(lens=None), 1),
                         (dict(k_codes=264), 4)):
        assert call(c=cache(**change)) == code and call(p=cache(**change)) == code, change
    for change in (dict(kv_heads=1), dict(head_dim=64), dict(block=32)):
        assert call(p=cache(n_seq=1, **change)) == 4, change          # not the cache's rows
    assert call(p=cache()) == 1                                       # two prefixes, and nobody says whose
    assert call(dt=0) == 2 and call(cb=None) == 5 and call(n=3) == 4 and call(heads=3) == 4 and call(new=-1) == 4 and call(sm=float("nan")) == 4
    assert call(path=4) == 9 and call(q=None) == 1 and call(out=None) == 1 and call(qs=511) == 4 and call(q=at(1025)) == 4 and call(out=at(1032)) == 4
    assert call(ws=None) == 7 and call(ws=at(264)) == 7 and call(size=1024) == 7
    assert call(n=0, starts=at(256), q=None) == 0
    assert call(out=at(1 << 20), w=at(256)) == 4 and call(out=at((1 << 20) + 1024), w=at(256)) == 4 and call(w=at(256), ws_=-1) == 4
    assert call(out=at((1 << 20) + 1024), path=1) == 4                # the general kernel's parts are read before, its queries are not copied
    assert call(q=at((1 << 20) + 2), path=2) == 9 and call(c=cache(page=8), path=2) == 9 and call(p=cache(n_seq=1, page=8), path=3) == 9
    size = ctypes.c_size_t()
    need = lambda c, p, n=2, heads=4, w=0, to=ctypes.byref(size): L.bqkv_attend_shared_workspace(c, p, n, heads, 1, 0, 0, 0, w, to)      # noqa: E731
    assert need(cache(), cache(n_seq=1), to=None) == 1 and need(None, cache()) == 1 and need(cache(), None) == 1 and need(cache(), cache(block=32)) == 4
    assert need(cache(), cache(), heads=3) == 4 and need(cache(), cache(), n=-1) == 4
    assert need(cache(), cache(n_seq=1)) == 0 and size.value >= 1024 + 2 * 2 * 4 * (128 + 2) * 4


def _pin(m) -> bool:
    rng = np.random.default_rng(1)
    n, length, prefix, h, g, d = 4, 9, 5, 2, 3, 8
    q, k, v, kp, vp = (rng.normal(size=s) for s in ((n, h * g, d), (length, h, d), (length, h, d), (prefix, h, d), (prefix, h, d)))
    r = m.attend(q, kp, vp, k, v, 0.3)
    tq, tk, tv = (torch.from_numpy(t) for t in (q, np.concatenate([kp, k]).repeat(g, 1), np.concatenate([vp, v]).repeat(g, 1)))
    x = torch.einsum("nhd,lhd->hnl", tq, tk) * 0.3
    hidden = torch.arange(prefix + length)[None] > (prefix + length - n + torch.arange(n))[:, None]
    p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
    ok = np.allclose(r["out"], torch.einsum("hnl,lhd->nhd", p, tv).numpy(), rtol=1e-12, atol=1e-14)
    ok &= np.allclose(r["weights"], p.sum(1).view(h, g, -1).sum(1)[:, prefix:].numpy(), rtol=1e-12, atol=1e-14)
    few = m.attend(q, kp, vp, k[:2], v[:2], 0.3)                     # two rows without a slot of their own: the prefix alone
    alone = torch.softmax(x[:, :2, :prefix], -1)
    ok &= np.allclose(few["out"][:2], torch.einsum("hnl,lhd->nhd", alone, tv[:prefix]).numpy(), rtol=1e-12, atol=1e-14)
    none = m.attend(q, kp[:0], vp[:0], k[:2], v[:2], 0.3)
    return bool(ok and np.all(none["out"][:2] == 0) and np.allclose(none["out"][2], np.repeat(v[0], g, 0)))


def test_oracle_and_planted_mistakes():
    import types
    text = open(os.path.join(ROOT, "oracle", "shared_oracle.py")).read()
    assert _pin(so)
    for old, new in (("max(length - n + i + 1, 0)", "max(length - n + i, 0)"), ("p[len(kp):]\n            heavy", "p[:own]\n            heavy"), ("k[:own]", "k"),
                     ("if len(keys) == 0", "if own == 0")):
        m = types.ModuleType("planted")
        assert text.count(old) >= 1, old
        exec(compile(text.replace(old, new), "planted", "exec"), m.__dict__)
        try:
            caught = not _pin(m)
        except Exception:
            caught = True
        assert caught, old
