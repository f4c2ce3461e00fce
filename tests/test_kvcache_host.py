"""The 4-bit key/value cache and the fused norm without a GPU: exported symbols, refusals before any device is touched, and pins
of their oracles (torch's softmax and codec in 64 bits, hand-worked evictions, planted mistakes)."""
import ctypes
import math
import os
import re

import numpy as np
import torch

from oracle import bq4_oracle as o4
from oracle import kvcache_oracle as ko
from oracle import mmd_oracle as mo
from oracle import norm_oracle as no

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_symbol_is_exported(bq):
    from paper_2407_19775_b200 import binding, kvcache
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "bq4.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(bqkv_[a-z_0-9]+)\s*\(", text))
    assert {"bqkv_append", "bqkv_read", "bqkv_attend", "bqkv_evict"} <= names == set(kvcache.SYMBOLS)
    for name in names:
        assert hasattr(binding.lib(), name), name


def test_cache_argument_errors_need_no_device(bq):
    from paper_2407_19775_b200 import kvcache
    L = kvcache._lib()
    one = ctypes.c_void_p(256)                                       # never dereferenced: every call below fails a check first
    cb = bq.Codebook4()

    def cache(**change):
        f = dict(k_codes=256, v_codes=256, k_scale=256, v_scale=256, table=256, lens=256, n_pages=8, kv_heads=2, page=16, head_dim=128, block=64, n_seq=2,
                 max_pages=4, table_stride=4)
        f.update(change)
        return ctypes.byref(kvcache._Cache(*f.values()))

    def append(c, dt=1, k=one, cb=cb.handle, n=2, stride=256, starts=None):
        return L.bqkv_append(c, cb, k, one, dt, stride, stride, starts, n, None)

    def attend(c=None, q=one, dt=1, n=2, heads=4, max_new=1, sm=0.1, w=None, ws=one, size=1 << 20, path=0, stride=512, out=one):
        return L.bqkv_attend(cache() if c is None else c, cb.handle, q, dt, stride, None, n, heads, max_new, 0, sm, w, 64, out, ws, size, path, None)

    for change, code in ((dict(head_dim=0), 4), (dict(head_dim=132), 4), (dict(head_dim=264), 4), (dict(block=12), 3), (dict(block=48), 3), (dict(block=0), 3),
                         (dict(kv_heads=0), 4), (dict(page=0), 4), (dict(n_pages=0), 4), (dict(n_seq=0), 4), (dict(n_seq=70000), 4), (dict(max_pages=0), 4),
                         (dict(table_stride=3), 4), (dict(max_pages=1 << 26, table_stride=1 << 26), 4), (dict(k_codes=None), 1), (dict(lens=None), 1),
                         (dict(table=None), 1), (dict(v_scale=264), 4), (dict(k_codes=264), 4)):
        assert append(cache(**change)) == code, change
        assert attend(cache(**change)) == code, change
        assert L.bqkv_read(cache(**change), cb.handle, None, 2, one, one, 1, None) == code, change
        assert L.bqkv_evict(cache(**change), one, 64, 8, 0, 0, one, 1 << 20, None) == code, change
    assert append(None) == 1 and append(cache(), dt=0) == 2 and append(cache(), k=None) == 1 and append(cache(), cb=None) == 5
    assert append(cache(), n=-1) == 4 and append(cache(), n=3) == 4 and append(cache(), stride=255) == 4 and append(cache(), k=ctypes.c_void_p(257)) == 4
    assert append(cache(), n=0, starts=one, k=None) == 0             # no rows: nothing to do
    assert attend(dt=0) == 2 and attend(n=3) == 4 and attend(heads=3) == 4 and attend(heads=0) == 4 and attend(max_new=-1) == 4
    assert attend(sm=float("inf")) == 4 and attend(q=None) == 1 and attend(out=None) == 1 and attend(stride=511) == 4 and attend(path=77) == 9
    assert attend(ws=None) == 7 and attend(ws=ctypes.c_void_p(264)) == 7 and attend(size=16) == 7 and attend(out=ctypes.c_void_p(258)) == 4
    assert L.bqkv_read(cache(), cb.handle, None, 2, one, None, 1, None) == 1 and L.bqkv_read(cache(), cb.handle, None, 2, one, one, 0, None) == 2
    assert L.bqkv_evict(cache(), None, 64, 8, 0, 0, one, 1 << 20, None) == 1 and L.bqkv_evict(cache(), one, 64, 0, 0, 0, one, 1 << 20, None) == 4
    assert L.bqkv_evict(cache(), one, 64, 8, 5, 4, one, 1 << 20, None) == 4 and L.bqkv_evict(cache(), one, 64, 8, 0, 0, one, 16, None) == 7
    size = ctypes.c_size_t()
    assert L.bqkv_attend_workspace(cache(), 2, 4, 1, 0, 1, None) == 1 and L.bqkv_attend_workspace(cache(), 2, 5, 1, 0, 1, ctypes.byref(size)) == 4
    assert L.bqkv_attend_workspace(cache(), 2, 4, 1, 0, 1, ctypes.byref(size)) == 0 and size.value >= 256 + 2 * 4 * 4
    assert L.bqkv_evict_workspace(cache(), 8, ctypes.byref(size)) == 0 and size.value >= 2 * 2 * 8 * 8
    assert L.bqkv_evict_workspace(cache(), 0, ctypes.byref(size)) == 4


def test_norm_argument_errors_need_no_device(bq):
    from paper_2407_19775_b200 import mmd
    L = mmd._lib()
    one, off = ctypes.c_void_p(256), ctypes.c_void_p(264)

    def norm(x=one, res=None, g=one, eps=1e-5, dt=1, R=4, K=64, ko=0, h=None, q=one, scale=one):
        return L.mmd_norm_rowquant(x, res, g, eps, dt, R, K, None, ko, h, q, scale, None, None)

    assert norm(dt=0) == 2 and norm(K=40) == 4 and norm(R=-1) == 4 and norm(ko=64) == 8 and norm(ko=3) == 1
    assert norm(R=0, x=None) == 0 and norm(x=None) == 1 and norm(g=None) == 1 and norm(res=one) == 1 and norm(q=None) == 1 and norm(scale=None) == 1
    assert norm(x=off) == 4 and norm(g=off) == 4 and norm(res=off, h=one) == 4 and norm(h=off) == 4 and norm(q=off) == 4
    assert norm(eps=-1.0) == 4 and norm(eps=float("nan")) == 4 and norm(eps=float("inf")) == 4
    assert L.mmd_norm_linear(None, one, None, one, 1e-5, 4, None, one, 1, one, 1 << 20, 0, None) == 1


def _attend_pin(m) -> bool:
    rng = np.random.default_rng(1)
    n, length, h, g, d = 4, 9, 2, 3, 8
    q, k, v = rng.normal(size=(n, h * g, d)), rng.normal(size=(length, h, d)), rng.normal(size=(length, h, d))
    r = m.attend(q, k, v, 0.3)
    tq, tk, tv = (torch.from_numpy(t) for t in (q, k.repeat(g, 1), v.repeat(g, 1)))
    x = torch.einsum("nhd,lhd->hnl", tq, tk) * 0.3
    mask = torch.arange(length)[None] > (length - n + torch.arange(n))[:, None]
    p = torch.softmax(x.masked_fill(mask, -math.inf), -1)
    ok = np.allclose(r["out"], torch.einsum("hnl,lhd->nhd", p, tv).numpy(), rtol=1e-12, atol=1e-14)
    ok &= np.allclose(r["weights"], p.sum(1).view(h, g, length).sum(1).numpy(), rtol=1e-12, atol=1e-14)
    few = m.attend(q, k[:2], v[:2], 0.3)                             # more rows than slots: the first two rows see nothing
    return ok and np.all(few["out"][:2] == 0) and np.allclose(few["out"][2], np.repeat(v[0], g, 0)) and abs(few["weights"].sum() - 2 * h * g) < 1e-9


def _evict_pin(m) -> bool:
    w = np.array([9.0, 1, 5, 5, 2, 5, 0, 7, 3, 4])
    ok = m.evict_places(w, 10, 10, 0, 0).tolist() == list(range(10))
    # sink 0; recent 8, 9; of 1..7 the three heaviest are 7 and the first two of the equal ones, 2 and 3
    ok &= m.evict_places(w, 10, 6, 1, 2).tolist() == [0, 7, 2, 3, 8, 9]
    ok &= m.evict_places(w, 10, 3, 0, 3).tolist() == [7, 8, 9] and m.evict_places(w, 10, 3, 3, 0).tolist() == [0, 1, 2]
    ok &= m.evict_places(np.array([np.nan, -1.0, 0.0, np.nan]), 4, 2, 0, 0).tolist() == [2, 1]
    return ok and m.evict_places(w, 10, 1, 0, 0).tolist() == [0]


def _norm_pin(m) -> bool:
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.normal(size=(5, 64)))
    x[:, 3] *= 20                                                    # a critical feature that would set the scale
    x = x.to(torch.bfloat16)
    res = torch.from_numpy(rng.normal(size=(5, 64))).to(torch.bfloat16)
    g = torch.from_numpy(1 + 0.1 * rng.normal(size=64)).to(torch.bfloat16)
    b = lambda t: t.view(torch.int16).numpy().view(np.uint16)        # noqa: E731
    r = m.norm_rowquant(b(x), b(res), b(g), 1e-5, mo.BF16, np.array([3, 9]))
    h = x + res
    y = h.double() / (h.double().square().mean(1, keepdim=True) + 1e-5).sqrt() * g.double()
    ok = np.array_equal(r["h"], b(h)) and np.allclose(r["normed"], y.numpy(), rtol=1e-6)
    ok &= np.allclose(r["side"][:, :2], y[:, [3, 9]].numpy(), rtol=1e-6) and np.all(r["side"][:, 2:] == 0)
    back = r["q"] * r["scale"][:, None]
    reg = np.setdiff1d(np.arange(64), [3, 9])
    return ok and np.all(r["q"][:, [3, 9]] == 0) and np.all(np.abs(back - y.numpy())[:, reg] <= r["scale"][:, None] * 0.5001) and np.abs(r["q"]).max() == 127


def test_oracles_and_planted_mistakes():
    import types
    src = {m: open(os.path.join(ROOT, "oracle", m + ".py")).read() for m in ("kvcache_oracle", "norm_oracle")}

    def module(name, old=None, new=None):
        text = src[name]
        if old is not None:
            assert text.count(old) >= 1, old
            text = text.replace(old, new)
        m = types.ModuleType("oracle." + name)
        m.__package__ = "oracle"
        exec(compile(text, name, "exec"), m.__dict__)
        return m

    assert _attend_pin(ko) and _evict_pin(ko) and _norm_pin(no)
    for pin, name, old, new in ((_attend_pin, "kvcache_oracle", "seen = length - n + i + 1", "seen = length - n + i"), (_attend_pin, "kvcache_oracle", "j // g", "j % h"),
                                (_attend_pin, "kvcache_oracle", "weights[j // g, :seen] += p", "weights[j // g, :seen] = p"),
                                (_evict_pin, "kvcache_oracle", "length - recent + i", "length - recent - i"), (_evict_pin, "kvcache_oracle", "-key[j][0], j)", "-key[j][0], -j)"),
                                (_norm_pin, "norm_oracle", ".mean(axis=1)", ".sum(axis=1)"),
                                (_norm_pin, "norm_oracle", "q[:, ~regular] = 0", "pass"), (_norm_pin, "norm_oracle", "t[:, idx]", "h[:, idx]"),
                                (_norm_pin, "norm_oracle", "np.abs(t[:, regular])", "np.abs(t)")):
        try:
            caught = not pin(module(name, old, new))
        except Exception:
            caught = True
        assert caught, (name, old)


def test_store_oracle_is_the_codec():
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.normal(size=(3, 2, 64))).to(torch.float16)
    b = x.view(torch.int16).numpy().view(np.uint16)
    cb = o4.make_codebook()
    packed, scale, vals = ko.store(b, o4.F16, 32, cb)
    p, s = o4.quantize_s16(b.reshape(-1), o4.F16, 32, cb)
    assert np.array_equal(packed.reshape(-1), p) and np.array_equal(scale.reshape(-1), s)
    assert np.array_equal(ko.read(vals, o4.F16).reshape(-1), o4.dequantize_s16(p, s, b.size, 32, cb, o4.F16))
