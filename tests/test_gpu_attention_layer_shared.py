"""Positions, shared prefixes and adapters run together in the attention layer, against the same steps on dense rows in fp64."""
import math

import pytest
import torch

from paper_2407_19775_b200 import attention_layer
from paper_2407_19775_b200.binding import BqError
from test_gpu_attention_layer import mod  # noqa: F401

pytestmark = pytest.mark.gpu
HIDDEN, H, G, HD = 512, 2, 4, 64


def make(bq, dtype, prefix=True, rotary=True, adapters=True, axes=1, budget=None, n_seq=4, capacity=128):
    kw = {}
    if rotary:
        kw["rotary"] = bq.Rotary(HD, sections=None if axes == 1 else [8, 12, 12])
    if prefix:
        kw["prefix"] = bq.KvCache4.empty(2, 96, H, HD, 32, bq.Codebook4())
        kw["members"] = torch.tensor([0, 2, n_seq - 1], dtype=torch.int32, device="cuda")      # the last sequence shares none
    layer = attention_layer.random_layer(n_seq, capacity, HIDDEN, H * G, H, HD, 32, dtype, seed=1, budget=budget, **kw)
    if adapters:
        layer.qkv_adapters, layer.out_adapters = (attention_layer.random_adapters(w, 3, 16, seed=i) for i, w in enumerate((layer.qkv, layer.out)))
    return layer


def dense_weights(dtype):
    g = torch.Generator().manual_seed(1)
    wq = (torch.randn((H * G + 2 * H) * HD, HIDDEN, generator=g) * HIDDEN ** -0.5).to(dtype).double().cuda()
    wo = (torch.randn(HIDDEN, H * G * HD, generator=g) * (H * G * HD) ** -0.5).to(dtype).double().cuda()
    gamma = ((torch.randn(HIDDEN, generator=g) * 0.1).to(dtype) + 1).double().cuda()
    return wq, wo, gamma


def turned(x, pos, rotary):
    """x [rows, heads, HD] by positions [axes, rows], halves layout."""
    f = torch.from_numpy(rotary.frequencies).cuda()
    of = torch.zeros(HD // 2, dtype=torch.long) if rotary.axes == 1 else torch.repeat_interleave(torch.arange(3), torch.tensor([8, 12, 12]))
    a = pos.double()[of.cuda()].t()[:, None] * f
    u, v = x.chunk(2, -1)
    return torch.cat([u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()], -1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("axes", [1, 3])
def test_all_of_them_against_dense_rows(bq, dtype, axes):
    layer = make(bq, dtype, axes=axes)
    wq, wo, gamma = dense_weights(dtype)
    g = torch.Generator().manual_seed(4)
    draw = lambda n: torch.randn(n, HIDDEN, generator=g).to(dtype).cuda()      # noqa: E731
    place = lambda p: p[None].repeat(axes, 1) + torch.arange(axes, dtype=torch.int32, device="cuda")[:, None] * 3 if axes > 1 else p      # noqa: E731

    def adapted(y, x, ad, row_ids):
        a, b, s = (t.double() for t in ad._tensors)
        for r, i in enumerate(row_ids):
            if i >= 0:
                y[r] += s[i] * (x[r] @ a[i].t()) @ b[i].t()
        return y

    def project(h, pos, row_ids):
        n = h / (h.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * gamma
        qkv = adapted(n @ wq.T, n, layer.qkv_adapters, row_ids).view(-1, H * G + 2 * H, HD)
        q, k, v = qkv.split((H * G, H, H), dim=1)
        pos = pos[None] if pos.dim() == 1 else pos
        return turned(q, pos, layer.rotary), turned(k, pos, layer.rotary), v

    def attend(q, k, v):
        kk, vv = (t.repeat_interleave(G, dim=1) for t in (k, v))
        n, total = q.shape[0], k.shape[0]
        seen = torch.arange(total, device="cuda")[None] <= torch.arange(total - n, total, device="cuda")[:, None]
        p = (torch.einsum("qhd,khd->hqk", q, kk) / math.sqrt(HD)).masked_fill(~seen, -math.inf).softmax(-1)
        return torch.einsum("hqk,khd->qhd", p, vv).reshape(n, -1)

    # the prefixes, in two calls
    beginnings = [[], []]
    for news in ((50, 20), (1, 13)):
        at = torch.tensor([0, news[0], sum(news)], dtype=torch.int32, device="cuda")
        x = draw(sum(news))
        first = [sum(len(t[0]) for t in b) for b in beginnings]
        pos = torch.cat([torch.arange(f, f + n, dtype=torch.int32) for f, n in zip(first, news)]).cuda()
        got, _ = layer.begin(x, None, at, max(news), positions=place(pos))
        q, k, v = project(x.double(), place(pos), [-1] * sum(news))
        rows = []
        for p in range(2):
            part = slice(int(at[p]), int(at[p + 1]))
            beginnings[p].append((k[part], v[part]))
            rows.append(attend(q[part], *(torch.cat([t[i] for t in beginnings[p]]) for i in (0, 1))))
        want = torch.cat(rows) @ wo.T
        assert float((got.double() - want).norm() / want.norm()) < 0.2
    plens = [51, 33]
    assert layer.prefix.lens.tolist() == plens
    keys = [tuple(torch.cat([t[i] for t in beginnings[p]]) for i in (0, 1)) for p in (0, 0, 1)] + [(torch.zeros(0, H, HD, dtype=torch.float64, device="cuda"),) * 2]
    had = [51, 51, 33, 0]
    ids = [2, -1, 0, 1]
    ids_dev = torch.tensor(ids, dtype=torch.int32, device="cuda")
    for i, news in enumerate(([40, 7, 1, 30], [1] * 4, [1] * 4)):
        n = sum(news)
        starts = None if i else torch.tensor([0, 40, 47, 48, 78], dtype=torch.int32, device="cuda")
        x, res = draw(n), draw(n) if i else None
        pos = torch.cat([torch.arange(h, h + m, dtype=torch.int32) for h, m in zip(had, news)]).cuda()
        got, h_got = layer(x, res, starts, max(news), positions=place(pos), ids=ids_dev)
        h = x.double() if res is None else (x.double() + res.double()).to(dtype).double()
        assert torch.equal(h_got.double(), h)
        row_ids = [a for a, m in zip(ids, news) for _ in range(m)]
        q, k, v = project(h, place(pos), row_ids)
        rows, lo = [], 0
        for s, m in enumerate(news):
            keys[s] = tuple(torch.cat([old, new[lo:lo + m]]) for old, new in zip(keys[s], (k, v)))
            rows.append(attend(q[lo:lo + m], *keys[s]))
            lo += m
        o = torch.cat(rows)
        want = adapted(o @ wo.T, o, layer.out_adapters, row_ids)
        # as in the layer without them: 4-bit rows of 32 normal numbers are off by about a tenth of their norm
        assert float((got.double() - want).norm() / want.norm()) < 0.2, i
        had = [a + m for a, m in zip(had, news)]
    assert layer.cache.kernel_status() == 0 and layer.prefix.kernel_status() == 0 and layer.qkv.kernel_status() == 0


def test_a_bounded_cache_behind_a_prefix(bq):
    """Own slots are bounded, the prefix is not touched, and weights are those of the own slots alone."""
    layer = make(bq, torch.float16, budget=40, adapters=False, capacity=96)
    layer.sinks, layer.recent = 2, 8
    x = torch.randn(100, HIDDEN, device="cuda").half()
    layer.begin(x[:70], None, torch.tensor([0, 50, 70], dtype=torch.int32, device="cuda"), 50)
    pools = [p.clone() for p in layer.prefix._pools]
    pos = torch.full((4,), 50, dtype=torch.int32, device="cuda")
    for i in range(60):
        y, _ = layer(x[:4] * (i + 1), positions=pos + i)
    assert layer.cache.lens.tolist() == [40] * 4 and bool(torch.isfinite(y).all())
    assert all(torch.equal(a, b) for a, b in zip(pools, layer.prefix._pools))
    got = layer.weights.sum(2).cpu()
    assert bool((layer.weights >= 0).all()) and float(got.max()) <= 60 * G * (1 + 1e-4)
    assert bool((layer.weights[:, :, 40:] == 0).all())


def test_captured_steps(bq):
    """A step with positions, prefix and adapters, replayed with other inputs."""
    def steps(layer, xs, poss, graph):
        ids = torch.tensor([0, 2, -1, 1], dtype=torch.int32, device="cuda")
        layer.begin(xs[0].repeat(20, 1)[:70] * 0.5, None, torch.tensor([0, 50, 70], dtype=torch.int32, device="cuda"), 50)
        x, pos, out = xs[0].clone(), poss[0].clone(), []
        out.append(layer(x, positions=pos, ids=ids)[0].clone())
        if graph:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                y, _ = layer(x, positions=pos, ids=ids)
        for i in range(1, 6):
            x.copy_(xs[i])
            pos.copy_(poss[i])
            if graph:
                g.replay()
            else:
                y, _ = layer(x, positions=pos, ids=ids)
            out.append(y.clone())
        torch.cuda.synchronize()
        return out, layer.cache.lens.tolist()

    xs = [torch.randn(4, HIDDEN, generator=torch.Generator().manual_seed(i)).half().cuda() for i in range(6)]
    poss = [torch.tensor([50 + i, 51 + i, 20 + i, i], dtype=torch.int32, device="cuda") for i in range(6)]
    plain, lens = steps(make(bq, torch.float16), xs, poss, False)
    replayed, lens2 = steps(make(bq, torch.float16), xs, poss, True)
    assert lens == lens2 == [6] * 4 and all(torch.equal(a, b) for a, b in zip(plain, replayed))


def test_refusals(bq):
    x = torch.zeros(4, HIDDEN, dtype=torch.float16, device="cuda")
    pos, ids = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    plain = make(bq, torch.float16, False, False, False)
    for kw in (dict(positions=pos), dict(ids=ids)):
        with pytest.raises(BqError):
            plain(x, **kw)
    with pytest.raises(BqError):
        plain.begin(x[:1])
    for layer in (make(bq, torch.float16), make(bq, torch.float16, prefix=False, budget=40)):
        with pytest.raises(BqError):
            layer(x)                                                 # nobody knows the positions
        assert layer.cache.lens.tolist() == [0] * 4
    layer = make(bq, torch.float16)
    for bad in (dict(positions=pos.long()), dict(positions=pos[:3]), dict(positions=pos, ids=ids.long()), dict(positions=pos, ids=ids[:3]), dict(positions=pos, residual=x[:2])):
        with pytest.raises(BqError):
            layer(x, **bad)
        assert layer.cache.lens.tolist() == [0] * 4                  # nothing was stored, and nothing is counted
    with pytest.raises(BqError):                                     # more rows than the two pages of 64 that a prefix of 96 rows was given
        layer.begin(torch.zeros(129, HIDDEN, dtype=torch.float16, device="cuda"), None, torch.tensor([0, 129, 129], dtype=torch.int32, device="cuda"), 129)
    assert layer.prefix.lens.tolist() == [0, 0]
    cache = bq.KvCache4.empty(4, 64, H, HD, 32, bq.Codebook4())
    w = torch.zeros((H * G + 2 * H) * HD, HIDDEN, dtype=torch.float16, device="cuda")
    args = (w, torch.zeros(HIDDEN, H * G * HD, dtype=torch.float16, device="cuda"), torch.ones(HIDDEN, dtype=torch.float16, device="cuda"), H * G, H, cache)
    for kw in (dict(rotary=bq.Rotary(2 * HD)), dict(members=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(BqError):
            attention_layer.AttentionLayer(*args, **kw)


def test_command(mod, monkeypatch, capsys):  # noqa: F811
    monkeypatch.setattr("sys.argv", ["attention_layer", "--sequences", "3", "--prompt", "90", "--steps", "4", "--budget", "50", "--hidden", "512",
                                     "--q-heads", "4", "--kv-heads", "2", "--positions", "--prefix", "70", "--adapters", "2"])
    mod.main()
    assert "slots [50, 50, 20]" in capsys.readouterr().out
