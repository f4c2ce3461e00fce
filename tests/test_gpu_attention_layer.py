"""The operators of an attention layer run together: against the same steps on a dense cache in fp64, and what a bounded cache holds."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mod():
    from paper_2407_19775_b200 import attention_layer
    return attention_layer


def run(layer, news, steps, hidden, dtype, seed=5):
    """Prompts, then single tokens; the inputs are drawn, so that two layers see the same ones."""
    g = torch.Generator().manual_seed(seed)
    starts = torch.tensor([0] + news).cumsum(0).int().cuda()
    xs = [torch.randn(sum(news), hidden, generator=g).to(dtype).cuda()]
    out = [layer(xs[0], None, starts, max(news))]
    for _ in range(steps):
        x, r = (torch.randn(len(news), hidden, generator=g).to(dtype).cuda() for _ in range(2))
        xs.append((x, r))
        out.append(layer(x, r))
    return xs, out, starts


def test_layer_against_a_dense_cache(mod):
    """Same weights, dense keys and values: what differs is 8-bit rows and weights and 4-bit keys and values."""
    hidden, H, G, hd, news = 512, 2, 4, 64, [70, 1, 33]
    layer = mod.random_layer(3, 128, hidden, H * G, H, hd, 32, torch.bfloat16, seed=1)
    g = torch.Generator().manual_seed(1)
    wq = (torch.randn((H * G + 2 * H) * hd, hidden, generator=g) * hidden ** -0.5).bfloat16().double().cuda()
    wo = (torch.randn(hidden, H * G * hd, generator=g) * (H * G * hd) ** -0.5).bfloat16().double().cuda()
    gamma = ((torch.randn(hidden, generator=g) * 0.1).bfloat16() + 1).double().cuda()
    xs, out, starts = run(layer, news, 3, hidden, torch.bfloat16)
    assert layer.cache.lens.tolist() == [n + 3 for n in news] and layer.cache.kernel_status() == 0
    keys = [None] * 3
    for i, (got, h_got) in enumerate(out):
        x, res = (xs[0], None) if i == 0 else xs[i]
        h = x.double() if res is None else (x.double() + res.double()).bfloat16().double()
        assert torch.equal(h_got.double(), h)
        qkv = (h / (h.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * gamma) @ wq.T
        qkv = qkv.view(-1, H * G + 2 * H, hd)
        at = starts.tolist() if i == 0 else [0, 1, 2, 3]
        rows = []
        for s in range(3):
            q, k, v = qkv[at[s]:at[s + 1]].split((H * G, H, H), dim=1)
            keys[s] = (k, v) if i == 0 else (torch.cat((keys[s][0], k)), torch.cat((keys[s][1], v)))
            K, V = (t.repeat_interleave(G, dim=1) for t in keys[s])
            score = torch.einsum("qhd,khd->hqk", q, K) / math.sqrt(hd)
            n, total = q.shape[0], K.shape[0]
            seen = torch.arange(total, device="cuda")[None] <= torch.arange(total - n, total, device="cuda")[:, None]
            rows.append(torch.einsum("hqk,khd->qhd", score.masked_fill(~seen, -math.inf).softmax(-1), V).reshape(n, -1))
        want = torch.cat(rows) @ wo.T
        # a 4-bit row of 32 normal numbers is off by about a tenth of its norm; attention averages keys' and values' errors
        assert float((got.double() - want).norm() / want.norm()) < 0.2, i


@pytest.mark.parametrize("budget,sinks,recent", [(48, 4, 16), (16, 0, 0), (9, 1, 8)])
def test_bounded_cache(mod, budget, sinks, recent):
    hidden, H, G, hd, news = 256, 2, 2, 64, [70, 5, 33, 48]
    layer = mod.random_layer(4, 96, hidden, H * G, H, hd, 64, torch.float16, budget=budget, sinks=sinks, recent=recent)
    _, out, _ = run(layer, news, 20, hidden, torch.float16)
    assert layer.cache.lens.tolist() == [min(n + 20, budget) for n in news] and layer.cache.kernel_status() == 0
    assert all(bool(torch.isfinite(y).all()) and bool(torch.isfinite(h).all()) for y, h in out)
    assert bool((layer.weights[:, :, budget:] == 0).all()) and bool((layer.weights >= 0).all())
    # every query head of every row handed out a weight of one; what was evicted took its own with it
    most = [(n + 20) * G for n in news]
    got = layer.weights.sum(2).cpu()
    assert all(float(got[s].max()) <= most[s] * (1 + 1e-4) for s in range(4))
    # two budgets that nothing exceeds give the same bits (both calls accumulate weights, so both take the same kernels)
    free = mod.random_layer(4, 96, hidden, H * G, H, hd, 64, torch.float16, budget=80, sinks=sinks, recent=recent)
    wide = mod.random_layer(4, 96, hidden, H * G, H, hd, 64, torch.float16, budget=96, sinks=sinks, recent=recent)
    for (a, _), (b, _) in zip(run(free, news, 3, hidden, torch.float16)[1], run(wide, news, 3, hidden, torch.float16)[1]):
        assert torch.equal(a, b)


def test_command(mod, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["attention_layer", "--sequences", "3", "--prompt", "90", "--steps", "4", "--budget", "50", "--hidden", "512",
                                     "--q-heads", "4", "--kv-heads", "2"])
    mod.main()
    assert "slots [50, 50, 20]" in capsys.readouterr().out
