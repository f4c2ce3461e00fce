"""How many bits the adapters' part keeps.  Rows and a are small multiples of powers of two, so that u is exact in fp32 however it is summed, and
b has one rank per column, so that a column is one product: with v = RN32(scale u), exact in 64 bits,

    |y - (base + v b)| <= 2^-23 |base| + e |v b| + c (2^-24 |v b| + 2^-24 |base + v b|),   c = 8

(base: exact integers times a product of two scales, three roundings; e: what the kernel carries of v; c: the parts' products meet in three sums
and join the base in one, tensor-core sums truncating to the larger operand, twice 2^-24 each), plus the output's half ulp.  e is 0 for fp32
outputs of bf16 layers and on the kernels that keep fp32, 2^-22 for fp16 layers, 2^-16 for 16-bit outputs of bf16 layers."""
import numpy as np
import pytest
import torch

from oracle import mmd_oracle as mo
from test_gpu_adapters import DT, HALF_ULP, Layer, bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,rank,news", [(264, 16, [40, 31, 70, 1]), (130, 64, [40, 31, 70, 1]), (136, 256, [300]), (512, 32, [1] * 24), (4096, 16, [400, 1, 300]), (4096, 80, [400, 1, 300])])
def test_bits(bq, N, rank, news, tdt):
    K, count = 320, 3
    c = Layer(bq, K, N, 0, count, rank, tdt, seed=9)
    g = torch.Generator().manual_seed(3)
    c.a = (torch.randint(-7, 8, (count, rank, K), generator=g) / 64).to(tdt)
    b = torch.zeros(count, N, rank)
    at = torch.randint(0, rank, (count, N, 1), generator=g)
    b.scatter_(2, at, torch.randn(count, N, 1, generator=g))
    c.b = b.to(tdt)
    for mine, t in zip(c.ad._tensors, (c.a, c.b, c.scale)):
        mine.copy_(t)
    M = sum(news)
    x = torch.randint(-15, 16, (M, K), generator=g).to(tdt)
    starts = [sum(news[:i]) for i in range(len(news) + 1)]
    ids = [i % 4 - (i % 4 == 3) * 4 for i in range(len(news))]
    q, s, side = mo.rowquant(bits(x), DT[tdt], c.idx.numpy())
    base, _ = c.base(q, s.astype(np.float64), mo.widen(side, DT[tdt]).astype(np.float64))
    part = np.zeros_like(base)
    for i, a in enumerate(ids):
        if a >= 0:
            u = x[starts[i]:starts[i + 1]].double().numpy() @ c.a[a].double().numpy().T
            v = (np.float32(c.scale[a].item()) * u.astype(np.float32)).astype(np.float64)
            part[starts[i]:starts[i + 1]] = v @ c.b[a].double().numpy().T
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")      # noqa: E731
    for out in (torch.float32, tdt):
        y = c.lin.linear(x.cuda(), out_dtype=out, adapters=c.ad, ids=dev(ids), starts=dev(starts)).double().cpu().numpy()
        e = 2.0 ** -22 if tdt == torch.float16 else 0.0 if out == torch.float32 else 2.0 ** -16
        tol = 2.0 ** -23 * np.abs(base) + e * np.abs(part) + 8 * 2.0 ** -24 * (np.abs(part) + np.abs(base + part)) + 2.0 ** -30
        if out != torch.float32:
            tol += HALF_ULP[out] * (np.abs(base + part) + tol)
        err = np.abs(y - base - part)
        assert np.all(err <= tol), float((err / tol).max())
