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
from oracle import norm_oracle as no
from test_gpu_adapters import DT, HALF_ULP, Layer, bits, make

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


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,rank,news", [(264, 16, [40, 31, 70, 1]), (136, 128, [300]), (512, 32, [1] * 24), (4096, 16, [400, 1, 300])])
def test_bits_behind_the_norm(bq, N, rank, news, tdt):
    """a has one feature per rank as well: a column is the product of one element x of the normed row with two numbers.  x is off by its factor's
    (K / 512 + 16) 2^-24 (derived in tests/test_gpu_norm.py) and by what two 16-bit parts leave, half a step of the second behind half a step of
    the first: bf16 2^-16; fp16 2^-22, and 2^-25 below fp16's normal range."""
    K, count = 640, 3
    c = Layer(bq, K, N, 0, count, rank, tdt, seed=10)
    g = torch.Generator().manual_seed(4)
    for name, shape in (("a", (count, rank, K)), ("b", (count, N, rank))):
        t = torch.zeros(shape)
        t.scatter_(2, torch.randint(0, shape[2], (*shape[:2], 1), generator=g), torch.randn(*shape[:2], 1, generator=g))
        setattr(c, name, t.to(tdt))
    for mine, t in zip(c.ad._tensors, (c.a, c.b, c.scale)):
        mine.copy_(t)
    M = sum(news)
    x, res, gamma, _ = make(M, K, 0, tdt, 5, True)
    starts = [sum(news[:i]) for i in range(len(news) + 1)]
    ids = [i % 4 - (i % 4 == 3) * 4 for i in range(len(news))]
    ref = no.norm_rowquant(bits(x), bits(res), bits(gamma[None])[0], 1e-5, DT[tdt], c.idx.numpy())
    rel = (K / 512 + 16) * 2.0 ** -24
    base, tol = c.base(ref["q"], ref["scale"], ref["side"])
    tol += rel * np.abs(base)
    want, of_x = base.copy(), 2.0 ** -16 if tdt == torch.bfloat16 else 2.0 ** -22
    for i, a in enumerate(ids):
        if a >= 0:
            lo, hi = starts[i], starts[i + 1]
            A, B, sc = c.a[a].double().numpy(), c.b[a].double().numpy(), float(c.scale[a])
            part = sc * (ref["normed"][lo:hi] @ A.T) @ B.T
            want[lo:hi] += part
            of_v = 2.0 ** -22 if tdt == torch.float16 else 0.0
            tol[lo:hi] += np.abs(part) * (rel + of_x + of_v + 12 * 2.0 ** -24) + abs(sc) * 2.0 ** -25 * (np.abs(A).sum(1) @ np.abs(B).T) * (tdt == torch.float16)
    tol += 8 * 2.0 ** -24 * np.abs(want) + 2.0 ** -30
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")      # noqa: E731
    y, _ = c.lin.norm_linear(x.cuda(), gamma.cuda(), 1e-5, residual=res.cuda(), out_dtype=torch.float32, adapters=c.ad, ids=dev(ids), starts=dev(starts))
    err = np.abs(y.double().cpu().numpy() - want)
    assert np.all(err <= tol), float((err / tol).max())
