"""GPU tests of mmd_norm_rowquant and mmd_norm_linear against the CPU oracle.

h and the codes are exact (the factor that depends on a sum's order divides out of the codes).  The row factor 1 / rms comes from
an fp32 sum of K squares in some order: a relative error of at most (K / 256 + 16) 2^-24 in the sum (a thread adds its own few,
then a tree), half of that after the root, and four roundings behind it, so scale and side are compared within
rel = (K / 512 + 16) 2^-24, plus the narrowing for the 16-bit side.
"""
import numpy as np
import pytest
import torch

from oracle import mmd_oracle as mo
from oracle import norm_oracle as no
from paper_2407_19775_b200 import workloads
from paper_2407_19775_b200.binding import BqError

pytestmark = pytest.mark.gpu
DT = {torch.float16: mo.F16, torch.bfloat16: mo.BF16}
HALF_ULP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}       # 11 and 8 significant bits, to nearest


def bits(t):
    return workloads.bits_2d(t.cpu())


def make(R, K, ko, tdt, seed, residual=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, K, generator=g) * 0.5
    idx = torch.randperm(K, generator=g)[:ko].sort().values.int()
    x[:, idx.long()] *= 30
    if R > 3:
        x[1] = 0
        x[2] *= 1e-3
        x[3] *= 200
    res = torch.randn(R, K, generator=g) * 0.5 if residual else None
    if residual and R > 3:
        res[1] = 0                                                   # a row of zeros
    gamma = 1 + 0.1 * torch.randn(K, generator=g)
    gamma[K // 2] = 0
    return x.to(tdt), None if res is None else res.to(tdt), gamma.to(tdt), idx


def check_rows(q, scale, side, h, x, res, gamma, idx, eps, tdt):
    K = x.shape[1]
    ref = no.norm_rowquant(bits(x), None if res is None else bits(res), bits(gamma[None])[0], eps, DT[tdt], idx.numpy())
    rel = (K / 512 + 16) * 2.0 ** -24
    assert np.array_equal(bits(h), ref["h"])
    assert np.array_equal(q.cpu().numpy(), ref["q"])
    assert np.all(np.abs(scale.cpu().numpy().astype(np.float64) - ref["scale"]) <= rel * ref["scale"] + 1e-45)
    got = side.double().cpu().numpy()
    tol = np.abs(ref["side"]) * (rel + HALF_ULP[tdt] * (1 + rel)) + (2.0 ** -25 if tdt == torch.float16 else 1e-40)
    assert np.all(np.abs(got - ref["side"]) <= tol)
    return ref


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("R,K,ko", [(1, 16, 0), (5, 48, 3), (37, 320, 7), (4, 8192, 8), (9, 6144, 64), (7, 8208, 65), (5, 16400, 1), (2, 40000, 100), (700, 1040, 5)])
def test_rows(bq, R, K, ko, residual, tdt):
    x, res, gamma, idx = make(R, K, ko, tdt, R * K + ko, residual)
    q, s, side, h = bq.mmd_norm_rowquant(x.cuda(), gamma.cuda(), 1e-5, idx.cuda() if ko else None, None if res is None else res.cuda())
    torch.cuda.synchronize()
    check_rows(q, s, side, h, x, res, gamma, idx, 1e-5, tdt)


def test_divisors_outside_the_reciprocal_window_and_in_place(bq):
    for amp in (1e-25, 1e25):
        x, res, gamma, idx = make(6, 1040, 5, torch.bfloat16, 3)
        x, res = (x.float() * amp).to(torch.bfloat16), (res.float() * amp).to(torch.bfloat16)
        xd, rd = x.cuda(), res.cuda()
        q, s, side, h = bq.mmd_norm_rowquant(xd, gamma.cuda(), 0.0 if amp > 1 else 1e-5, idx.cuda(), rd)
        ref = no.norm_rowquant(bits(x), bits(res), bits(gamma[None])[0], 1e-5, mo.BF16, idx.numpy())
        assert np.array_equal(q.cpu().numpy(), ref["q"]) and np.array_equal(bits(h), ref["h"])
    for target in (0, 1):
        x, res, gamma, idx = make(6, 1040, 5, torch.float16, 4)
        xd, rd = x.cuda(), res.cuda()
        into = (xd, rd)[target]
        q, s, side, h = bq.mmd_norm_rowquant(xd, gamma.cuda(), 1e-5, idx.cuda(), rd, h_out=into)
        torch.cuda.synchronize()
        assert h.data_ptr() == into.data_ptr()
        check_rows(q, s, side, h, x, res, gamma, idx, 1e-5, torch.float16)


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,K,N,ko", [(1, 320, 72, 3), (37, 320, 72, 0), (64, 2048, 1024, 8), (300, 1024, 2048, 16), (130, 640, 264, 40)])
def test_layer(bq, M, K, N, ko, tdt):
    """The fused call is the layer over the rows the norm call gives: the same workspace contents, the same product."""
    x, res, gamma, idx = make(M, K, ko, tdt, M + K)
    W = (torch.randn(N, K, generator=torch.Generator().manual_seed(7)) * 0.02).to(tdt)
    lin = bq.DecomposedLinear(W.cuda(), idx.numpy())
    for out_dtype in (torch.float32, tdt):
        y, h = lin.norm_linear(x.cuda(), gamma.cuda(), 1e-5, residual=res.cuda(), out_dtype=out_dtype)
        torch.cuda.synchronize()
        qx, sx, sd = (t.clone() for t in lin.workspace_parts(M))
        ref = check_rows(qx, sx, sd, h, x, res, gamma, idx, 1e-5, tdt)
        assert lin.kernel_status() == 0
        qw, sw, wo = mo.rowquant(bits(W), DT[tdt], idx.numpy())
        s32 = sx.cpu().numpy().astype(np.float64)
        acc = mo.int_product(ref["q"], qw).astype(np.float32).astype(np.float64)
        side_x, side_w = sd.double().cpu().numpy(), mo.widen(wo, DT[tdt]).astype(np.float64)
        want = acc * (s32[:, None] * sw[None, :].astype(np.float64)).astype(np.float32).astype(np.float64) + side_x @ side_w.T
        sabs = np.abs(side_x) @ np.abs(side_w).T
        tol = 2.0 ** -23 * np.abs(want) + (wo.shape[1] + 2) * 2.0 ** -22 * sabs + (0 if out_dtype == torch.float32 else HALF_ULP[tdt] * np.abs(want) + 2.0 ** -25)
        assert np.all(np.abs(y.double().cpu().numpy() - want) <= tol)
        full = no.norm_rowquant(bits(x), bits(res), bits(gamma[None])[0], 1e-5, DT[tdt], idx.numpy())["normed"] @ mo.widen(bits(W), DT[tdt]).astype(np.float64).T
        assert np.linalg.norm(want - full) <= 0.03 * np.linalg.norm(full)      # and it is the norm through the layer


def test_chain_through_one_workspace(bq):
    """Back-to-back calls without synchronising: a call's rows are not overwritten while the call before still reads them."""
    K = N = 2048
    x, res, gamma, idx = make(64, K, 8, torch.float16, 1)
    W = (torch.randn(N, K, generator=torch.Generator().manual_seed(7)) * 0.02).to(torch.float16)
    lin = bq.DecomposedLinear(W.cuda(), idx.numpy())
    xs = [(x * (1 + i)).cuda() for i in range(6)]
    want = []
    for t in xs:
        want.append(lin.norm_linear(t, gamma.cuda(), 1e-5, residual=res.cuda())[0].clone())
        torch.cuda.synchronize()
    rd, gd = res.cuda(), gamma.cuda()
    got = [lin.norm_linear(t, gd, 1e-5, residual=rd)[0] if i % 2 else lin.norm_linear(t, gd, 1e-5, residual=rd)[0] for i, t in enumerate(xs)]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_refusals(bq):
    x = torch.zeros(4, 64, dtype=torch.float16, device="cuda")
    g = torch.ones(64, dtype=torch.float16, device="cuda")
    lin = bq.DecomposedLinear(torch.zeros(8, 64, dtype=torch.float16, device="cuda"), [])
    flat = torch.zeros(4 * 64 + 1, dtype=torch.float16, device="cuda")
    for bad in (lambda: bq.mmd_norm_rowquant(x.float(), g.float(), 1e-5), lambda: bq.mmd_norm_rowquant(x, g[:32], 1e-5), lambda: bq.mmd_norm_rowquant(x, g.bfloat16(), 1e-5),
                lambda: bq.mmd_norm_rowquant(x, g, -1.0), lambda: bq.mmd_norm_rowquant(x, g, float("nan")), lambda: bq.mmd_norm_rowquant(x, g, 1e-5, residual=x[:2]),
                lambda: bq.mmd_norm_rowquant(x[:, :40].contiguous(), g[:40], 1e-5), lambda: bq.mmd_norm_rowquant(flat[1:].view(4, 64), g, 1e-5),
                lambda: bq.mmd_norm_rowquant(x, g, 1e-5, residual=x, h_out=x.float()), lambda: lin.norm_linear(x.bfloat16(), g.bfloat16(), 1e-5),
                lambda: lin.norm_linear(x, g, 1e-5, path=bq.mmd.PATH_TENSOR_STREAMK), lambda: lin.norm_linear(x[:, :32].contiguous(), g[:32], 1e-5)):
        with pytest.raises(BqError):
            bad()
    y, h = lin.norm_linear(x[:0], g, 1e-5)
    assert y.shape == (0, 8) and h.shape == (0, 64)
