"""GPU tests of the norm at the edges of its ranges, within the bounds of tests/test_gpu_norm.py."""
import pytest
import torch

from test_gpu_norm import check_rows, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("target", ["x", "residual"])
@pytest.mark.parametrize("R,K,ko", [(4, 8192, 8), (5, 16400, 1), (3, 40000, 100), (300, 8208, 65), (170, 16400, 3)])
def test_in_place(bq, R, K, ko, target, tdt):
    """h into x or into the residual, rows in registers and rows that are read again."""
    x, res, gamma, idx = make(R, K, ko, tdt, R + K)
    xd, rd = x.cuda(), res.cuda()
    into = xd if target == "x" else rd
    q, s, side, h = bq.mmd_norm_rowquant(xd, gamma.cuda(), 1e-5, idx.cuda(), rd, h_out=into)
    torch.cuda.synchronize()
    assert h.data_ptr() == into.data_ptr()
    check_rows(q, s, side, h, x, res, gamma, idx, 1e-5, tdt)


@pytest.mark.parametrize("R,K,ko", [(6, 1040, 5), (5, 8208, 65), (4, 40000, 7), (160, 8208, 3)])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("amp,eps", [(1e25, 0.0), (1e25, 1e-5), (1e19, 1e-5), (2e20, 1e30), (1e-25, 0.0), (1e-25, 1e-5), (1e-25, 1e-38), (3e-23, 2.0 ** -149), (1e-20, 1e-31), (1e-14, 0.0)])
def test_rows_whose_squares_leave_the_range(bq, R, K, ko, residual, amp, eps):
    """bf16 rows up to about 2^100 and down to 2^-95, whose squares fp32 does not hold: codes, factors and side columns as for any
    row.  Rows of ordinary size and of zeros are among them."""
    x, res, gamma, idx = make(R, K, ko, torch.bfloat16, R + K, residual)
    small = x[-1].clone()
    x = (x.float() * amp).to(torch.bfloat16)
    x[-1] = small
    if residual:
        res = (res.float() * amp).to(torch.bfloat16)
        res[-1] = 0
    if eps == 0.0:
        x[1] = x[0]                                                  # a row of zeros has no factor then
        if residual:
            res[1] = res[0]
    q, s, side, h = bq.mmd_norm_rowquant(x.cuda(), gamma.cuda(), eps, idx.cuda(), None if res is None else res.cuda())
    torch.cuda.synchronize()
    check_rows(q, s, side, h, x, res, gamma, idx, eps, torch.bfloat16)
