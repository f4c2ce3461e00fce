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
