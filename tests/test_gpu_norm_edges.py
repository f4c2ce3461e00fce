"""GPU tests of the norm at the edges of its ranges, within the bounds of tests/test_gpu_norm.py."""
import pytest
import torch

from paper_2407_19775_b200.binding import BqError
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


def test_a_shifted_h_out_is_refused(bq):
    """h_out may be an input itself; one that overlaps an input at another place would be written before it is read."""
    room = torch.randn(40, 64, device="cuda").half()
    gamma, res = torch.ones(64, dtype=torch.float16, device="cuda"), torch.randn(8, 64, device="cuda").half()
    lin = bq.DecomposedLinear(torch.zeros(8, 64, dtype=torch.float16, device="cuda"), [])
    for at in (9, 10, 13, 15, 17, 19, 23):
        for x, r in ((room[16:24], res), (res, room[16:24])):
            before = room.clone()
            with pytest.raises(BqError):
                bq.mmd_norm_rowquant(x, gamma, 1e-5, None, r, room[at:at + 8])
            with pytest.raises(BqError):
                lin.norm_linear(x, gamma, 1e-5, residual=r, h_out=room[at:at + 8])
            assert torch.equal(room, before)
    for at in (8, 24, 0):                                            # next to it
        h = bq.mmd_norm_rowquant(room[16:24], gamma, 1e-5, None, res, room[at:at + 8])[3]
        assert torch.equal(h, room[16:24] + res)
