"""Host-side checks of the cache, the norm and the layer, without a GPU: stand-ins take the place of tensors on a device, so that a
refusal is seen before any kernel could run."""
import pytest
import torch

from paper_2407_19775_b200.binding import BqError


class OnDevice:
    """A CPU tensor that answers the checks as one on cuda:`index` would; its address is never handed to a kernel."""

    def __init__(self, t: torch.Tensor, index: int = 0):
        self.t, self.device, self.is_cuda = t, torch.device("cuda", index), True

    def __getattr__(self, name):
        return getattr(self.t, name)


def pools(pages=8, heads=2, page=16, dim=64, block=64):
    codes = [OnDevice(torch.zeros(pages, heads, page, dim // 2, dtype=torch.uint8)) for _ in range(2)]
    return codes + [OnDevice(torch.zeros(pages, heads, page, dim // block, dtype=torch.bfloat16)) for _ in range(2)]


def test_tables_with_overlapping_rows_are_refused(bq):
    """A kernel reads row s at s * stride: rows that share memory would be taken for rows a whole row apart, past the tensor's end."""
    cb = bq.Codebook4()
    base = torch.arange(12, dtype=torch.int32)
    lens = OnDevice(torch.zeros(4, dtype=torch.int32))
    for table in (base[:3].expand(4, 3), base.as_strided((4, 3), (1, 1)), base.as_strided((4, 3), (2, 1))):
        with pytest.raises(BqError):
            bq.KvCache4(*pools(), OnDevice(table), lens, cb)
    for table, stride in ((base.view(4, 3), 3), (torch.zeros(4, 9, dtype=torch.int32)[:, :3], 9)):
        assert bq.KvCache4(*pools(), OnDevice(table), lens, cb)._c.table_stride == stride
    one = bq.KvCache4(*pools(), OnDevice(base[:3].expand(1, 3)), OnDevice(torch.zeros(1, dtype=torch.int32)), cb)
    assert one._c.table_stride == 3                                  # the one row's stride means nothing
