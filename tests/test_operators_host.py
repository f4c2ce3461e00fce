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


def layer(bq, K=64, N=24):
    """A handle without a device: every call below fails a check before the library sees it."""
    lin = bq.DecomposedLinear.__new__(bq.DecomposedLinear)
    lin.N, lin.K, lin.dtype, lin.device, lin._h, lin._need = N, K, torch.float16, torch.device("cuda", 0), None, {}
    return lin


def test_outputs_of_a_layer_are_checked(bq):
    """The kernels write [M, N] elements from y_out's start on, whatever the tensor holds."""
    lin = layer(bq)
    x, g = OnDevice(torch.zeros(4, 64, dtype=torch.float16)), OnDevice(torch.ones(64, dtype=torch.float16))
    ws = OnDevice(torch.zeros(1 << 16, dtype=torch.uint8))

    class Reached(Exception):
        pass

    def stop(*_):
        raise Reached

    calls = (lambda y, w=ws: lin.linear(x, y_out=y, workspace=w), lambda y, w=ws: lin.norm_linear(x, g, 1e-5, y_out=y, workspace=w),
             lambda y, w=ws: lin.linear_static(x, y_out=y))
    import paper_2407_19775_b200.mmd as mmd
    good = OnDevice(torch.zeros(4, 24, dtype=torch.float16))
    with pytest.MonkeyPatch.context() as m:
        m.setattr(mmd, "_lib", stop)                                 # only what passes the checks gets there
        m.setattr(torch.cuda, "device", lambda d: __import__("contextlib").nullcontext())
        m.setattr(torch.cuda, "current_device", lambda: 0)
        m.setattr(mmd, "_stream", lambda x: 0)
        for call in calls:
            for bad in (torch.zeros(3, 24), torch.zeros(4, 23), torch.zeros(95), torch.zeros(0, 24), torch.zeros(4, 24).double()):
                with pytest.raises(BqError):
                    call(OnDevice(bad.half() if bad.dtype == torch.float32 else bad))
            with pytest.raises(BqError):
                call(OnDevice(torch.zeros(4, 24, dtype=torch.float16), 1))      # on another device
            with pytest.raises(Reached):
                call(good)
        for call in calls[:2]:                                       # a workspace that a kernel could not write
            for bad in (torch.zeros(1 << 16, dtype=torch.uint8), OnDevice(torch.zeros(1 << 16, dtype=torch.uint8), 1)):
                with pytest.raises(BqError):
                    call(good, bad)


def test_operands_of_the_norm_share_a_device(bq):
    """Every address is read by a kernel on x's device; idx as 32-bit integers."""
    import paper_2407_19775_b200.mmd as mmd
    half = lambda *shape, index=0: OnDevice(torch.zeros(*shape, dtype=torch.float16), index)      # noqa: E731
    x, g, lin = half(4, 64), half(64), layer(bq)
    here = {"gamma": g, "residual": half(4, 64), "h_out": half(4, 64)}
    assert mmd._norm_args(x, here["gamma"], here["residual"], here["h_out"])[0] is here["h_out"]
    for name, away in (("gamma", half(64, index=1)), ("residual", half(4, 64, index=1)), ("h_out", half(4, 64, index=1))):
        args = {**here, name: away}
        with pytest.raises(BqError):
            bq.mmd_norm_rowquant(x, args["gamma"], 1e-5, None, args["residual"], args["h_out"])
        with pytest.raises(BqError):
            lin.norm_linear(x, args["gamma"], 1e-5, residual=args["residual"], h_out=args["h_out"])
    for idx in (torch.zeros(3, dtype=torch.int64), torch.zeros(3)):
        with pytest.raises(BqError):
            bq.mmd_norm_rowquant(x, g, 1e-5, OnDevice(idx))
    with pytest.raises(BqError):
        bq.mmd_norm_rowquant(x, g, 1e-5, OnDevice(torch.zeros(3, dtype=torch.int32), 1))
