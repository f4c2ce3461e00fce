"""Low-rank adapters beside a decomposed layer without a GPU: refusals before any device is touched."""
import ctypes

import pytest
import torch

from paper_2407_19775_b200.binding import BqError


def test_refusals_need_no_device(bq):
    from paper_2407_19775_b200 import mmd
    L = mmd._lib()
    at = lambda n: ctypes.c_void_p(n)                                # noqa: E731

    def adapters(a=256, b=256, scale=256, count=3, rank=16):
        return ctypes.byref(mmd._Adapters(a, b, scale, count, rank))

    def call(w=None, ad=None, ids=at(256), starts=None, n_seq=4, M=4, path=0):
        return L.mmd_linear_adapted(w, adapters() if ad is None else ad, ids, starts, n_seq, at(256), M, at(512), 1, at(1024), 1 << 30, path, None)

    def norm(w=None, ad=None, n_seq=4, M=4):
        return L.mmd_norm_linear_adapted(w, adapters() if ad is None else ad, at(256), None, n_seq, at(256), None, at(256), 1e-5, M, None, at(512), 1, at(1024), 1 << 30, 0, None)

    assert call() == 1 and norm() == 1                               # no layer
    size = ctypes.c_size_t()
    assert L.mmd_adapted_workspace(None, 4, 4, 16, 0, ctypes.byref(size)) == 1


def test_handles_refuse_what_the_layer_could_not_read(bq):
    a, b, s = torch.zeros(3, 16, 64, dtype=torch.float16), torch.zeros(3, 24, 16, dtype=torch.float16), torch.ones(3)
    with pytest.raises(BqError, match="CUDA"):
        bq.Adapters(a, b, s)
    for pairs, scales in (([], []), ([(a[0], b[0])], []), ([(a[0], b[0, :, :8])], [1.0]), ([(a[0], b[0]), (a[0, :, :32], b[0])], [1.0, 1.0]),
                          ([(a[0], b[0]), (a[0], b[0, :8])], [1.0, 1.0]), ([(a[0], b[0].bfloat16())], [1.0]), ([(a, b[0])], [1.0])):
        with pytest.raises(BqError):
            bq.Adapters.pack(pairs, scales)
