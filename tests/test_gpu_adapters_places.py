"""GPU tests of where the results of a layer with adapters may lie: at any multiple of their element's size, with nothing beside them written."""
import pytest
import torch

from test_gpu_adapters import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,rank", [(264, 16), (268, 64)])
@pytest.mark.parametrize("path", [0, 1])
def test_results_at_any_place(bq, path, N, rank, out):
    """Columns a multiple of eight and of four only; one to three elements behind a 16-byte address (8 and 12 bytes of 16-bit outputs among
    them), rows that several sequences share and single ones."""
    tdt = torch.float16 if out == torch.float32 else out
    c = Layer(bq, 320, N, 3, 3, rank, tdt, seed=8)
    for news in ([90, 0, 40, 3], [1] * 20):
        starts, M = [sum(news[:i]) for i in range(len(news) + 1)], sum(news)
        ids = [i % 4 - (i == 3) for i in range(len(news))]
        x = c.rows(M)
        want = c.linear(x, ids, starts, out_dtype=out, path=path)
        for off in (1, 2, 3, 4, 6):
            flat = torch.full((M * N + 16,), 7.0, dtype=out, device="cuda")
            y = c.linear(x, ids, starts, y_out=flat[off:off + M * N].view(M, N), path=path)
            assert bool((flat[:off] == 7).all()) and bool((flat[off + M * N:] == 7).all())
            if path == 1:                                              # the same kernels
                assert torch.equal(y, want)


def test_results_inside_an_element_are_refused(bq):
    c = Layer(bq, 320, 72, 0, 2, 16, torch.float16)
    L, x = bq.mmd._lib(), c.rows(4).cuda()
    ids, y = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.full((4 * 72 + 8,), 7.0, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    at = lambda t, off=0: t.data_ptr() + off                            # noqa: E731
    for dt, offs in ((0, (1, 2, 3, 6)), (1, (1, 3, 5))):
        for off in offs:
            assert L.mmd_linear(c.lin.handle, at(x), 4, at(y, off), dt, at(ws), ws.numel(), 1, None) == 4
            assert L.mmd_linear_adapted(c.lin.handle, c.ad._ref, at(ids), None, 4, at(x), 4, at(y, off), dt, at(ws), ws.numel(), 0, None) == 4
    torch.cuda.synchronize()
    assert bool((y == 7).all())
