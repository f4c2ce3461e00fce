"""GPU tests of the workspaces that a cache and a layer keep between calls: streams."""
import pytest
import torch

from test_gpu_kvcache import Case

pytestmark = pytest.mark.gpu


def make_layer(bq, K=2048, N=8192):
    g = torch.Generator().manual_seed(3)
    lin = bq.DecomposedLinear((torch.randn(N, K, generator=g) * 0.02).to(torch.float16).cuda(), [3, 70])
    return lin, torch.ones(K, dtype=torch.float16, device="cuda")


@pytest.mark.parametrize("call", ["linear", "norm_linear"])
def test_a_layer_on_two_streams(bq, call):
    """Calls of one layer that overlap on the device do not see each other's rows."""
    lin, gamma = make_layer(bq)
    run = (lambda x, y=None: lin.linear(x, y_out=y)) if call == "linear" else (lambda x, y=None: lin.norm_linear(x, gamma, 1e-5, y_out=y)[0])
    xs = [[(torch.randn(2048, 2048, device="cuda") * (1 + i + 10 * s)).half() for i in range(4)] for s in range(2)]
    want = []
    for s in range(2):
        want.append([run(x) for x in xs[s]])
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[torch.empty_like(want[0][0]) for _ in range(12)] for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(12):
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                run(xs[s][k % 4], got[s][k])
    torch.cuda.synchronize()
    for s in range(2):
        for k, y in enumerate(got[s]):
            assert torch.equal(y, want[s][k % 4]), (s, k)


@pytest.mark.parametrize("path,dim,block", [(1, 80, 40), (2, 128, 64), (3, 128, 64), (2, 64, 32), (3, 64, 64)])
def test_nothing_but_the_header_has_to_be_zero(bq, path, dim, block):
    c = Case(bq, [900, 0, 70, 333], [1, 1, 3, 2], 2, 4, dim, block, 16, torch.float16)
    want = c.attend(True, path=path)
    for buf, address, nbytes in c.cache._scratch.all("attend"):
        off = address - buf.data_ptr()
        assert not bool(buf[off:off + 1024].any())                  # every call leaves it as it found it
        buf[off + 1024:off + nbytes] = 0xFF
    got = c.attend(True, path=path)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
