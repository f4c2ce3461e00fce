"""GPU tests of the workspaces that a cache and a layer keep between calls: streams, captured graphs, growth."""
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


def replay_after(graph, stream, larger, nbytes):
    """A larger call on the stream of a capture, then the replay; memory that has become free in between (nbytes a piece) is not
    written."""
    with torch.cuda.stream(stream):
        larger()
        free = [torch.full((nbytes + 256,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(8)]
        with torch.cuda.stream(torch.cuda.default_stream()):
            free += [torch.full((nbytes + 256,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        graph.replay()
        stream.synchronize()
        assert all(bool((t == 0x5A).all()) for t in free)


def test_a_captured_layer_call_followed_by_a_larger_one(bq):
    lin, gamma = make_layer(bq)
    x = torch.randn(16, 2048, device="cuda").half()
    want = lin.norm_linear(x, gamma, 1e-5)[0].clone()
    s = torch.cuda.Stream()
    y = torch.empty_like(want)
    with torch.cuda.stream(s):
        lin.norm_linear(x, gamma, 1e-5, y_out=y)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            lin.norm_linear(x, gamma, 1e-5, y_out=y)
    y.zero_()
    replay_after(graph, s, lambda: lin.norm_linear(torch.randn(700, 2048, device="cuda").half(), gamma, 1e-5),
                 lin.workspace_layout(16)[1])
    assert torch.equal(y, want)


def test_a_captured_attention_followed_by_a_larger_one(bq):
    c = Case(bq, [3000, 2900], [2, 2], 2, 2, 128, 64, 16, torch.bfloat16)
    q = c.q.cuda()
    want, _ = c.attend(False, path=2)
    s = torch.cuda.Stream()
    out = torch.empty_like(q)
    with torch.cuda.stream(s):
        c.cache.attend(q, c.starts, 2, out=out, path=2)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.cache.attend(q, c.starts, 2, out=out, path=2)
    out.zero_()
    w = torch.zeros(2, 2, c.cache.capacity, device="cuda")
    need, = c.cache._need.values()                                   # one size so far
    replay_after(graph, s, lambda: c.cache.attend(torch.randn(900, 4, 128, device="cuda").bfloat16(), torch.tensor([0, 450, 900], dtype=torch.int32, device="cuda"),
                                                  450, weights=w, path=2), need)
    assert torch.equal(out, want)
    assert c.cache.kernel_status() == 0


@pytest.mark.parametrize("path", [1, 2, 3])
def test_graphs_without_a_call_before_them(bq, path):
    """Captured on a stream that no call has used: each graph is whole, whatever the order of replays, and calls outside of graphs
    on that stream find a workspace of their own."""
    c = Case(bq, [900, 70, 333], [1, 3, 2], 2, 4, 128, 64, 16, torch.bfloat16)
    q = c.q.cuda()
    want, want_w = c.attend(True, path=path)
    s = torch.cuda.Stream()
    outs, ws, graphs = [], [], []
    for _ in range(3):
        outs.append(torch.zeros_like(q))
        ws.append(torch.full_like(want_w, 0.25))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            c.cache.attend(q, c.starts, 3, weights=ws[-1], out=outs[-1], path=path)
    for i in (2, 0, 1):
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want) and torch.equal(ws[i], want_w), i
    with torch.cuda.stream(s):
        out, w = c.attend(True, path=path)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(w, want_w)


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
