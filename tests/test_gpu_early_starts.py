"""Chains of calls over the same buffers, nothing waiting in between: each kernel starts under the one before, which still writes what it reads."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("news,heads,dim,block", [([1] * 4, 8, 128, 64), ([1, 70, 0, 5], 4, 64, 32), ([3] * 4, 2, 80, 40), ([1] * 4, 32, 128, 32)])
def test_projection_store_and_attention(bq, news, heads, dim, block, dtype):
    """A step's rows are projected into one buffer, whose queries are turned in place, stored and attended with; the buffer is the next step's too."""
    H, steps, hidden = 2, 10, 256
    g = torch.Generator().manual_seed(6)
    lin = bq.DecomposedLinear((torch.randn((heads + 2 * H) * dim, hidden, generator=g) * hidden ** -0.5).to(dtype).cuda(), ())
    xs = [(torch.randn(sum(news), hidden, generator=g) * (i + 1)).to(dtype).cuda() for i in range(steps)]
    n = sum(news)
    starts = torch.tensor([sum(news[:i]) for i in range(5)], dtype=torch.int32, device="cuda")
    more = starts[1:] - starts[:-1]
    rotary = bq.Rotary(dim)

    def run(wait, graph):
        cb = bq.Codebook4()
        prefix, cache = bq.KvCache4.empty(1, 500, H, dim, block, cb), bq.KvCache4.empty(4, 1024, H, dim, block, cb)
        rows = torch.randn(500, H, dim, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
        prefix.lens.fill_(500)
        prefix.append(rows, rows.flip(0), torch.tensor([0, 500], dtype=torch.int32, device="cuda"))
        qkv, outs = torch.empty(n, (heads + 2 * H) * dim, dtype=dtype, device="cuda"), [torch.empty(n, heads, dim, dtype=dtype, device="cuda") for _ in range(steps)]

        def chain():
            for i in range(steps):
                cache.lens.add_(more)
                lin.linear(xs[i], y_out=qkv)
                q, k, v = qkv.view(n, heads + 2 * H, dim).split((heads, H, H), dim=1)
                cache.append_rotary(q, k, v, rotary, None, starts, q)
                cache.attend_shared(q, prefix, None, starts, max(news), 0, out=outs[i])
                if wait:
                    torch.cuda.synchronize()

        chain()
        if graph:                                                      # all of it again, over what the first time left
            cache.lens.zero_()
            for o in outs:
                o.zero_()
            torch.cuda.synchronize()
            replayed = torch.cuda.CUDAGraph()
            with torch.cuda.graph(replayed):
                chain()
            replayed.replay()
        torch.cuda.synchronize()
        assert cache.kernel_status() == 0
        return outs + [cache.lens] + list(cache._pools)

    want = run(True, False)
    for graph in (False, True):
        assert all(torch.equal(a, b) for a, b in zip(run(False, graph), want))
