"""GPU tests of low-rank adapters beside a decomposed layer (mmd_linear_adapted, mmd_norm_linear_adapted of include/mmd.h).

The layer's own value is bit-exact where it has no critical features (the integer sums are); with them its fp32 side sum is off by up to
(side columns + 2) 2^-22 sum |x w| as in tests/test_gpu_norm.py.  The adapters' part against 64 bits, with S_j = sum_k |x_k A_jk| and
v_j = scale u_j:

    |u_j - exact| <= (K + 16) 2^-24 S_j x 2        K products summed in fp32 in some order; tensor-core sums may truncate: twice
    |sum_j v_j B_j - exact| <= scale sum_j |B_j| (that) + (rank + 3) 2^-24 sum_j |v_j B_j|      (v's rounding, the products' and the sums')

and the whole one rounding to the output's type behind that.  Where the first product's numbers are carried in two 16-bit parts, of bf16
16 bits: 2^-16 of v_j instead of its fp32 rounding.  With the norm x is the normed row in its 16-bit type: its factor 1 / rms is off by
(K / 512 + 16) 2^-24 (derived in tests/test_gpu_norm.py), which moves an element across a rounding border now and then: half an ulp
more in every x_k, ulp of the type.
"""
import numpy as np
import pytest
import torch

from oracle import mmd_oracle as mo
from oracle import norm_oracle as no
from paper_2407_19775_b200.binding import BqError
from test_gpu_norm import DT, HALF_ULP, bits, make

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, bq, K, N, ko, count, rank, tdt, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.K, self.N, self.tdt, self.rank, self.count = K, N, tdt, rank, count
        self.W = (torch.randn(N, K, generator=g) * 0.02).to(tdt)
        self.idx = torch.randperm(K, generator=g)[:ko].sort().values.int()
        self.lin = bq.DecomposedLinear(self.W.cuda(), self.idx.numpy())
        self.a = (torch.randn(count, rank, K, generator=g) * K ** -0.5).to(tdt)
        self.b = (torch.randn(count, N, rank, generator=g) * 0.3).to(tdt)
        self.scale = torch.rand(count, generator=g) * 2 - 0.5
        self.ad = bq.Adapters(self.a.cuda(), self.b.cuda(), self.scale.cuda())
        self.qw, self.sw, self.wo = mo.rowquant(bits(self.W), DT[tdt], self.idx.numpy())

    def rows(self, M, seed=1):
        x = torch.randn(M, self.K, generator=torch.Generator().manual_seed(seed)) * 0.5
        x[:, self.idx.long()] *= 30
        if M > 2:
            x[1] = 0
        return x.to(self.tdt)

    def base(self, q, s32, side_x):
        """The layer's own value in 64 bits, and the error of its side sum."""
        acc = mo.int_product(q, self.qw).astype(np.float32).astype(np.float64)
        side_w = mo.widen(self.wo, DT[self.tdt]).astype(np.float64)
        want = acc * (s32[:, None] * self.sw[None, :].astype(np.float64)).astype(np.float32).astype(np.float64) + side_x @ side_w.T
        return want, 2.0 ** -23 * np.abs(want) + (self.wo.shape[1] + 2) * 2.0 ** -22 * (np.abs(side_x) @ np.abs(side_w).T)

    def check(self, y, base, base_tol, x, ids, starts, x_ulp=0.0):
        """y against base + adapters of x (float64) by sequence; x_ulp: relative error of x's elements."""
        want, tol = base.copy(), base_tol.copy()
        for s, a in enumerate(ids):
            lo, hi = (s, s + 1) if starts is None else (starts[s], starts[s + 1])
            if not 0 <= a < self.count or hi <= lo:
                continue
            A, B, sc = self.a[a].double().numpy(), self.b[a].double().numpy(), float(self.scale[a])
            v = sc * (x[lo:hi] @ A.T)
            du = np.abs(x[lo:hi]) @ np.abs(A).T * (2 * (self.K + 16) * 2.0 ** -24 + x_ulp)
            want[lo:hi] += v @ B.T
            split = 2.0 ** -16 if self.tdt == torch.bfloat16 else 2.0 ** -21
            tol[lo:hi] += abs(sc) * (du @ np.abs(B).T) + (self.rank + 3) * 2.0 ** -24 * (np.abs(v) @ np.abs(B).T) + split * (np.abs(v) @ np.abs(B).T)
        tol += 2.0 ** -23 * np.abs(want)
        if y.dtype != torch.float32:
            tol += HALF_ULP[y.dtype] * (np.abs(want) + tol) + 2.0 ** -25
        err = np.abs(y.double().cpu().numpy() - want)
        assert np.all(err <= tol), float((err / np.maximum(tol, 1e-30)).max())

    def linear(self, x, ids, starts=None, **kw):
        st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
        y = self.lin.linear(x.cuda(), adapters=self.ad, ids=torch.tensor(ids, dtype=torch.int32, device="cuda"), starts=st, **kw)
        torch.cuda.synchronize()
        assert self.lin.kernel_status() == 0
        q, s, side = mo.rowquant(bits(x), DT[self.tdt], self.idx.numpy())
        base, tol = self.base(q, s.astype(np.float64), mo.widen(side, DT[self.tdt]).astype(np.float64))
        self.check(y, base, tol, x.double().numpy(), ids, starts)
        return y


SIZES = [                                                            # K, N, critical, adapters, rank
    (320, 72, 3, 3, 16), (2048, 1024, 8, 5, 16), (1040, 2056, 0, 2, 32), (640, 264, 40, 4, 64), (16, 8, 0, 1, 16), (48, 77, 1, 2, 16), (8192, 512, 8, 9, 48), (256, 256, 0, 3, 256)]


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("K,N,ko,count,rank", SIZES)
def test_single_rows(bq, K, N, ko, count, rank, tdt):
    """A row per sequence: every adapter, the same one twice, none (-1, past the end, far away)."""
    c = Layer(bq, K, N, ko, count, rank, tdt)
    ids = [0, count - 1, -1, 0, count, 1 % count, 2 ** 31 - 1, -2 ** 31]
    for M in (1, 3, 8):
        for out in (tdt, torch.float32):
            c.linear(c.rows(M), ids[:M], out_dtype=out)
    c.linear(c.rows(64), [i % (count + 1) for i in range(64)])


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("K,N,ko,count,rank", SIZES)
def test_ragged_sequences(bq, K, N, ko, count, rank, tdt):
    """Sequences of no rows, one, around the tiles; rows before the first and behind the last."""
    c = Layer(bq, K, N, ko, count, rank, tdt, seed=2)
    news = [0, 1, 31, 32, 33, 0, 65, 7]
    starts = [3 + sum(news[:i]) for i in range(len(news) + 1)]
    ids = [0, count - 1, -1, 0, 1 % count, 0, count // 2, count + 3]
    c.linear(c.rows(starts[-1] + 5), ids, starts)


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("K,N,ko,count,rank,news", [(1024, 2048, 6, 3, 16, [700, 1, 0, 499, 133]), (512, 4096, 0, 2, 64, [1100, 37]), (2048, 2304, 20, 5, 32, [90] * 15),
                                                    (1024, 4104, 5, 12, 16, [130] * 10), (272, 4096, 2, 3, 48, [1000, 200, 77])])
def test_prompts(bq, K, N, ko, count, rank, news, tdt):
    c = Layer(bq, K, N, ko, count, rank, tdt, seed=3)
    starts = [sum(news[:i]) for i in range(len(news) + 1)]
    ids = [(3 * i + 1) % (count + 1) - (i == 2) for i in range(len(news))]
    x = c.rows(starts[-1])
    for out in (tdt, torch.float32):
        c.linear(x, ids, starts, out_dtype=out)


@pytest.mark.parametrize("path", [0, 1, 2, 3, 4])
def test_every_path(bq, path):
    c = Layer(bq, 512, 4096, 4, 3, 16, torch.bfloat16, seed=4)
    starts = [0, 300, 300, 1000, 1281]
    c.linear(c.rows(1281), [2, 0, -1, 1], starts, path=path)


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,K,N,ko,rank", [(1, 320, 72, 3, 16), (37, 320, 72, 0, 32), (64, 2048, 1024, 8, 16), (300, 1024, 2048, 16, 16), (130, 640, 264, 40, 64), (1200, 512, 4096, 5, 16)])
@pytest.mark.parametrize("residual", [True, False])
def test_behind_the_norm(bq, M, K, N, ko, rank, tdt, residual):
    c = Layer(bq, K, N, ko, 3, rank, tdt, seed=5)
    x, res, gamma, _ = make(M, K, 0, tdt, M + K, residual)
    news = [M // 3, 0, M - M // 3 - M // 5, M // 5]
    starts, ids = [sum(news[:i]) for i in range(5)], [2, 1, 0, -1]
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    y, h = c.lin.norm_linear(x.cuda(), gamma.cuda(), 1e-5, residual=None if res is None else res.cuda(), adapters=c.ad,
                             ids=torch.tensor(ids, dtype=torch.int32, device="cuda"), starts=st)
    torch.cuda.synchronize()
    ref = no.norm_rowquant(bits(x), None if res is None else bits(res), bits(gamma[None])[0], 1e-5, DT[tdt], c.idx.numpy())
    assert np.array_equal(bits(h), ref["h"])
    rel = (K / 512 + 16) * 2.0 ** -24
    base, tol = c.base(ref["q"], ref["scale"], ref["side"])
    tol += rel * np.abs(base) + (2 * HALF_ULP[tdt] + rel) * (np.abs(ref["side"]) @ np.abs(mo.widen(c.wo, DT[tdt]).astype(np.float64)).T)
    c.check(y, base, tol, ref["normed"], ids, starts, x_ulp=2 * HALF_ULP[tdt] + rel)


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("K,N", [(512, 4099), (272, 1001), (2048, 129), (1024, 77), (8192, 66), (512, 2047)])
def test_columns_that_are_no_multiple_of_eight(bq, K, N, tdt):
    """They lie eight apart in the workspace on their way; every kernel of the product, and both kernels behind it."""
    c = Layer(bq, K, N, 5, 3, 32, tdt, seed=6)
    for news, n in (([700, 1, 0, 600], 1301), ([90, 0, 40, 3], 133), ([1] * 40, 40)):
        starts = [sum(news[:i]) for i in range(len(news) + 1)]
        ids = [i % 4 - (i == 3) for i in range(len(news))]
        x = c.rows(n)
        for out in (tdt, torch.float32):
            c.linear(x, ids, starts, out_dtype=out)
    flat = torch.full((133 * N + 9,), 7.0, dtype=tdt, device="cuda")     # results at an odd place, and nothing behind them
    news = [90, 0, 40, 3]
    c.linear(c.rows(133), [0, 1, 2, -1], [sum(news[:i]) for i in range(5)], y_out=flat[1:1 + 133 * N].view(133, N))
    assert bool((flat[:1] == 7).all()) and bool((flat[1 + 133 * N:] == 7).all())


def test_rows_without_an_adapter_are_the_layers_own(bq):
    for M, n in ((64, 64), (1300, 4)):
        c = Layer(bq, 512, 4096, 3, 2, 16, torch.float16)
        x = c.rows(M).cuda()
        ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")
        starts = torch.arange(n + 1, dtype=torch.int32, device="cuda") * (M // n)
        assert torch.equal(c.lin.linear(x, adapters=c.ad, ids=ids, starts=starts), c.lin.linear(x))


def test_same_bits_twice_in_a_chain_captured_and_on_another_stream(bq):
    c = Layer(bq, 2048, 2048, 8, 6, 16, torch.float16)
    xs = [(c.rows(64, seed=i) * (i + 1)).cuda() for i in range(5)]
    ids = torch.tensor([i % 7 - 1 for i in range(64)], dtype=torch.int32, device="cuda")
    want = []
    for x in xs:
        want.append(c.lin.linear(x, adapters=c.ad, ids=ids).clone())
        torch.cuda.synchronize()
    got = [c.lin.linear(x, adapters=c.ad, ids=ids) for x in xs]       # nothing waits in between
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(want[0]) for _ in range(10)]
    torch.cuda.synchronize()
    for i in range(5):                                               # two streams at once
        c.lin.linear(xs[i], adapters=c.ad, ids=ids, y_out=outs[i])
        with torch.cuda.stream(side):
            c.lin.linear(xs[4 - i], adapters=c.ad, ids=ids, y_out=outs[5 + i])
    torch.cuda.synchronize()
    assert all(torch.equal(outs[i], want[i]) and torch.equal(outs[5 + i], want[4 - i]) for i in range(5))
    x, y = xs[0].clone(), torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.lin.linear(x, adapters=c.ad, ids=ids, y_out=y)
    for i in (3, 1):
        x.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])


def test_ids_and_starts_written_by_the_kernel_before(bq):
    """A call sees what was written to its ids and starts by the kernels in front of it, in a replayed graph too."""
    c = Layer(bq, 1024, 264, 3, 6, 16, torch.bfloat16)
    g = torch.Generator().manual_seed(5)
    x = c.rows(48).cuda()
    who = torch.randint(-1, 6, (20, 48), generator=g).int().cuda()
    cuts = torch.cat([torch.zeros(20, 1), torch.sort(torch.randint(0, 49, (20, 47), generator=g).float(), dim=1).values, torch.full((20, 1), 48.0)], 1).int().cuda()
    for starts in (None, cuts[0].clone()):
        ids, want = who[0].clone(), []
        for i in range(20):
            at = None if starts is None else cuts[i].clone()
            torch.cuda.synchronize()
            want.append(c.lin.linear(x, adapters=c.ad, ids=who[i].clone(), starts=at))
            torch.cuda.synchronize()
        got = [torch.empty_like(want[0]) for _ in range(20)]
        for i in range(20):
            ids.copy_(who[i])
            if starts is not None:
                starts.copy_(cuts[i])
            c.lin.linear(x, adapters=c.ad, ids=ids, starts=starts, y_out=got[i])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for i in range(20):
                ids.copy_(who[i])
                if starts is not None:
                    starts.copy_(cuts[i])
                c.lin.linear(x, adapters=c.ad, ids=ids, starts=starts, y_out=got[i])
        for y in got:
            y.zero_()
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_contents_may_change_and_ranks_are_padded(bq):
    g = torch.Generator().manual_seed(1)
    pairs = [((torch.randn(r, 320, generator=g) * 0.05).half().cuda(), (torch.randn(72, r, generator=g) * 0.3).half().cuda()) for r in (4, 16, 1, 23)]
    ad = bq.Adapters.pack(pairs, [1.0, 0.5, -2.0, 1.5])
    assert ad.rank == 32 and ad.count == 4
    c = Layer(bq, 320, 72, 3, 4, 32, torch.float16)
    for t in (0, 1, 2):
        assert c.ad._tensors[t].shape == ad._tensors[t].shape
        c.ad._tensors[t].copy_(ad._tensors[t])
    c.a, c.b, c.scale = (t.cpu() for t in ad._tensors)
    c.linear(c.rows(9), [0, 1, 2, 3, 3, 2, 1, 0, -1])


def test_refusals(bq):
    c = Layer(bq, 320, 72, 3, 3, 16, torch.float16)
    x, ids = c.rows(4).cuda(), torch.zeros(4, dtype=torch.int32, device="cuda")
    starts = torch.arange(5, dtype=torch.int32, device="cuda")
    a, b, s = c.ad._tensors
    other = Layer(bq, 320, 80, 0, 3, 16, torch.float16).ad
    good = dict(X=x, adapters=c.ad, ids=ids, starts=starts)
    for bad in (dict(ids=None), dict(ids=ids.long()), dict(ids=ids[:3]), dict(ids=ids.cpu()), dict(ids=ids[:3], starts=None), dict(starts=starts.long()), dict(starts=starts[:4]),
                dict(starts=starts.cpu()), dict(adapters=other), dict(adapters=None), dict(path=5), dict(path=6), dict(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(BqError):
            c.lin.linear(**{**good, **bad})
    gamma = torch.ones(320, dtype=torch.float16, device="cuda")
    for bad in (dict(ids=None), dict(ids=ids[:3], starts=None), dict(adapters=other), dict(path=5), dict(adapters=None)):
        with pytest.raises(BqError):
            c.lin.norm_linear(**{**good, **bad}, gamma=gamma, eps=1e-5)
    for args in ((a[:, :8].contiguous(), b[:, :, :8].contiguous(), s), (a, b[:2], s), (a, b, s[:2]), (a, b, s.double()), (a.float(), b.float(), s), (a, b.bfloat16(), s),
                 (a[:, :, ::2], b, s), (a[:0], b[:0], s[:0]), (a.repeat(1, 17, 1), b.repeat(1, 1, 17), s)):
        with pytest.raises(BqError):
            bq.Adapters(*args)
    empty = c.lin.linear(x[:0], adapters=c.ad, ids=ids[:1], starts=torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert empty.shape == (0, 72)
