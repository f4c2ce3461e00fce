"""GPU tests of attention behind shared prefixes (bqkv_attend_shared of include/bq4.h) against the oracle in 64 bits.

The tolerances are those of tests/test_gpu_kvcache.py (there derived): each side's products and probabilities are rounded as there,
and the join multiplies the sides by factors that are off by a few 2^-23, which its 2^-10 covers.
"""
import math

import numpy as np
import pytest
import torch

from oracle import shared_oracle as so
from paper_2407_19775_b200.binding import BqError
from test_gpu_kvcache import HALF_ULP, SHAPES, TINY, Case

pytestmark = pytest.mark.gpu


class Shared:
    def __init__(self, bq, plens, members, lens, news, h, g, dim, block, page, tdt, seed=0, prefix_page=None, scale=1.0, prefix_scale=1.0):
        self.own = Case(bq, lens, news, h, g, dim, block, page, tdt, seed=seed, scale=scale)
        self.pre = Case(bq, plens, [0] * len(plens), h, g, dim, block, prefix_page or page, tdt, seed=seed + 1, scale=prefix_scale)
        self.members_host = members
        self.members = None if members is None else torch.tensor(members, dtype=torch.int32, device="cuda")
        self.tdt, self.dim, self.g, self.h = tdt, dim, g, h

    def prefix_of(self, s):
        if self.members_host is None:
            return 0
        at = [p for p in range(len(self.members_host) - 1) if self.members_host[p] <= s < self.members_host[p + 1]]
        return at[0] if at else None

    def attend(self, weights=False, path=0, q=None, **kw):
        c = self.own
        w = torch.full((len(c.lens), self.h, c.cache.capacity), 0.25, device="cuda") if weights else None
        args = dict(max_new=max(1, max(c.news)), weights=w, path=path)
        args.update(kw)
        out = c.cache.attend_shared(c.q.cuda() if q is None else q, self.pre.cache, self.members, c.starts, **args)
        torch.cuda.synchronize()
        assert c.cache.kernel_status() == 0
        return out, w

    def check(self, out, w=None, sm=None):
        c = self.own
        sm = 1 / math.sqrt(self.dim) if sm is None else sm
        got, qd = out.double().cpu().numpy(), c.q.double().numpy()
        for s, (k, v) in enumerate(c.values):
            lo, hi = c.starts_host[s], c.starts_host[s + 1]
            p = self.prefix_of(s)
            kp, vp = self.pre.values[p] if p is not None else (k[:0], v[:0])
            ref = so.attend(qd[lo:hi], kp, vp, k, v, sm)
            ds = (self.dim + 8) * 2.0 ** -22 * ref["spread"][..., None]
            tol = HALF_ULP[self.tdt] * np.abs(ref["out"]) + TINY[self.tdt] + (2.0 ** -10 + 2 * ds) * ref["mass"] * (1 + HALF_ULP[self.tdt])
            err = np.abs(got[lo:hi] - ref["out"])
            assert np.all(err <= tol), (s, float(np.nanmax(err / np.maximum(tol, 1e-30))), int(np.isnan(got[lo:hi]).sum()))
            if w is not None:
                n = c.lens[s]
                got_w = w[s].double().cpu().numpy() - 0.25
                wtol = 2 * (self.dim + 8) * 2.0 ** -22 * ref["heavy"] + (2 * (hi - lo) * self.g + 16) * 2.0 ** -23 * (ref["weights"] + 0.25)
                werr = np.abs(got_w[:, :n] - ref["weights"])
                assert np.all(werr <= wtol), (s, float((werr / np.maximum(wtol, 1e-30)).max()))
                assert np.all(got_w[:, n:] == 0)


def fits(dim, block, page, path):
    return path < 2 or (page % 16 == 0 and (dim, block) in ((64, 64), (64, 32), (128, 128), (128, 64), (128, 32)))


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,g,dim,block,page", SHAPES)
@pytest.mark.parametrize("path", [0, 1, 2, 3])
def test_single_tokens_behind_one_prefix(bq, h, g, dim, block, page, tdt, path):
    """Sequences without own slots, with one, and around tiles; prefixes around tiles and pages."""
    if not fits(dim, block, page, path):
        pytest.skip("not a shape of this kernel")
    lens = [1, 0, 2, 17, 63, 64, 65, 130]
    for plen in (300, 1, 64):
        c = Shared(bq, [plen], None, lens, [1] * len(lens), h, g, dim, block, page, tdt, seed=dim + page + g)
        for weights in (False, True):
            c.check(*c.attend(weights, path=path))


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,g,dim,block,page", SHAPES)
@pytest.mark.parametrize("path", [0, 2, 3])
def test_ragged_rows_and_several_prefixes(bq, h, g, dim, block, page, tdt, path):
    """Prefixes of no slots, of nobody; sequences that share none, without rows, with more rows than slots."""
    if not fits(dim, block, page, path):
        pytest.skip("not a shape of this kernel")
    lens, news = [5, 40, 0, 70, 33, 3, 129, 9], [5, 1, 0, 3, 33, 9, 2, 9]
    c = Shared(bq, [200, 0, 77, 31], [1, 3, 4, 4, 7], lens, news, h, g, dim, block, page, tdt, seed=dim + page)
    for weights in (False, True):
        c.check(*c.attend(weights, path=path))


@pytest.mark.parametrize("h,g,dim,block,page,tdt", [(2, 4, 128, 128, 64, torch.bfloat16), (1, 7, 64, 64, 32, torch.float16), (2, 1, 128, 64, 16, torch.float16)])
@pytest.mark.parametrize("path", [0, 2, 3])
def test_many_rows_and_long_prefixes(bq, h, g, dim, block, page, tdt, path):
    lens, news = [130, 300, 257, 1], [130, 150, 30, 1]
    c = Shared(bq, [1500, 900], [0, 2, 4], lens, news, h, g, dim, block, page, tdt, seed=11, prefix_page=32)
    for weights in (False, True):
        c.check(*c.attend(weights, path=path))


@pytest.mark.parametrize("path", [0, 1, 2, 3])
def test_sides_of_very_different_size(bq, path):
    """One side's scores, or values, far above the other's: each way round."""
    for scale, prefix_scale in ((8.0, 2.0 ** -30), (2.0 ** -30, 8.0), (2.0 ** -60, 2.0 ** -60)):
        c = Shared(bq, [200], None, [100, 3, 1], [2, 1, 1], 2, 4, 128, 64, 16, torch.bfloat16, seed=5, scale=scale, prefix_scale=prefix_scale)
        out, _ = c.attend(path=path)
        c.check(out)


@pytest.mark.parametrize("path", [0, 1, 2, 3])
def test_bounds_that_are_too_small_and_other_arguments(bq, path):
    """The bounds size launches only; the scale may be negative; queries are a slice of a projection."""
    lens, news = [300, 20, 7], [9, 20, 1]
    c = Shared(bq, [700, 90], [0, 2, 3], lens, news, 2, 4, 128, 64, 16, torch.float16, seed=3)
    wide = torch.zeros(30, 12 * 128, dtype=torch.float16, device="cuda")
    wide[:, 256:256 + 8 * 128] = c.own.q.cuda().view(30, -1)
    q = wide[:, 256:256 + 8 * 128].unflatten(1, (8, 128))
    for kw in (dict(max_new=1, max_len=16, max_shared=1, max_prefix=16), dict(max_new=100, max_len=1 << 20, max_shared=1 << 20, max_prefix=1 << 20)):
        out, w = c.attend(True, path, q, **kw)
        c.check(out, w)
    out, _ = c.attend(path=path, sm_scale=-0.2)
    c.check(out, sm=-0.2)


@pytest.mark.parametrize("path", [0, 1, 2, 3])
def test_as_one_sequence(bq, path):
    """Prefix and own slots over one pool: what attend gives for the sequences with all their slots, within the tolerances of both."""
    whole = Case(bq, [80 + 16 * i for i in range(4)], [1, 3, 1, 2], 2, 4, 128, 64, 16, torch.bfloat16, seed=8)
    # the first four pages of sequence 0 are everybody's beginning
    table = whole.cache.table.clone()
    table[:, :4] = table[0, :4]
    for s in range(1, 4):
        for t in (0, 1):
            whole.values[s][t][:64] = whole.values[0][t][:64]
    lens = whole.cache.lens
    full = bq.KvCache4(*whole.pools, table, lens, bq.Codebook4())
    own = bq.KvCache4(*whole.pools, table[:, 4:], lens - 64, bq.Codebook4())
    prefix = bq.KvCache4(*whole.pools, table[:1, :4], torch.tensor([64], dtype=torch.int32, device="cuda"), bq.Codebook4())
    q = whole.q.cuda()
    whole.check(full.attend(q, whole.starts, 3))
    whole.check(own.attend_shared(q, prefix, None, whole.starts, 3, path=path))


def test_rows_of_no_sequence_stay(bq):
    for path in (2, 3):
        c = Shared(bq, [100], None, [30, 5], [2, 1], 2, 4, 128, 64, 16, torch.float16)
        q = torch.cat([c.own.q, torch.full((2, 8, 128), 9.0, dtype=torch.float16)]).cuda()
        out = torch.full_like(q, 7.0)
        got = c.own.cache.attend_shared(q, c.pre.cache, None, c.own.starts, 2, out=out, path=path)
        assert got is out and bool((out[3:] == 7.0).all())
        c.check(out[:3])


@pytest.mark.parametrize("path", [0, 2, 3])
def test_in_place_same_bits_twice_and_captured(bq, path):
    c = Shared(bq, [600, 70], [0, 3, 5], [40, 9, 100, 3, 64], [1] * 5, 2, 8, 128, 64, 16, torch.bfloat16, seed=2)
    out, _ = c.attend(path=path)
    again, _ = c.attend(path=path)
    assert torch.equal(out, again)
    q = c.own.q.cuda()
    c.own.cache.attend_shared(q, c.pre.cache, c.members, None, out=q, path=path)
    assert torch.equal(q, out)
    q = c.own.q.cuda()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = c.own.cache.attend_shared(q, c.pre.cache, c.members, None, path=path)
    for _ in range(2):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, out)
    assert c.own.cache.kernel_status() == 0


def test_more_rows_than_blocks_of_the_general_kernel(bq):
    """Rows of one sequence in more blocks than the launch has CTAs for a sequence; the other sequences have one row."""
    news = [700] + [1] * 9
    c = Shared(bq, [50, 33], [0, 1, 10], [n + 5 for n in news], news, 16, 1, 24, 8, 7, torch.float16, seed=4)
    for kw in ({}, dict(max_new=1, max_shared=1)):
        out, w = c.attend(True, **kw)
        c.check(out, w)


@pytest.mark.parametrize("dim,block,page", [(128, 64, 16), (80, 40, 9)])
def test_masked_slots_of_the_general_kernel_stay_out(bq, dim, block, page):
    """Values of infinity and NaN (which nothing that was stored from finite rows holds) in the slot of a sequence's last row are that row's alone."""
    for bad in (math.inf, math.nan):
        lens, news = [70, 9], [6, 9]
        c = Shared(bq, [90], None, lens, news, 2, 4, dim, block, page, torch.bfloat16, seed=6)
        want, _ = c.attend(path=1)
        table = c.own.cache.table.cpu()
        for s, n in enumerate(lens):
            c.own.pools[3][int(table[s, (n - 1) // page]), :, (n - 1) % page] = bad
        got, _ = c.attend(path=1)
        last = (c.own.starts[1:] - 1).long()
        rest = torch.ones(15, dtype=torch.bool, device="cuda")
        rest[last] = False
        assert torch.equal(got[rest], want[rest]) and not bool(got[last].isfinite().all())


@pytest.mark.parametrize("dim,block,page", [(128, 64, 16), (80, 40, 9)])
def test_members_out_of_range_and_rows_of_no_sequence(bq, dim, block, page):
    c = Shared(bq, [60, 20], [0, 2, 3], [30, 5, 8], [2, 1, 3], 2, 4, dim, block, page, torch.float16, seed=9)
    want, _ = c.attend()
    q = torch.cat([c.own.q, torch.full((3, 8, dim), 9.0, dtype=torch.float16)]).cuda()
    for path in (0, 1):
        c.members = torch.tensor([-5, 2, 1000], dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.0)
        c.own.cache.attend_shared(q, c.pre.cache, c.members, c.own.starts, 3, out=out, path=path)
        assert bool((out[6:] == 7.0).all())
        c.check(out[:6])
    assert torch.equal(out[:6], want) or dim == 128


def test_general_in_place_twice_and_captured(bq):
    c = Shared(bq, [600, 70], [0, 3, 5], [40, 9, 100, 3, 64], [1] * 5, 2, 5, 80, 40, 16, torch.bfloat16, seed=2)
    out, _ = c.attend()
    c.check(out)
    assert torch.equal(out, c.attend()[0])
    q = c.own.q.cuda()
    c.own.cache.attend_shared(q, c.pre.cache, c.members, None, out=q)
    assert torch.equal(q, out)
    q = c.own.q.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        y = c.own.cache.attend_shared(q, c.pre.cache, c.members, None)
    for _ in range(2):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, out)


@pytest.mark.parametrize("dim,block", [(128, 64), (80, 40)])
def test_two_graphs_of_one_cache_and_a_call_in_between(bq, dim, block):
    """Two captured calls of different sizes and an eager one, replayed in any order, keep out of each other's workspace."""
    c = Shared(bq, [300], None, [40, 9, 100], [1] * 3, 2, 4, dim, block, 16, torch.bfloat16, seed=2)
    qs = [torch.randn(3, 8, dim, generator=torch.Generator().manual_seed(i)).bfloat16().cuda() for i in range(3)]
    call = lambda q, **kw: c.own.cache.attend_shared(q, c.pre.cache, None, None, **kw)
    kws = (dict(path=0), dict(path=1), dict(max_len=16, max_prefix=64))
    want = [call(q, **kw) for q, kw in zip(qs, kws)]
    graphs, ys = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph, q, kw in zip(graphs, qs, kws):
        with torch.cuda.graph(graph):
            ys.append(call(q, **kw))
    for order in ((0, 1), (1, 0), (1, 1, 0, 0)):
        for y in ys:
            y.zero_()
        for k in order:
            graphs[k].replay()
            assert torch.equal(call(qs[2], **kws[2]), want[2])
        torch.cuda.synchronize()
        assert torch.equal(ys[0], want[0]) and torch.equal(ys[1], want[1])


def test_no_rows(bq):
    c = Shared(bq, [20], None, [5, 0], [0, 0], 2, 4, 128, 64, 16, torch.float16)
    q = torch.empty(0, 8, 128, dtype=torch.float16, device="cuda")
    for path in (0, 1, 2, 3):
        assert c.own.cache.attend_shared(q, c.pre.cache, None, c.own.starts, path=path).shape == (0, 8, 128)
    k = torch.empty(0, 2, 128, dtype=torch.float16, device="cuda")
    before = [t.clone() for t in c.own.pools]
    assert c.own.cache.append_rotary(q, k, k, bq.Rotary(128), None, c.own.starts).shape == (0, 8, 128)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, c.own.pools))


def test_refusals(bq):
    c = Shared(bq, [100, 20], [0, 1, 2], [30, 5], [1, 1], 2, 4, 128, 64, 16, torch.float16)
    q = c.own.q.cuda()
    other = Case(bq, [5], [0], 2, 4, 128, 32, 16, torch.float16)
    linear = np.arange(-8, 8, dtype=np.float32) / 8
    book = Case(bq, [5, 5], [0, 0], 2, 4, 128, 64, 16, torch.float16, values=linear)
    call = c.own.cache.attend_shared
    for bad in (dict(members=None), dict(members=c.members.long()), dict(members=c.members[:2]), dict(members=c.members.cpu()), dict(prefix=other.cache, members=None),
                dict(prefix=book.cache), dict(q=q[:1]), dict(q=q[:, :3]), dict(q=q.float()), dict(out=q.bfloat16()), dict(path=4), dict(path=-1),
                dict(weights=torch.zeros(2, 2, 9, device="cuda")[:, :, ::2]), dict(weights=torch.zeros(2, 2, 64, device="cuda"), out=q), dict(sm_scale=math.inf)):
        with pytest.raises(BqError):
            call(**{**dict(q=q, prefix=c.pre.cache, members=c.members), **bad})
