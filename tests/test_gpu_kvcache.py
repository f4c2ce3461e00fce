"""GPU tests of the 4-bit key/value cache (the bqkv_* calls of include/bq4.h) against the oracle in 64 bits.

Store and read are exact: the codec's bits.  Evictions are exact: whole rows move.  Attention is compared within

    tol = ulp/2 of the output type at |out| + (2^-10 + 2 ds) sum_j p_j |v_j|,   ds = (dim + 8) 2^-22 max_j sm sum_d |q_d k_jd|

ulp/2: the one rounding to the output type; ds: the error of a score (one rounding per accumulated product and for the few
factors behind it, times 4 for tensor-core sums that truncate), which moves a probability by a relative ds and the softmax sum
by as much again; 2^-10: probabilities and scaled values that enter the second product rounded to 11 bits each (2^-12 + 2^-12 on
average, 2^-11 + 2^-11 at most).  Accumulated weights are fp32 sums of probabilities: tol = sum_rows p (2 ds + (rows + 16) 2^-23).
"""
import math

import numpy as np
import pytest
import torch

from oracle import bq4_oracle as o4
from oracle import kvcache_oracle as ko
from paper_2407_19775_b200 import workloads
from paper_2407_19775_b200.binding import BqError

pytestmark = pytest.mark.gpu
DT = {torch.float16: o4.F16, torch.bfloat16: o4.BF16}
HALF_ULP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}       # 11 and 8 significant bits, to nearest
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}


def bits(t: torch.Tensor) -> np.ndarray:
    return workloads.as_numpy_bits(t.detach().cpu().contiguous().reshape(-1)).reshape(tuple(t.shape))


class Case:
    """A cache with shuffled pages whose unused rows hold NaN scales, its rows in 64 bits, and queries."""

    def __init__(self, bq, lens, news, kv_heads, group, dim, block, page, tdt, seed=0, scale=1.0, pad_pages=2, values=None):
        g = torch.Generator().manual_seed(seed)
        self.tdt, self.lens, self.news, self.dim, self.group, self.h = tdt, lens, news, dim, group, kv_heads
        self.cb_ref = o4.make_codebook() if values is None else np.asarray(values, np.float32)
        cb = bq.Codebook4() if values is None else bq.Codebook4(bq.USER, values)
        width = max(1, -(-max(max(lens), 1) // page)) + 1
        n_pages = len(lens) * width + pad_pages
        table = torch.randperm(n_pages, generator=g)[:len(lens) * width].view(len(lens), width).int()
        codes = [torch.randint(0, 256, (n_pages, kv_heads, page, dim // 2), dtype=torch.uint8, generator=g) for _ in range(2)]
        scales = [torch.full((n_pages, kv_heads, page, dim // block), float("nan"), dtype=torch.bfloat16) for _ in range(2)]
        self.values = []                                             # per sequence (k, v) in float64
        for s, n in enumerate(lens):
            kv = []
            for t, amp in ((0, 1.0), (1, 0.7)):
                x = torch.randn(n, kv_heads, dim, generator=g) * amp * scale
                x[..., dim // 3] *= 5
                if n > 2:
                    x[1] = 0                                         # a row of zeros: scale 0
                packed, sc, vals = ko.store(bits(x.to(tdt)), DT[tdt], block, self.cb_ref)
                for j in range(n):
                    pg, row = int(table[s, j // page]), j % page
                    codes[t][pg, :, row] = torch.from_numpy(packed[j])
                    scales[t][pg, :, row] = torch.from_numpy(sc[j].view(np.int16)).view(torch.bfloat16)
                kv.append(vals)
            self.values.append(kv)
        dev = torch.device("cuda")
        self.pools = [t.to(dev) for t in codes + scales]
        self.cache = bq.KvCache4(*self.pools, table.to(dev), torch.tensor(lens, dtype=torch.int32, device=dev), cb)
        starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.starts_host, self.starts = starts, torch.from_numpy(starts).to(dev)
        self.q = torch.randn(int(starts[-1]), kv_heads * group, dim, generator=g).to(tdt)

    def attend(self, weights=False, path=0, max_new=None, max_len=None, q=None, sm=None):
        dev = self.cache.device
        w = torch.zeros(len(self.lens), self.h, self.cache.capacity, device=dev) if weights else None
        if weights:
            w += 0.25                                                # it is added to
        q = self.q.to(dev) if q is None else q
        out = self.cache.attend(q, self.starts, max(1, max(self.news)) if max_new is None else max_new, max_len=0 if max_len is None else max_len,
                                sm_scale=sm, weights=w, path=path)
        torch.cuda.synchronize()
        assert self.cache.kernel_status() == 0
        return out, w

    def check(self, out, w=None, sm=None, values_11_bits=False):
        sm = 1 / math.sqrt(self.dim) if sm is None else sm
        qd = self.q.double().numpy()
        got = out.double().cpu().numpy()
        for s, (k, v) in enumerate(self.values):
            lo, hi = self.starts_host[s], self.starts_host[s + 1]
            ref = ko.attend(qd[lo:hi], k, v, sm)
            # a codebook whose values take more than 11 bits: each is off by up to 2^-11 in both products
            ds = ((self.dim + 8) * 2.0 ** -22 + (2.0 ** -11 if values_11_bits else 0)) * ref["spread"][..., None]
            extra = 2.0 ** -10 + (2.0 ** -11 if values_11_bits else 0)
            tol = HALF_ULP[self.tdt] * np.abs(ref["out"]) + TINY[self.tdt] + (extra + 2 * ds) * ref["mass"] * (1 + HALF_ULP[self.tdt])
            err = np.abs(got[lo:hi] - ref["out"])
            assert np.all(err <= tol), (s, float(np.nanmax(err / np.maximum(tol, 1e-30))), np.isnan(got[lo:hi]).sum())
            if w is not None:
                n = self.lens[s]
                got_w = w[s].double().cpu().numpy() - 0.25
                wtol = 2 * (self.dim + 8) * 2.0 ** -22 * ref["heavy"] + (2 * (hi - lo) * self.group + 16) * 2.0 ** -23 * (ref["weights"] + 0.25)
                werr = np.abs(got_w[:, :n] - ref["weights"])
                assert np.all(werr <= wtol), (s, float((werr / np.maximum(wtol, 1e-30)).max()))
                assert np.all(got_w[:, n:] == 0)                     # slots past the length are not touched


SHAPES = [                                                           # kv heads, group, dim, block, page
    (2, 4, 128, 128, 64), (2, 1, 128, 64, 16), (1, 8, 64, 64, 32), (3, 7, 64, 32, 16), (2, 2, 128, 32, 128), (1, 16, 128, 64, 64),
    (2, 5, 80, 40, 16), (1, 3, 256, 128, 64), (2, 2, 72, 8, 7), (1, 1, 8, 8, 1), (1, 20, 128, 128, 64)]


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,g,dim,block,page", SHAPES)
@pytest.mark.parametrize("path", [1, 0])
def test_single_tokens(bq, h, g, dim, block, page, tdt, path):
    """One row per sequence: no slots at all, one, lengths on both sides of tiles and pages."""
    lens = [1, 0, 2, 15, 16, 17, 63, 64, 65, 130, 257]
    c = Case(bq, lens, [1] * len(lens), h, g, dim, block, page, tdt, seed=dim + page + g)
    for weights in (False, True):
        c.check(*c.attend(weights, path=path))


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,g,dim,block,page", SHAPES)
@pytest.mark.parametrize("path", [1, 0])
def test_several_rows(bq, h, g, dim, block, page, tdt, path):
    """Ragged rows of a call: none, a few, more than the sequence has slots (the first rows then see nothing)."""
    lens, news = [5, 0, 70, 33, 3, 129], [5, 0, 3, 33, 9, 2]
    c = Case(bq, lens, news, h, g, dim, block, page, tdt, seed=dim + page)
    for weights in (False, True):
        c.check(*c.attend(weights, path=path))


@pytest.mark.parametrize("h,g,dim,block,page,tdt", [(2, 4, 128, 128, 64, torch.bfloat16), (1, 7, 64, 64, 32, torch.float16), (2, 1, 128, 64, 16, torch.float16)])
def test_prompts(bq, h, g, dim, block, page, tdt):
    lens, news = [300, 257, 128, 140], [300, 130, 128, 1]
    c = Case(bq, lens, news, h, g, dim, block, page, tdt, seed=11)
    for weights in (False, True):
        c.check(*c.attend(weights))


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,g,dim,block,page", [s for s in SHAPES if s[2] in (64, 128) and s[3] >= 32])
@pytest.mark.parametrize("path", [2, 3])
def test_every_kernel_takes_every_number_of_rows(bq, h, g, dim, block, page, tdt, path):
    """The kernel for few rows on many (several groups of rows per head) and the one for many on few."""
    for lens, news in (([70, 0, 33, 129, 1], [1, 1, 1, 1, 1]), ([5, 0, 200, 33, 3], [5, 0, 70, 33, 9])):
        c = Case(bq, lens, news, h, g, dim, block, page, tdt, seed=dim + page + path)
        for weights in (False, True):
            c.check(*c.attend(weights, path=path))


def test_store_and_read_are_the_codec(bq):
    """Rows into shuffled pages, from contiguous and from strided and unaligned tensors: every pool byte is the codec's, rows of
    other slots keep what they held, and a read gives the codec's values."""
    for tdt, (h, _, dim, block, page) in [(torch.float16, s) for s in SHAPES] + [(torch.bfloat16, s) for s in SHAPES]:
        lens, news = [9, 40, 0, 3, 17], [9, 5, 0, 0, 2]
        c = Case(bq, lens, news, h, 1, dim, block, page, tdt, seed=3)
        before = [t.clone() for t in c.pools]
        g = torch.Generator().manual_seed(5)
        n = sum(news)
        wide = (torch.randn(n, 3 * h + 1, dim, generator=g) * 2).to(tdt)
        wide[0, 0] = 0
        flat = torch.zeros(n * (3 * h + 1) * dim + 3, dtype=tdt, device="cuda")
        flat[3:] = wide.cuda().reshape(-1)                           # three elements off the alignment
        odd = flat[3:].view(n, 3 * h + 1, dim)
        for src in (wide.cuda(), odd):
            for t, b in zip(c.pools, before):
                t.copy_(b)
            k, v = src[:, :h], src[:, h:2 * h]
            c.cache.append(k, v, c.starts)
            want = [b.clone().cpu() for b in before]
            table = c.cache.table.cpu()
            rows = []
            for x, ci, si in ((wide[:, :h], 0, 2), (wide[:, h:2 * h], 1, 3)):
                packed, sc, vals = ko.store(bits(x), DT[tdt], block, c.cb_ref)
                rows.append(ko.read(vals, DT[tdt]))
                for s in range(len(lens)):
                    for i in range(news[s]):
                        j, r = lens[s] - news[s] + i, int(c.starts_host[s]) + i
                        pg = int(table[s, j // page])
                        want[ci][pg, :, j % page] = torch.from_numpy(packed[r])
                        want[si][pg, :, j % page] = torch.from_numpy(sc[r].view(np.int16)).view(torch.bfloat16)
            for t, b in zip(c.pools, want):
                assert torch.equal(t.cpu().view(torch.uint8), b.view(torch.uint8))
            got = c.cache.read(c.starts, n, tdt)
            for t, b in zip(got, rows):
                assert np.array_equal(bits(t), b)


def test_store_matches_the_tensor_call(bq):
    """A page of one head is the layout of bq4_quantize_s16 on its rows."""
    cb = bq.Codebook4()
    cache = bq.KvCache4.empty(3, 32, 2, 128, 64, cb, page=32)
    x = torch.randn(96, 2, 128, device="cuda").to(torch.bfloat16)
    cache.lens.fill_(32)
    starts = torch.tensor([0, 32, 64, 96], dtype=torch.int32, device="cuda")
    cache.append(x, x * 2, starts)
    rows = x.view(3, 32, 2, 128).transpose(1, 2).contiguous()
    for pool, y in ((0, rows), (1, rows * 2)):
        packed, scale = bq.bq4_quantize_s16(y.reshape(-1), 64, cb)
        assert torch.equal(cache._pools[pool].reshape(-1), packed) and torch.equal(cache._pools[pool + 2].reshape(-1), scale)


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,dim,block,page", [(3, 128, 64, 32), (1, 64, 32, 16), (2, 256, 16, 5), (5, 64, 64, 64), (2, 80, 40, 16)])
def test_many_rows_stored_and_read(bq, h, dim, block, page, tdt):
    """Enough rows for the kernels that take many at once: against the tensor calls on the same rows, slots that do not exist
    among them."""
    cb = bq.Codebook4()
    news = [3000, 1, 0, 2500, 700]
    cache = bq.KvCache4.empty(5, 3000, h, dim, block, cb, page=page)
    cache.lens.copy_(torch.tensor([3000, 1, 7, 2600, 650], dtype=torch.int32))
    starts = torch.from_numpy(np.concatenate([[0], np.cumsum(news)]).astype(np.int32)).cuda()
    x = (torch.randn(sum(news), 2, h, dim, generator=torch.Generator().manual_seed(3)) * 1.5).to(tdt).cuda()
    x[5] = 0
    cache.append(x[:, 0], x[:, 1], starts)
    k, v = cache.read(starts, sum(news), tdt)
    for got, y in ((k, x[:, 0].contiguous()), (v, x[:, 1].contiguous())):
        packed, scale = bq.bq4_quantize_s16(y.reshape(-1), block, cb)
        want = bq.bq4_dequantize_s16(packed, scale, y.numel(), block, cb, tdt).view_as(y)
        want[5501:5551] = 0                                          # the last sequence has 700 rows for 650 slots
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def test_rows_past_the_table_are_dropped(bq):
    cb = bq.Codebook4()
    cache = bq.KvCache4.empty(2, 16, 1, 64, 64, cb, page=16)
    cache.lens.copy_(torch.tensor([19, 2]))
    x = torch.randn(8, 1, 64, device="cuda").to(torch.float16)
    before = [p.clone() for p in cache._pools]
    cache.append(x, x, torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"))      # lens is clamped to 16; 4 rows for 2 slots
    k, _ = cache.read(torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"), 8, torch.float16)
    assert torch.all(k[4:6] == 0) and torch.any(k[:4] != 0) and torch.any(k[6:] != 0)
    assert torch.equal(cache._pools[0][0, :, :12], before[0][0, :, :12]) and torch.equal(cache._pools[0][1, :, 2:], before[0][1, :, 2:])


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("path", [0, 2, 3])
@pytest.mark.parametrize("h,g,dim,block,page", [(2, 4, 128, 128, 64), (1, 3, 128, 32, 48), (2, 2, 64, 64, 16), (1, 5, 64, 32, 32)])
def test_rows_on_both_sides_of_a_pass(bq, h, g, dim, block, page, path, tdt):
    """Numbers of query rows around 16, 128 and 256, where a kernel's passes, row tiles and blocks end; one sequence with none."""
    for rows in (15, 17, 127, 129, 255, 257):
        news = [-(-rows // g), 0, rows // g]
        c = Case(bq, [n + 90 for n in news], news, h, g, dim, block, page, tdt, seed=rows + path)
        c.check(*c.attend(path=path))


@pytest.mark.parametrize("h,g,dim,block,page", [(2, 2, 80, 40, 16), (1, 3, 256, 128, 64), (1, 1, 8, 8, 1), (1, 2, 128, 128, 64)])
@pytest.mark.parametrize("weights", [False, True])
def test_general_kernel_over_long_contexts(bq, h, g, dim, block, page, weights):
    """Few rows: their slots are shared by several CTAs, some of which have none (short sequences, an empty one)."""
    lens = [1, 255, 256, 257, 0, 1500, 700]
    c = Case(bq, lens, [1, 1, 1, 2, 0, 1, 3], h, g, dim, block, page, torch.float16, seed=dim)
    c.check(*c.attend(weights, path=1))


@pytest.mark.parametrize("path,dim,block", [(1, 80, 40), (1, 128, 128), (2, 128, 64), (3, 128, 64), (3, 64, 64)])
def test_nan_stays_in_its_row(bq, path, dim, block):
    lens, news = [900, 70, 3], [2, 3, 3]
    c = Case(bq, lens, news, 2, 2, dim, block, 16, torch.bfloat16, seed=3)
    q = c.q.to(c.cache.device)
    good = c.cache.attend(q, c.starts, 3, path=path)
    bad = q.clone()
    bad[1, 2, 5] = float("nan")
    got = c.cache.attend(bad, c.starts, 3, path=path)
    assert bool(torch.isnan(got[1, 2]).all())
    keep = torch.ones(got.shape[:2], dtype=torch.bool)
    keep[1, 2] = False
    assert torch.equal(got[keep.to(got.device)], good[keep.to(got.device)])


@pytest.mark.parametrize("path", [1, 0])
def test_bounds_are_hints(bq, path):
    """max_new and max_len size the launch; smaller than the truth they still give right results."""
    c = Case(bq, [200, 9, 64], [40, 3, 1], 2, 4, 128, 128, 16, torch.bfloat16)
    out, w = c.attend(True, path=path, max_new=1, max_len=8)
    c.check(out, w)


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 60.0, 1e4])
def test_magnitudes(bq, scale):
    """Keys and values far below and above one (fp16 and bf16 ranges), scores kept in range by sm_scale."""
    tdt = torch.bfloat16 if scale in (1e-6, 1e4) else torch.float16
    for news in ([1, 1], [40, 40]):
        c = Case(bq, [150, 77], news, 2, 4, 128, 64, 16, tdt, scale=scale)
        sm = 1 / (math.sqrt(128) * scale)
        c.check(*c.attend(True, sm=sm), sm=sm)


@pytest.mark.parametrize("new", [1, 40])
def test_wide_range_of_value_scales(bq, new):
    """A sequence whose values grow by 2^20 along it, the large ones behind small probabilities and the other way round."""
    for flip in (False, True):
        c = Case(bq, [256], [new], 1, 4, 128, 128, 16, torch.bfloat16)
        k, v = c.values[0]
        f = 2.0 ** np.round(np.linspace(-10, 10, 256))
        f = f[::-1] if flip else f
        v *= f[:, None, None]
        sc = c.pools[3]
        table = c.cache.table.cpu()
        for j in range(256):
            sc[int(table[0, j // 16]), :, j % 16] *= float(f[j])
        out, _ = c.attend(False)
        # scaled values of one tile share a power of two: rounding to 11 bits of the tile's largest, not of each value's own
        c.check(out)


@pytest.mark.parametrize("regular", [True, False])
def test_user_codebooks(bq, regular):
    """A linear map (multiples of 1 / 8) and an irregular one whose values are rounded to 11 bits in the products."""
    values = [i / 8 for i in range(-8, 8)] if regular else [-1, -0.6961928, -0.5250731, -0.3949175, -0.2844414, -0.1847734, -0.0910500, 0, 0.0795803, 0.1609302,
                                                            0.2461123, 0.3379152, 0.4407098, 0.5626170, 0.7229568, 1.0]
    for news in ([1, 1], [40, 30]):
        c = Case(bq, [100, 61], news, 2, 4, 128, 64, 16, torch.float16, values=values)
        out, _ = c.attend(False, sm=0.02)
        c.check(out, sm=0.02, values_11_bits=not regular)


def test_strided_queries_other_streams_and_repeats(bq):
    c = Case(bq, [300, 31], [1, 1], 2, 4, 128, 128, 64, torch.float16)
    ref, w = c.attend(True)
    wide = torch.randn(2, 24, 128).to(torch.float16)
    wide[:, 4:12] = c.q
    out, _ = c.attend(False, q=wide.cuda()[:, 4:12])
    assert torch.equal(out, ref)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(5):
            out2, w2 = c.attend(True)
            assert torch.equal(out2, ref) and torch.equal(w2, w)     # the same bits every time


def test_graph_capture(bq):
    """A decode step captured once and replayed as lens grows on the device."""
    c = Case(bq, [60, 61], [1, 1], 2, 4, 64, 64, 16, torch.float16)
    q = c.q.cuda()
    c.cache.lens.copy_(torch.tensor([10, 20]))
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out = torch.empty_like(q)
        for _ in range(2):
            c.cache.attend(q, None, max_len=80, out=out)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.cache.attend(q, None, max_len=80, out=out)
    c.cache.lens.copy_(torch.tensor([60, 61]))
    graph.replay()
    torch.cuda.synchronize()
    c.check(out)


@pytest.mark.parametrize("budget,sinks,recent", [(16, 2, 4), (1, 0, 0), (5, 0, 5), (5, 5, 0), (40, 4, 8), (64, 0, 0), (200, 10, 30), (259, 3, 256), (300, 1, 2)])
@pytest.mark.parametrize("h,dim,block,page", [(2, 128, 64, 16), (3, 80, 40, 7), (1, 256, 8, 64)])
def test_evict(bq, budget, sinks, recent, h, dim, block, page):
    lens = [300, 40, 0, 260, 17, 5, 261]
    c = Case(bq, lens, [1] * len(lens), h, 1, dim, block, page, torch.bfloat16, seed=budget)
    g = torch.Generator().manual_seed(budget)
    w = torch.rand(len(lens), h, c.cache.capacity, generator=g) ** 4
    w[0, :, ::3] = 0.125                                             # ties
    w[3] = (w[3] * 4).floor() / 4
    w[6, 0, 7] = float("nan")
    w[6, 0, 9] = float("inf")
    w[6, 0, 11] = -1.0
    w[5] = 0
    wd = w.cuda()
    c.cache.evict(wd, budget, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    new = [min(n, budget) for n in lens]
    assert c.cache.lens.cpu().tolist() == new
    want_w = w.clone()
    ks, vs = c.cache.read(torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda(), sum(new), torch.float16)
    at = 0
    for s, n in enumerate(lens):
        for j in range(h):
            place = ko.evict_places(w[s, j].numpy(), n, budget, sinks, recent)
            if n > budget:
                want_w[s, j, :budget] = w[s, j, torch.from_numpy(place)]
            for t, vals in ((ks, c.values[s][0]), (vs, c.values[s][1])):
                assert np.array_equal(bits(t[at:at + new[s], j]), ko.read(vals[place, j], o4.F16)), (s, j)
        at += new[s]
    assert torch.equal(wd.cpu().view(torch.int32), want_w.view(torch.int32))


def test_evict_long(bq):
    """Longer than a CTA's passes, many ties, heads that differ; attention afterwards reads the kept rows."""
    n, budget = 5000, 1500
    c = Case(bq, [n], [1], 2, 4, 64, 64, 64, torch.float16, seed=1)
    out, w = c.attend(True)
    c.check(out, w)
    host = w.cpu()
    c.cache.evict(w, budget, sinks=4, recent=100)
    places = [ko.evict_places(host[0, j].numpy(), n, budget, 4, 100) for j in range(2)]
    c.values = [[np.stack([t[places[j], j] for j in range(2)], 1) for t in c.values[0]]]
    c.lens = [budget]
    assert c.cache.lens.tolist() == [budget]
    out, _ = c.attend(False)
    c.check(out)


def test_refusals(bq):
    cb = bq.Codebook4()
    cache = bq.KvCache4.empty(2, 64, 2, 128, 64, cb, page=16)
    q = torch.zeros(2, 4, 128, dtype=torch.float16, device="cuda")
    kv = torch.zeros(2, 2, 128, dtype=torch.float16, device="cuda")
    w = torch.zeros(2, 2, 64, device="cuda")
    for bad in (lambda: cache.attend(q.float()), lambda: cache.attend(q[:, :3]), lambda: cache.attend(q[..., :64]), lambda: cache.attend(q[:1]),
                lambda: cache.attend(q.transpose(0, 1)), lambda: cache.attend(q, out=torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda")),
                lambda: cache.attend(q, weights=w[:1]), lambda: cache.attend(q, weights=w.half()), lambda: cache.attend(q, path=99),
                lambda: cache.attend(q, sm_scale=float("nan")), lambda: cache.attend(q, max_new=-1), lambda: cache.attend(q.cpu()),
                lambda: cache.attend(q, torch.zeros(3, dtype=torch.int64, device="cuda")), lambda: cache.attend(q, torch.zeros(2, dtype=torch.int32, device="cuda")),
                lambda: cache.append(kv, kv[:1]), lambda: cache.append(kv, kv.bfloat16()), lambda: cache.append(kv.float(), kv.float()),
                lambda: cache.append(kv[:, :1], kv[:, :1]), lambda: cache.read(None, 1, torch.float16), lambda: cache.read(None, 2, torch.float32),
                lambda: cache.evict(w, 0), lambda: cache.evict(w, 8, sinks=5, recent=4), lambda: cache.evict(w, 8, sinks=-1), lambda: cache.evict(None, 8),
                lambda: bq.KvCache4(*cache._pools, cache.table.long(), cache.lens, cb), lambda: bq.KvCache4(*cache._pools, cache.table, cache.lens[:1], cb),
                lambda: bq.KvCache4(cache._pools[0], cache._pools[1], cache._pools[2].float(), cache._pools[3], cache.table, cache.lens, cb)):
        with pytest.raises(BqError):
            bad()
    assert cache.attend(q[:0], torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 4, 128)      # no rows: nothing to do
    torch.cuda.synchronize()
