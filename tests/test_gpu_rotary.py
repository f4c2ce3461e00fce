"""GPU tests of the store with positions (bqkv_append_rotary of include/bq4.h) against the oracle.

Keys are exact: the oracle's turn in extended precision, rounded to fp32, through the codec's oracle, bit for bit; so are values.
Queries are turned in fp32 and rounded once:

    tol = ulp/2 of the type at |y| + 4 2^-24 (|u| + |v|)

ulp/2: the rounding to the type; the rest: cos and sin rounded to fp32 (2^-24 of each product), two products' roundings and the sum's.
"""
import numpy as np
import pytest
import torch

from oracle import bq4_oracle as o4
from oracle import rotary_oracle as ro
from paper_2407_19775_b200.binding import BqError
from test_gpu_kvcache import DT, HALF_ULP, TINY, bits

pytestmark = pytest.mark.gpu
U8 = 0xA5


class Store:
    """An empty cache (every byte U8) with shuffled pages, and the projection whose slices a call takes."""

    def __init__(self, bq, lens, news, kv_heads, q_heads, dim, block, page, tdt, seed=0, behind=0, odd=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.news, self.h, self.hq, self.dim, self.block, self.page, self.tdt = lens, news, kv_heads, q_heads, dim, block, page, tdt
        width = max(1, -(-max(max(lens), 1) // page))
        self.n_pages = len(lens) * width + 1
        self.table = torch.randperm(self.n_pages, generator=g)[:len(lens) * width].view(len(lens), width).int()
        dev = torch.device("cuda")
        self.pools = [torch.full((self.n_pages, kv_heads, page, dim // 2), U8, dtype=torch.uint8, device=dev) for _ in range(2)]
        self.pools += [torch.full((self.n_pages, kv_heads, page, dim // block * 2), U8, dtype=torch.uint8, device=dev).view(torch.bfloat16) for _ in range(2)]
        self.cache = bq.KvCache4(*self.pools, self.table.to(dev), torch.tensor(lens, dtype=torch.int32, device=dev), bq.Codebook4())
        starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.rows = int(starts[-1]) + behind
        self.starts = torch.from_numpy(starts).to(dev)
        x = torch.randn(self.rows, (q_heads + 2 * kv_heads) * dim + odd, generator=g)
        x[:, dim // 3::dim] *= 4
        x[self.rows // 2] = 0                                        # a row of zeros: scale 0
        self.qkv = x.to(tdt).to(dev)

    def slices(self):
        heads = self.qkv[:, self.qkv.shape[1] - (self.hq + 2 * self.h) * self.dim:].unflatten(1, (-1, self.dim))
        return heads.split((self.hq, self.h, self.h), dim=1)

    def places(self):
        """Sequence and place of every row; sequence -1 for rows behind the last start."""
        at = [(s, n - m + i) for s, (n, m) in enumerate(zip(self.lens, self.news)) for i in range(m)]
        return at + [(-1, 0)] * (self.rows - len(at))

    def check(self, q_out, rot, positions=None, q0=None, untouched=None):
        at = self.places()
        q, k, v = (t.double().cpu().numpy() for t in self.slices())
        q = q if q0 is None else q0
        pos = np.array([[p for _, p in at]] * rot.axes) if positions is None else positions.cpu().numpy().reshape(rot.axes, -1)
        of = rot.of_pair if hasattr(rot, "of_pair") else np.zeros(rot.dim // 2, int)
        own = [r for r, (s, _) in enumerate(at) if s >= 0]
        if q_out is not None:
            ref = ro.turn(q, pos, rot.frequencies, of, rot.interleaved)
            mag = np.abs(q).copy()
            for i in range(rot.dim // 2):
                a, b = (2 * i, 2 * i + 1) if rot.interleaved else (i, i + rot.dim // 2)
                mag[..., a] = mag[..., b] = np.abs(q[..., a]) + np.abs(q[..., b])
            tol = HALF_ULP[self.tdt] * np.abs(ref) * (1 + 2.0 ** -20) + TINY[self.tdt] + 4 * 2.0 ** -24 * mag
            got = q_out.double().cpu().numpy()
            assert np.all(np.abs(got - ref)[own] <= tol[own]), float(np.max((np.abs(got - ref) / np.maximum(tol, 1e-30))[own]))
            assert np.array_equal(got[own][..., rot.dim:], q[own][..., rot.dim:])
            if untouched is not None:
                rest = [r for r in range(self.rows) if r not in own]
                assert torch.equal(q_out[rest], untouched[rest])
        k32 = ro.turn(k, pos, rot.frequencies, of, rot.interleaved).astype(np.float32)
        want = [np.full((self.n_pages, self.h, self.page, self.dim // 2), U8, np.uint8) for _ in range(2)]
        want += [np.full((self.n_pages, self.h, self.page, self.dim // self.block), U8 * 257, np.uint16) for _ in range(2)]
        cb = o4.make_codebook()
        cap = self.table.shape[1] * self.page
        for r, (s, p) in enumerate(at):
            if s < 0 or p < 0 or p >= cap:
                continue
            pg = int(self.table[s, p // self.page])
            for t, x in ((0, k32[r]), (1, v[r].astype(np.float32))):
                codes, scale = o4.quantize_s16(np.ascontiguousarray(x).reshape(-1), o4.F32, self.block, cb)
                want[t][pg, :, p % self.page] = codes.reshape(self.h, -1)
                want[2 + t][pg, :, p % self.page] = scale.reshape(self.h, -1)
        for t in range(4):
            got = self.pools[t].cpu()
            got = got.numpy() if t < 2 else got.view(torch.int16).numpy().view(np.uint16)
            assert np.array_equal(got, want[t]), (t, int((got != want[t]).sum()), got.size)


def rotary(bq, dim, **kw):
    r = bq.Rotary(dim, **kw)
    if kw.get("sections"):
        r.of_pair = np.repeat(np.arange(len(kw["sections"])), kw["sections"])
    elif kw.get("axes"):
        r.of_pair = np.array(kw["axes"])
    return r


SHAPES = [                                                           # kv heads, query heads, dim, block, page, turned
    (2, 8, 128, 128, 64, 128), (1, 1, 128, 64, 16, 128), (8, 8, 128, 32, 64, 128), (3, 21, 64, 32, 16, 64), (1, 8, 64, 64, 32, 64), (2, 2, 64, 8, 16, 64),
    (5, 15, 128, 16, 7, 128), (2, 10, 80, 40, 16, 80), (2, 4, 128, 64, 64, 64), (1, 3, 256, 128, 64, 256), (2, 2, 72, 8, 7, 36), (1, 1, 8, 8, 1, 2)]


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,hq,dim,block,page,turned", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_single_tokens_at_far_positions(bq, h, hq, dim, block, page, turned, interleaved, tdt):
    lens = [1, 0, 2, 17, 33, 64, 5]
    c = Store(bq, lens, [1] * len(lens), h, hq, dim, block, page, tdt, seed=dim + page)
    rot = rotary(bq, turned, interleaved=interleaved)
    pos = torch.tensor([0, 5, 1000003, -77, 2 ** 31 - 1, -2 ** 31, 131071], dtype=torch.int32, device="cuda")
    q, k, v = c.slices()
    c.check(c.cache.append_rotary(q, k, v, rot, pos), rot, pos)


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,hq,dim,block,page,turned", SHAPES)
def test_ragged_rows_take_their_places(bq, h, hq, dim, block, page, turned, tdt):
    """No positions: the places.  Sequences without rows, more rows than slots, rows behind the last start."""
    lens, news = [5, 0, 70, 3, 130, 0], [5, 0, 3, 9, 66, 2]
    c = Store(bq, lens, news, h, hq, dim, block, page, tdt, seed=dim + page, behind=3)
    rot = rotary(bq, turned, base=500.0)
    q, k, v = c.slices()
    out = torch.full_like(q, 7.0, memory_format=torch.contiguous_format)
    c.check(c.cache.append_rotary(q, k, v, rot, None, c.starts, out), rot, untouched=torch.full_like(out, 7.0))


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("h,hq,dim,block,page,sections,interleaved", [
    (2, 6, 128, 64, 64, [16, 24, 24], False), (4, 28, 128, 128, 32, [22, 21, 21], True), (2, 4, 64, 32, 16, [0, 32], False), (1, 2, 80, 40, 16, [10, 15, 15], False)])
def test_several_axes(bq, h, hq, dim, block, page, sections, interleaved, tdt):
    lens, news = [100, 40], [60, 40]
    c = Store(bq, lens, news, h, hq, dim, block, page, tdt, seed=3)
    rot = rotary(bq, dim, sections=sections, interleaved=interleaved)
    wide = torch.randint(-5, 4000, (len(sections), 140), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    pos = wide[:, 20:120]                                            # axes further apart than the rows
    q, k, v = c.slices()
    c.check(c.cache.append_rotary(q, k, v, rot, pos, c.starts), rot, pos.contiguous())


def test_axes_in_any_order_and_many_rows(bq):
    lens = news = [1500, 801, 2048, 1]
    c = Store(bq, lens, news, 2, 6, 128, 64, 64, torch.bfloat16, seed=5)
    rot = rotary(bq, 128, axes=[i % 3 for i in range(64)])
    pos = torch.randint(0, 3000, (3, c.rows), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    q, k, v = c.slices()
    c.check(c.cache.append_rotary(q, k, v, rot, pos, c.starts), rot, pos)


@pytest.mark.parametrize("news", [[1, 1, 1], [40, 1, 700]])
@pytest.mark.parametrize("h,hq,dim,block,turned", [(2, 8, 128, 64, 128), (2, 8, 128, 64, 96), (2, 6, 64, 64, 64), (1, 2, 80, 40, 80)])
def test_in_place_and_at_any_alignment(bq, h, hq, dim, block, turned, news):
    """q_out is q inside the projection; odd row pitches and element offsets; keys and values as they were."""
    for odd in (0, 1, 2, 8):
        c = Store(bq, news, news, h, hq, dim, block, 16, torch.float16, seed=odd, odd=odd)
        rot = rotary(bq, turned)
        q, k, v = c.slices()
        q0, kv = q.double().cpu().numpy(), c.qkv.clone()
        got = c.cache.append_rotary(q, k, v, rot, None, c.starts, q)
        assert got is q
        c.check(got, rot, q0=q0)
        assert torch.equal(c.qkv[:, odd + hq * dim:], kv[:, odd + hq * dim:]) and torch.equal(c.qkv[:, :odd], kv[:, :odd])


def test_without_queries_and_user_frequencies(bq):
    c = Store(bq, [9, 40], [9, 2], 2, 4, 128, 64, 16, torch.bfloat16)
    f = np.concatenate([[0.0, 2 * np.pi, np.pi / 2, -0.75, 65536.0, 1e-9], np.geomspace(3.0, 1e-7, 58)])
    rot = rotary(bq, 128, frequencies=f)
    _, k, v = c.slices()
    assert c.cache.append_rotary(None, k, v, rot, None, c.starts) is None
    c.check(None, rot)


def test_position_zero_is_append_and_turns_add_up(bq):
    """Zero angles store what append stores and hand queries back; scores go by the difference of positions."""
    c = Store(bq, [30], [30], 2, 4, 128, 64, 16, torch.float16)
    q, k, v = c.slices()
    zero = torch.zeros(30, dtype=torch.int32, device="cuda")
    out = c.cache.append_rotary(q, k, v, bq.Rotary(128), zero, c.starts)
    first = [p.clone() for p in c.pools]
    c.cache.append(k, v, c.starts)
    assert torch.equal(out, q) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(first, c.pools))


def test_captured_and_on_another_stream(bq):
    c = Store(bq, [40, 7], [1, 1], 2, 8, 128, 64, 16, torch.bfloat16)
    rot = bq.Rotary(128)
    pos = torch.tensor([3, 9], dtype=torch.int32, device="cuda")
    q, k, v = c.slices()
    out = torch.zeros_like(q, memory_format=torch.contiguous_format)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.cache.append_rotary(q, k, v, rot, pos, None, out)
    torch.cuda.synchronize()
    c.check(out, rot, pos)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.append_rotary(q, k, v, rot, pos, None, out)
    pos += 12345                                                     # the next step's
    graph.replay()
    torch.cuda.synchronize()
    c.check(out, rot, pos)


def test_refusals(bq):
    c = Store(bq, [4, 4], [1, 1], 2, 4, 128, 64, 16, torch.float16)
    rot, rot3 = bq.Rotary(128), bq.Rotary(128, sections=[16, 24, 24])
    q, k, v = c.slices()
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    call = c.cache.append_rotary
    for bad in (dict(q=q.bfloat16()), dict(k=k[:1]), dict(v=v[:, :1]), dict(q=q[:1]), dict(positions=pos.long()), dict(positions=pos.cpu()), dict(positions=pos[:1]),
                dict(rotary=rot3, positions=pos), dict(rotary=rot3, positions=torch.zeros(3, 2, dtype=torch.int32, device="cuda").t().contiguous().t()),
                dict(rotary=rot3, positions=pos.expand(3, 2)), dict(q=None, q_out=torch.empty_like(q)), dict(q_out=torch.empty_like(q[:, :2])),
                dict(q_out=torch.empty_like(q.float())), dict(q=q.cpu()), dict(starts=c.starts.long()), dict(rotary=bq.Rotary(256)), dict(q_out=c.qkv[:, 128:640].unflatten(1, (4, 128)))):
        with pytest.raises(BqError):
            call(**{**dict(q=q, k=k, v=v, rotary=rot, positions=pos, starts=c.starts), **bad})
    assert all(bool((p.view(torch.uint8) == U8).all()) for p in c.pools)
