"""GPU tests of the 4-bit cache at the edges of its limits: sequences counted past their table, values of very
different sizes, light tokens, launches sized too small, many sequences, long evictions; against the same plain
implementations and within the same bounds as tests/test_gpu_kvcache.py."""
import numpy as np
import pytest
import torch

from oracle import kvcache_oracle as ko
from paper_2407_19775_b200.binding import BqError
from test_gpu_kvcache import DT, HALF_ULP, TINY, Case, bits

pytestmark = pytest.mark.gpu


def check_rows(c, out, w, seen, sm, floor=0.0):
    """Case.check with the slots that each row sees given: seen[s][i].  floor: the smallest step of what enters the second product,
    half of it, relative to the row's largest product of probability and value scale; each slot adds that much error at most, times
    a code's value (1 at most).  The largest product is at most 1.13 times the largest column's sum of p |v|: a scale is the block's
    largest magnitude or up to 2^-7 more, and the code of that element is worth 1, or -0.8875 where it is negative."""
    got, qd = out.double().cpu().numpy(), c.q.double().numpy()
    for s, (k, v) in enumerate(c.values):
        lo, hi = c.starts_host[s], c.starts_host[s + 1]
        weights, heavy = np.zeros((c.h, len(k))), np.zeros((c.h, len(k)))
        for i in range(hi - lo):
            n = seen[s][i]
            ref = ko.attend(qd[lo + i:lo + i + 1], k[:n], v[:n], sm)
            ds = (c.dim + 8) * 2.0 ** -22 * ref["spread"][..., None]
            tol = HALF_ULP[c.tdt] * np.abs(ref["out"]) + TINY[c.tdt] + (2.0 ** -10 + 2 * ds) * ref["mass"] * (1 + HALF_ULP[c.tdt])
            tol += floor * n * 1.13 * ref["mass"].max(-1, keepdims=True)
            assert np.all(np.abs(got[lo + i:lo + i + 1] - ref["out"]) <= tol), (s, i)
            weights[:, :n] += ref["weights"]
            heavy[:, :n] += ref["heavy"]
        if w is not None:
            wtol = 2 * (c.dim + 8) * 2.0 ** -22 * heavy + (2 * (hi - lo) * c.group + 16) * 2.0 ** -23 * (weights + 0.25)
            held = w[s].double().cpu().numpy() - 0.25
            assert np.all(np.abs(held[:, :len(k)] - weights) <= wtol) and np.all(held[:, len(k):] == 0), s


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("many", [False, True])
def test_rows_past_the_table_leave_the_others_alone(bq, tdt, many):
    """15 slots held of 16 and four new rows: the first has slot 15, the others none.  The rows before keep every byte."""
    cb = bq.Codebook4()
    seqs = 1500 if many else 2                                       # many: the kernels for thousands of rows
    cache = bq.KvCache4.empty(seqs, 16, 1, 64, 64, cb, page=16)
    g = torch.Generator().manual_seed(1)
    old = torch.randn(seqs * 15, 2, 1, 64, generator=g).to(tdt).cuda()
    cache.lens.fill_(15)
    cache.append(old[:, 0], old[:, 1], torch.arange(0, 15 * seqs + 1, 15, dtype=torch.int32, device="cuda"))
    before = [p.clone() for p in cache._pools]
    new = torch.randn(seqs * 4, 2, 1, 64, generator=g).to(tdt).cuda()
    starts = torch.arange(0, 4 * seqs + 1, 4, dtype=torch.int32, device="cuda")
    cache.lens.fill_(19)
    cache.append(new[:, 0], new[:, 1], starts)
    for t, pool in enumerate(cache._pools):
        assert torch.equal(pool[:, :, :15].view(torch.uint8), before[t][:, :, :15].view(torch.uint8))
    for t in range(2):
        packed, scale = bq.bq4_quantize_s16(new[::4, t].reshape(-1), 64, cb)
        assert torch.equal(cache._pools[t][:, 0, 15].reshape(-1), packed) and torch.equal(cache._pools[2 + t][:, 0, 15].reshape(-1), scale)
    for t, got in enumerate(cache.read(starts, 4 * seqs, tdt)):
        packed, scale = bq.bq4_quantize_s16(new[::4, t].reshape(-1), 64, cb)
        want = torch.zeros(seqs, 4, 64, dtype=tdt, device="cuda")
        want[:, 0] = bq.bq4_dequantize_s16(packed, scale, seqs * 64, 64, cb, tdt).view(seqs, 64)
        assert torch.equal(got.view(seqs, 4, 64), want)
    cache.lens.fill_(40)                                             # and far past it: nothing at all is written
    before = [p.clone() for p in cache._pools]
    cache.append(new[:, 0], new[:, 1], starts)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache._pools, before))


@pytest.mark.parametrize("path,dim,block", [(1, 80, 40), (1, 128, 128), (2, 128, 64), (2, 64, 64), (3, 128, 64), (3, 64, 32)])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_of_rows_past_the_table(bq, path, dim, block, weights):
    """A row sees the slots up to its own place, and all that are held where its place lies past the end."""
    page, lens, news = 16, [32, 32, 20, 32], [40, 3, 5, 6]
    c = Case(bq, lens, news, 2, 3, dim, block, page, torch.bfloat16, seed=dim + path)
    c.cache = bq.KvCache4(*c.pools, c.cache.table[:, :2].contiguous(), c.cache.lens, c.cache.codebook)      # 32 slots and no more
    counted = [45, 33, 20, 100]
    c.cache.lens.copy_(torch.tensor(counted))
    seen = [[max(0, min(counted[s] - news[s] + i + 1, 32)) for i in range(news[s])] for s in range(4)]
    sm = dim ** -0.5
    out, w = c.attend(weights, path=path, sm=sm)
    check_rows(c, out, w, seen, sm)


def test_rows_behind_the_last_start_have_no_slot(bq):
    """starts that end before the rows do (they should not): the rows behind belong to no sequence, so nothing is stored for them."""
    cb = bq.Codebook4()
    cache = bq.KvCache4.empty(2, 32, 1, 64, 64, cb, page=16)
    x = torch.randn(9, 1, 64, device="cuda").to(torch.float16)
    cache.lens.copy_(torch.tensor([2, 3]))
    before = [p.clone() for p in cache._pools]
    starts = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    cache.append(x, x, starts)
    k, v = cache.read(starts, 9, torch.float16)
    assert bool(torch.all(k[5:] == 0)) and bool(torch.all(v[5:] == 0)) and bool(torch.all(k[:5].abs().amax((1, 2)) > 0))
    for a, b in zip(cache._pools, before):                           # sequences have two pages each: rows 0 .. 2 of pages 0 and 2
        assert torch.equal(a[::2, :, 3:].view(torch.uint8), b[::2, :, 3:].view(torch.uint8)) and torch.equal(a[1::2].view(torch.uint8), b[1::2].view(torch.uint8))
    out = cache.attend(x, starts, 3, path=1)
    assert bool(torch.all(out[5:] == 0)) and bool(torch.isfinite(out[:5]).all())


@pytest.mark.parametrize("n,budget,sinks,recent", [(41500, 1000, 4, 100), (41500, 41400, 0, 300), (45003, 20000, 7, 0), (45003, 3, 1, 1), (40961, 1, 0, 0)])
def test_evict_from_more_slots_than_shared_memory_has_keys_for(bq, n, budget, sinks, recent):
    """Around and beyond the 40960 keys that a CTA keeps: every byte of every slot, and the weights, against the plain form."""
    h, page = 2, 64
    g = torch.Generator().manual_seed(n + budget)
    cache = bq.KvCache4.empty(2, n, h, 64, 64, bq.Codebook4(), page=page)
    for p in cache._pools:
        p.view(torch.uint8).copy_(torch.randint(0, 255, p.view(torch.uint8).shape, generator=g, dtype=torch.uint8))
    cache.table.copy_(torch.randperm(cache.table.numel(), generator=g).view_as(cache.table))
    lens = [n, n - 700]                                              # the second on the other side of the limit, in most cases
    cache.lens.copy_(torch.tensor(lens))
    w = torch.rand(2, h, cache.capacity, generator=g) ** 3
    w[:, 1] = (w[:, 1] * 50).floor() / 50                            # few values, many ties
    flat = lambda pool: pool.view(torch.uint8)[cache.table.long()].transpose(2, 3).reshape(2, -1, h, pool.view(torch.uint8).shape[-1]).cpu()      # noqa: E731
    before = [flat(p) for p in cache._pools]                         # [sequence, slot, head, bytes]
    wd = w.cuda()
    cache.evict(wd, budget, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    after, got_w = [flat(p) for p in cache._pools], wd.cpu()
    assert cache.lens.tolist() == [min(k, budget) for k in lens]
    for s, length in enumerate(lens):
        for j in range(h):
            place = torch.from_numpy(ko.evict_places(w[s, j].numpy(), length, budget, sinks, recent))
            m = len(place)
            for a, b in zip(after, before):
                assert torch.equal(a[s, :m, j], b[s, place, j]) and torch.equal(a[s, m:, j], b[s, m:, j])
            assert torch.equal(got_w[s, j, :m], w[s, j, place]) and torch.equal(got_w[s, j, m:], w[s, j, m:])


# fp16's step below its normal numbers is 2^-24; the largest product is 2^7 or more in the kernel of path 2, 2^10 or more in that of
# path 3, and path 1 has fp32
FLOOR = {1: 0.0, 2: 2.0 ** -32, 3: 2.0 ** -35}


def scale_values(c, s, slots, f):
    """Multiplies the stored values of slots of sequence s by a power of two (through their scales)."""
    table, page = c.cache.table.cpu(), c.cache.page
    c.values[s][1][slots] *= f
    for j in slots:
        c.pools[3][int(table[s, j // page]), :, j % page] *= f


@pytest.mark.parametrize("path,dim,block", [(1, 80, 40), (2, 128, 128), (2, 128, 64), (2, 64, 32), (3, 128, 128), (3, 128, 64), (3, 128, 32), (3, 64, 64), (3, 64, 32)])
@pytest.mark.parametrize("f", [2.0 ** 30, 2.0 ** 80, 2.0 ** -80])
def test_a_row_does_not_depend_on_values_it_cannot_see(bq, path, dim, block, f):
    """One slot's values are far larger (or all others far smaller) than the rest: rows before it, in the same tile, hide it."""
    lens, news = [100, 200], [60, 150]
    c = Case(bq, lens, news, 2, 2, dim, block, 16, torch.bfloat16, seed=dim + block)
    want, _ = c.attend(False, path=path)
    at = (70, 101)
    for s in range(2):
        scale_values(c, s, [at[s]], f) if f > 1 else scale_values(c, s, [j for j in range(lens[s]) if j != at[s]], f)
    seen = [[lens[s] - news[s] + i + 1 for i in range(news[s])] for s in range(2)]
    check_rows(c, *c.attend(True, path=path), seen, dim ** -0.5, FLOOR[path])
    for s in range(2):                                               # the rows before it: as without it, but for the power of two
        lo, first = int(c.starts_host[s]), lens[s] - news[s]
        n = at[s] - first
        got = c.attend(False, path=path)[0][lo:lo + n].double().cpu()
        ref = want[lo:lo + n].double().cpu() * (1.0 if f > 1 else f)
        assert bool(((got - ref).abs() <= 2.0 ** -7 * ref.abs() + 2.0 ** -9 * ref.abs().max()).all()), s


@pytest.mark.parametrize("path,dim,block", [(1, 80, 40), (2, 128, 128), (2, 128, 64), (3, 128, 128), (3, 128, 64), (3, 64, 32)])
@pytest.mark.parametrize("new", [1, 40])
def test_large_values_of_no_weight_leave_the_others_their_bits(bq, path, dim, block, new):
    """A slot whose values are 2^50 times the others' and whose score is 100 and more below theirs."""
    c = Case(bq, [130], [new], 2, 2, dim, block, 16, torch.bfloat16, seed=dim)
    c.q = c.q.abs()
    j, table = 75, c.cache.table.cpu()
    pg, row = int(table[0, j // 16]), j % 16
    c.pools[0][pg, :, row] = 0                                       # the lowest code, times 12: far from every query
    c.pools[2][pg, :, row] = 12.0
    c.values[0][0][j] = float(c.cb_ref[0]) * 12.0
    scale_values(c, 0, [j], 2.0 ** 50)
    c.check(*c.attend(True, path=path))


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("path,dim,block", [(1, 80, 40), (2, 128, 128), (2, 128, 64), (2, 64, 32), (3, 128, 128), (3, 64, 32)])
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("seqs,n", [(1, 131072), (1776, 4096)])
def test_many_light_slots_beside_a_heavy_one(bq, path, dim, block, tdt, first, seqs, n):
    """Slots of about 2^-26.5 of the heavy slot's probability each: 0.14 % of the whole if there are 131071, and in all columns but
    one everything there is.  The heavy slot at the start of the context or near its end; one sequence, which is spread over the
    device, or as many as leave a context whole (they read the same pages)."""
    page, nb = 64, dim // block
    cache = bq.KvCache4.empty(1, n, 1, dim, block, bq.Codebook4(), page=page)
    cache = bq.KvCache4(*cache._pools, cache.table.repeat(seqs, 1), torch.full((seqs,), n, dtype=torch.int32, device="cuda"), cache.codebook)
    cb = torch.from_numpy(bq.Codebook4().values.astype(np.float64)).cuda()
    g = torch.Generator().manual_seed(dim)
    heavy = 3 if first else n - 1000
    codes = torch.randint(0, 16, (2, n, dim), generator=g).cuda()
    codes[1].clamp_(min=9)                                           # values of one sign, so that the light slots add up
    scale = torch.full((2, n, nb), 0.02, dtype=torch.bfloat16, device="cuda")
    scale[1] = 1.0
    sm = dim ** -0.5
    codes[0, heavy], codes[1, heavy] = 15, 7                         # 1 and 0
    scale[0, heavy] = 26.5 * np.log(2) / (sm * dim)
    codes[1, heavy, 5] = 15
    for t in range(2):
        cache._pools[t].view(n, dim // 2).copy_((codes[t, :, 0::2] | codes[t, :, 1::2] << 4).to(torch.uint8))
        cache._pools[2 + t].view(n, nb).copy_(scale[t])
    q = torch.ones(1, 2, dim, dtype=tdt, device="cuda")
    q[0, 1] = 0.875
    k, v = (cb[codes[t]] * scale[t].double().repeat_interleave(block, 1) for t in range(2))
    x = (q[0].double() @ k.T) * sm
    p = torch.softmax(x, -1)
    want, spread = p @ v, (q[0].double() @ k.abs().T).amax(-1, keepdim=True) * sm
    ds = (dim + 8) * 2.0 ** -22 * spread
    # the largest product of probability and scale is the heavy slot's, below 1
    tol = HALF_ULP[tdt] * want + TINY[tdt] + (2.0 ** -10 + 2 * ds) * want * (1 + HALF_ULP[tdt]) + n * FLOOR[path]
    got = cache.attend(q.repeat(seqs, 1, 1), path=path).double()
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("path,dim,block,news", [(1, 80, 40, 3), (2, 128, 128, 1), (2, 128, 128, 3), (2, 128, 64, 1), (2, 128, 32, 3), (2, 64, 64, 3), (2, 64, 32, 1), (3, 128, 128, 3), (3, 64, 64, 3), (3, 128, 64, 3), (3, 128, 32, 1), (3, 64, 32, 3)])
def test_fp16_outputs_are_off_by_their_own_rounding_alone(bq, path, dim, block, news):
    """The root mean square of the errors against 64 bits is that of rounding the exact outputs to fp16, within 5 %: what the scores'
    fp32 sums and probabilities of 22 bits add is below 2^-16 of the outputs, a thirty-second of that rounding.  (Probabilities of 11 bits
    add as much as the outputs' own 11 bits do for few slots, a third of it here.)"""
    lens = [40, 300, 90, 170]
    c = Case(bq, lens, [news] * 4, 4, 4, dim, block, 16, torch.float16, seed=dim + block + news)
    sm = 0.02                                                        # scores, and with them what fp32 loses of them, are small
    out, _ = c.attend(False, path=path, sm=sm)
    got, qd = out.double().cpu().numpy(), c.q.double().numpy()
    want = np.concatenate([ko.attend(qd[c.starts_host[s]:c.starts_host[s + 1]], *c.values[s], sm)["out"] for s in range(4)])
    rms = lambda x: float(np.sqrt(np.mean(x * x)))                   # noqa: E731
    assert rms(got - want) <= 1.05 * rms(want.astype(np.float16).astype(np.float64) - want)


def visible(c):
    return [[max(0, c.lens[s] - c.news[s] + i + 1) for i in range(c.news[s])] for s in range(len(c.lens))]


@pytest.mark.parametrize("path,dim,block", [(1, 80, 40), (2, 128, 128), (2, 128, 64), (2, 64, 32), (3, 128, 128), (3, 128, 64), (3, 64, 32)])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("flip", [False, True])
def test_values_that_grow_along_a_sequence(bq, path, dim, block, new, flip):
    """By 2^20 from one end to the other, on every kernel: the outputs' scale changes on the way."""
    c = Case(bq, [256], [new], 1, 4, dim, block, 16, torch.bfloat16)
    f = 2.0 ** np.round(np.linspace(-10, 10, 256))
    for j, x in enumerate(f[::-1] if flip else f):
        scale_values(c, 0, [j], float(x))
    check_rows(c, *c.attend(True, path=path), visible(c), dim ** -0.5, FLOOR[path])


IRREGULAR = [-1, -0.6961928, -0.5250731, -0.3949175, -0.2844414, -0.1847734, -0.0910500, 0, 0.0795803, 0.1609302, 0.2461123, 0.3379152, 0.4407098, 0.5626170, 0.7229568, 1.0]


@pytest.mark.parametrize("path,dim,block", [(1, 80, 40), (2, 128, 64), (2, 64, 64), (3, 128, 64), (3, 64, 64)])
@pytest.mark.parametrize("regular", [True, False])
@pytest.mark.parametrize("news", [[1, 1], [40, 30]])
def test_user_codebooks_on_every_kernel(bq, path, dim, block, regular, news):
    values = [i / 8 for i in range(-8, 8)] if regular else IRREGULAR
    c = Case(bq, [100, 61], news, 2, 4, dim, block, 16, torch.float16, values=values)
    c.check(c.attend(False, path=path, sm=0.02)[0], sm=0.02, values_11_bits=not regular and path != 1)


@pytest.mark.parametrize("tdt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,block", [(128, 128), (128, 32), (64, 64)])
@pytest.mark.parametrize("weights", [False, True])
def test_prompts_beyond_the_bounds_of_the_launch(bq, dim, block, weights, tdt):
    """max_new and max_len far below the truth: a CTA of the prompt kernels takes several blocks of rows, and several of slots, one
    after the other; sequences with no rows, or rows that see nothing, in between."""
    lens, news = [700, 0, 5, 400, 300, 130], [600, 0, 200, 0, 300, 130]
    c = Case(bq, lens, news, 1, 3, dim, block, 16, tdt, seed=dim + block)
    c.check(*c.attend(weights, path=3, max_new=1, max_len=8))


@pytest.mark.parametrize("path,dim,block,group", [(1, 80, 40, 2), (2, 128, 64, 2), (2, 64, 64, 12), (3, 64, 64, 2), (0, 128, 128, 1)])
@pytest.mark.parametrize("seqs", [33, 70, 1100])
def test_many_sequences(bq, path, dim, block, group, seqs):
    """More sequences than a warp has lanes, and than two steps of the search for a row's sequence cover; some without rows, some
    without slots, several such in a row.  Store and read of the same rows too."""
    rng = np.random.default_rng(seqs)
    top = 70 if seqs < 1000 else 24
    lens = [0 if s % 7 == 3 else int(rng.integers(1, top)) for s in range(seqs)]
    news = [0 if s % 5 in (1, 2) or 40 <= s < 44 else int(rng.integers(1, 4)) for s in range(seqs)]
    c = Case(bq, lens, news, 1, group, dim, block, 16, torch.bfloat16, seed=seqs)
    for weights in (False, True):
        c.check(*c.attend(weights, path=path))
    n = int(c.starts_host[-1])
    k, v = c.cache.read(c.starts, n, torch.bfloat16)
    want = np.zeros((2, n, 1, dim), np.uint16)
    for s in range(seqs):
        for i in range(news[s]):
            j = lens[s] - news[s] + i
            if j >= 0:
                for t in range(2):
                    want[t, c.starts_host[s] + i] = ko.read(c.values[s][t][j], DT[torch.bfloat16])
    assert np.array_equal(bits(k), want[0]) and np.array_equal(bits(v), want[1])
    before = [p.clone() for p in c.pools]
    c.cache.append(k, v, c.starts)                                   # what was read, quantized again, into the same slots and no others
    again = c.cache.read(c.starts, n, torch.bfloat16)
    hit = torch.zeros(c.pools[0].shape[0], 16, dtype=torch.bool)
    table = c.cache.table.cpu()
    for s in range(seqs):
        for j in range(max(0, lens[s] - news[s]), lens[s]):
            hit[int(table[s, j // 16]), j % 16] = True
    hit = hit.cuda()
    for p, b in zip(c.pools, before):
        p, b = p.view(torch.uint8).transpose(1, 2), b.view(torch.uint8).transpose(1, 2)
        assert torch.equal(p[~hit], b[~hit])
    assert all(bool(torch.isfinite(a).all()) for a in again)


def test_evict_of_many_sequences(bq):
    lens = [(s * 37) % 120 for s in range(300)]
    c = Case(bq, lens, [1] * 300, 1, 1, 64, 64, 16, torch.bfloat16)
    g = torch.Generator().manual_seed(1)
    w = torch.rand(300, 1, c.cache.capacity, generator=g)
    wd = w.cuda()
    c.cache.evict(wd, 50, sinks=2, recent=9)
    new = [min(n, 50) for n in lens]
    assert c.cache.lens.tolist() == new
    ks, vs = c.cache.read(torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda(), sum(new), torch.bfloat16)
    at = 0
    for s, n in enumerate(lens):
        place = ko.evict_places(w[s, 0].numpy(), n, 50, 2, 9)
        for t, vals in ((ks, c.values[s][0]), (vs, c.values[s][1])):
            assert np.array_equal(bits(t[at:at + new[s], 0]), ko.read(vals[place, 0], DT[torch.bfloat16])), s
        at += new[s]


def test_the_stride_of_a_single_row_means_nothing(bq):
    """One row cut from a wider tensor, whatever its stride says: the same kernels, the same bits."""
    c = Case(bq, [130], [1], 2, 4, 128, 64, 16, torch.float16)
    q = c.q.cuda()
    for stride in (1025, 1, 0):
        cut = torch.empty_strided((1, 8, 128), (stride, 128, 1), dtype=torch.float16, device="cuda").copy_(q)
        for path in (1, 2, 3):
            for weights in (False, True):
                want, got = c.attend(weights, path=path), c.attend(weights, path=path, q=cut)
                assert torch.equal(got[0], want[0]) and (not weights or torch.equal(got[1], want[1]))
    kv = torch.randn(1, 2, 128, device="cuda").half()
    c.cache.append(kv, kv * 2)
    want = [p.clone() for p in c.pools]
    for p in c.pools:
        p[c.cache.table[0, 8].item(), :, 1] = 0
    cut = torch.empty_strided((1, 2, 128), (3, 128, 1), dtype=torch.float16, device="cuda").copy_(kv)
    c.cache.append(cut, kv * 2)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(c.pools, want))


@pytest.mark.parametrize("path", [1, 2, 3])
def test_outputs_in_place_of_the_queries(bq, path):
    """Without weights out may be q; weights read the queries again, and a shifted out is never what a caller means."""
    for lens, news in (([130, 9000, 0], [3, 2, 1]), ([300, 20, 0], [200, 20, 7])):
        c = Case(bq, lens, news, 2, 4, 128, 64, 16, torch.bfloat16)
        want, want_w = c.attend(True, path=path)
        q = c.q.cuda()
        w = torch.full_like(want_w, 0.25)
        with pytest.raises(BqError):
            c.cache.attend(q, c.starts, max(news), weights=w, out=q, path=path)
        assert torch.equal(q, c.q.cuda()) and bool((w == 0.25).all())
        assert torch.equal(c.cache.attend(q, c.starts, max(news), out=q, path=path), want) and torch.equal(q, want)
        n = q.shape[0]
        room = torch.zeros(2 * n + 1, 8, 128, dtype=torch.bfloat16, device="cuda")
        room[:n] = c.q.cuda()
        for shift in (1, n - 1):
            with pytest.raises(BqError):
                c.cache.attend(room[:n], c.starts, max(news), out=room[shift:shift + n], path=path)
        c.cache.attend(room[:n], c.starts, max(news), out=room[n:2 * n], path=path)      # next to it: no memory shared
        assert torch.equal(room[n:2 * n], want)
        wide = torch.zeros(n, 24, 128, dtype=torch.bfloat16, device="cuda")
        wide[:, :8] = c.q.cuda()
        with pytest.raises(BqError):
            c.cache.attend(wide[:, :8], c.starts, max(news), out=wide.view(-1)[:n * 1024].view(n, 8, 128), path=path)
