"""Operators of a decoder layer that serves many requests at once, around the 4-bit cache and the decomposed linear layers:
queries and keys turned by their positions on the way into the cache, attention of a batch whose sequences begin with the
same rows, and the low-rank adapters of the requests beside a shared projection.  Every case can be run in a plain form
(elementary torch operations in fp32, in 64 bits in front of the cache's codes) or through the package's calls.

A cache holds, per page and head, rows of packed codes (element 2i in the low nibble of byte i) and one bf16 scale per
`block` elements of a row: value = codebook[code] * scale.  `lens` counts a sequence's rows, those of the present call
included; the rows of a call are the last ones of their sequence.
"""
import math

import numpy as np
import torch

own = False

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
BASE = 10000.0


# ---------------------------------------------------------------------------------------------- cases
def _rotary(name, seqs, new, ctx, far, heads, group, dim, block, page, axes, interleaved, dtype):
    return {"name": name, "op": "rotary", "seqs": seqs, "new": new, "ctx": ctx, "far": far, "heads": heads, "group": group, "dim": dim, "block": block,
            "page": page, "axes": axes, "interleaved": interleaved, "dtype": dtype}


def _shared(name, prefixes, prefix, seqs, new, ctx, heads, group, dim, block, page, dtype, weights):
    return {"name": name, "op": "shared", "prefixes": prefixes, "prefix": prefix, "seqs": seqs, "new": new, "ctx": ctx, "heads": heads, "group": group,
            "dim": dim, "block": block, "page": page, "dtype": dtype, "weights": weights}


def _adapted(name, seqs, new, k, n, features, adapters, rank, norm, dtype):
    return {"name": name, "op": "adapted", "seqs": seqs, "new": new, "k": k, "n": n, "features": features, "adapters": adapters, "rank": rank,
            "norm": norm, "dtype": dtype}


def listed():
    return [
        # a single user's next token: latency
        _rotary("rotary_one", 1, 1, 500, 0, 8, 4, 128, 128, 64, 1, False, "f16"),
        # a decode step of a batch whose bounded caches hold far fewer rows than their sequences have had tokens
        _rotary("rotary_step", 64, 1, 300, 1000000, 8, 8, 128, 64, 64, 1, False, "bf16"),
        # prompts of a batch, ragged, written at once
        _rotary("rotary_prompts", 8, 2048, 0, 0, 8, 4, 128, 128, 64, 1, False, "bf16"),
        # images and video frames: positions in time, height and width
        _rotary("rotary_frames", 3, 1500, 77, 0, 4, 7, 128, 64, 32, 3, True, "f16"),
        # a few answers to one question, sampled side by side
        _shared("shared_few", 1, 2000, 4, 1, 40, 8, 4, 128, 128, 64, "f16", False),
        # a decode step of a serving batch behind one long system prompt
        _shared("shared_step", 1, 8192, 64, 1, 511, 8, 8, 128, 64, 64, "bf16", False),
        # three tenants' prompts of different lengths; the weights that an eviction of the own rows goes by
        _shared("shared_tenants", 3, 16000, 48, 1, 900, 16, 2, 64, 32, 16, "f16", True),
        # questions of up to 200 tokens behind the same documents
        _shared("shared_questions", 2, 6000, 16, 200, 0, 8, 4, 128, 128, 64, "bf16", False),
        # one request with its adapter: latency
        _adapted("adapted_one", 1, 1, 4096, 4096, 0, 3, 16, False, "bf16"),
        # a decode step of 64 requests on 40 adapters, some without one
        _adapted("adapted_step", 64, 1, 8192, 8192, 8, 40, 16, False, "f16"),
        # ragged prompts with larger adapters, odd sizes
        _adapted("adapted_mixed", 33, 57, 2048, 2312, 6, 9, 64, False, "f16"),
        # a prefill batch behind the norm
        _adapted("adapted_prefill", 5, 1400, 6144, 16384, 6, 8, 16, True, "bf16"),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, v))


def draw(rng):
    op = rng.choice(["rotary", "shared", "adapted"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "adapted":
        seqs = _log(rng, 1, 64)
        new = _log(rng, 1, max(1, 4096 // seqs)) if rng.random() < 0.6 else 1
        k, n = 16 * _log(rng, 16, 512), _log(rng, 64, 8192)
        c = _adapted("", seqs, new, k, n if rng.random() < 0.2 else (n + 7) // 8 * 8, rng.choice([0, 1, 6, 16, 40]), _log(rng, 1, 48), rng.choice([16, 16, 32, 64]),
                     rng.random() < 0.5, dtype)
    else:
        dim, block = rng.choice([(128, 128), (128, 64), (128, 32), (64, 64), (64, 32), (128, 64), (80, 40)])
        page, heads, group = rng.choice([16, 32, 64, 128]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
        if op == "rotary":
            seqs = _log(rng, 1, 64)
            new = _log(rng, 1, 8192 // seqs) if rng.random() < 0.7 else 1
            c = _rotary("", seqs, new, rng.randrange(0, 400), rng.choice([0, 0, _log(rng, 1000, 2000000)]), heads, group, dim, block, page,
                        rng.choice([1, 1, 2, 3]), rng.random() < 0.4, dtype)
        else:
            prefixes = rng.choice([1, 1, 1, 2, 5])
            seqs = _log(rng, prefixes, 64)
            new = 1 if rng.random() < 0.6 else _log(rng, 1, max(1, 1024 // seqs))
            c = _shared("", prefixes, _log(rng, 16, (16384 if new == 1 else 6000) // prefixes), seqs, new, rng.randrange(0, 600), heads, group, dim, block, page, dtype, rng.random() < 0.3)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------- sizes that go by the case alone
def _news(case):
    """New rows of each sequence: the first has all of `new`, the others between a quarter and all of it."""
    s, new = case["seqs"], case["new"]
    return [max(1, new - (i * 7 % s) * (new * 3 // 4) // s) for i in range(s)]


def _lens(case):
    """Own rows of each sequence at the call: the first has the longest context, the others down to a quarter of it."""
    s = case["seqs"]
    return [case["ctx"] - (i * 5 % s) * (case["ctx"] * 3 // 4) // s + n for i, n in enumerate(_news(case))]


def _prefixes(case):
    """Rows of each shared beginning, and the sequences that share them: all but an equal share may go to the first."""
    p, s = case["prefixes"], case["seqs"]
    lens = [case["prefix"] - (i * 3 % p) * (case["prefix"] // 2) // p for i in range(p)]
    return lens, [i * i * s // (p * p) if i < p else s for i in range(p + 1)]


def _ids(case):
    """The adapter of each sequence; every seventh has none."""
    return [-1 if i % 7 == 5 else (i * 11 + 2) % case["adapters"] for i in range(case["seqs"])]


def _row_bytes(case):
    return case["dim"] // 2 + 2 * (case["dim"] // case["block"])


def work(case):
    op, news = case["op"], _news(case)
    rows = sum(news)
    if op == "adapted":
        k, n, f, r = case["k"], case["n"], case["features"], case["rank"]
        used = len({i for i in _ids(case) if i >= 0})
        adapted = sum(m for m, i in zip(news, _ids(case)) if i >= 0)
        bytes_ = rows * k * 2 * (3 if case["norm"] else 1) + n * k + 4 * n + 2 * f * (rows + n) + 2 * rows * n + used * r * (k + n) * 2
        return {"bytes": bytes_, "flops": 2.0 * rows * n * k + 2.0 * adapted * r * (k + n)}
    h, d, g = case["heads"], case["dim"], case["group"]
    if op == "rotary":
        # queries in and out; keys and values in, into the cache and out of it through the 16-bit type
        return {"bytes": rows * (2 * 2 * h * g * d + 2 * h * (2 * 2 * d + 2 * _row_bytes(case))) + 4 * rows * case["axes"], "flops": 3.0 * rows * h * d * (g + 1)}
    lens, (plens, members) = _lens(case), _prefixes(case)
    pairs = sum(n * (l - n) + n * (n + 1) // 2 for n, l in zip(news, lens))
    for p, l in enumerate(plens):
        pairs += l * sum(news[members[p]:members[p + 1]])
    w = 8 * sum(lens) * h if case["weights"] else 0
    return {"bytes": 2 * 2 * rows * h * g * d + (sum(lens) + sum(plens)) * h * 2 * _row_bytes(case) + w, "flops": 4.0 * pairs * h * g * d}


# ---------------------------------------------------------------------------------------------- the 4-bit rows, plain
def _codebook():
    """The 16 values of the 4-bit dynamic map and the 15 midpoints rounded toward -inf, as fp32."""
    mags = [np.float32(float(2 ** (k + 1) + 9 * (2 * j + 1)) / float(2 ** (k + 1) * 10 ** (3 - k))) for k in range(3) for j in range(2 ** k)]
    vals = np.sort(np.array([0.0, 1.0] + mags + [-m for m in mags], np.float32))
    mid = (vals[:-1].astype(np.float64) + vals[1:].astype(np.float64)) / 2
    thr = mid.astype(np.float32)
    thr = np.where(thr.astype(np.float64) > mid, np.nextafter(thr, np.float32(-np.inf)), thr)
    return vals, thr


def _quantize(x, block, thr):
    """Rows [..., D] -> packed codes [..., D / 2] and bf16 scales [..., D / block]."""
    f = x.float().unflatten(-1, (-1, block))
    a = f.abs().amax(-1)
    up = ((a.view(torch.int32) + 0xFFFF) & -65536).clamp(max=0x7F7F0000).view(torch.float32)      # toward +infinity to a bf16
    xhat = f / torch.where(up == 0, torch.ones_like(up), up)[..., None]
    c = torch.bucketize(xhat, thr, out_int32=True).flatten(-2)                                    # the number of midpoints below xhat
    return (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8), up.to(torch.bfloat16)


def _dequantize(codes, scale, vals):
    """The fp32 values of packed rows."""
    byte = torch.arange(256, device=codes.device)
    lut = torch.stack([vals[byte & 15], vals[byte >> 4]], -1)
    f = lut.index_select(0, codes.reshape(-1).int()).view(*codes.shape[:-1], -1)
    return (f.unflatten(-1, (scale.shape[-1], -1)) * scale.float()[..., None]).flatten(-2)


def _fetch(st, table, slots):
    """The fp32 keys and values of slots 0 .. slots - 1 of every sequence of a table: [S, H, slots, D]."""
    s, h, page = table.shape[0], st["kc"].shape[1], st["page"]
    at = torch.arange(slots, device=table.device)
    pg = table.long()[:, at // page][:, None].expand(s, h, slots)
    hd = torch.arange(h, device=table.device)[None, :, None]
    row = (at % page)[None, None]
    return [_dequantize(st[c][pg, hd, row], st[b][pg, hd, row], st["vals"]) for c, b in (("kc", "ks"), ("vc", "vs"))]


# ---------------------------------------------------------------------------------------------- inputs
def _pools(case, lens, gen, dev, fill):
    """Page table of shuffled pages, and pools with a page more than the sequences need.  `fill`: rows as a model writes them."""
    page, h, d, block = case["page"], case["heads"], case["dim"], case["block"]
    width = (max(lens) + page - 1) // page
    n_pages = len(lens) * width + 1
    table = torch.randperm(n_pages, generator=gen, device=dev)[:len(lens) * width].view(len(lens), width).int()
    vals, thr = (torch.from_numpy(a).to(dev) for a in _codebook())
    st = {"table": table, "page": page, "block": block, "vals": vals, "thr": thr}
    for c, b, amp in (("kc", "ks", 1.0), ("vc", "vs", 0.7)):
        st[c] = torch.zeros((n_pages, h, page, d // 2), dtype=torch.uint8, device=dev)
        st[b] = torch.zeros((n_pages, h, page, d // block), dtype=torch.bfloat16, device=dev)
        step = max(1, (1 << 25) // (h * page * d))
        for p in range(0, n_pages if fill else 0, step):
            x = torch.randn((min(step, n_pages - p), h, page, d), generator=gen, device=dev) * amp
            x[..., d // 3] *= 4                                       # a heavy channel, as keys and values have them
            st[c][p:p + step], st[b][p:p + step] = _quantize(x.to(torch.bfloat16), block, thr)
    return st


def _starts(news, dev):
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    return torch.tensor(starts, dtype=torch.int32, device=dev), starts[-1]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 2 + 1)
    return {"rotary": _prepare_rotary, "shared": _prepare_shared, "adapted": _prepare_adapted}[case["op"]](case, gen, dev)


def _sections(case):
    """Pairs of a head's row that turn with each axis: time has fewer, the rest is shared evenly."""
    half, axes = case["dim"] // 2, case["axes"]
    first = half if axes == 1 else half // (axes + 1)
    rest = [(half - first) // max(1, axes - 1)] * (axes - 1)
    return [half - sum(rest)] + rest


def _frequencies(case):
    return [BASE ** (-2.0 * i / case["dim"]) for i in range(case["dim"] // 2)]


def _prepare_rotary(case, gen, dev):
    news, lens, h, d, dt = _news(case), _lens(case), case["heads"], case["dim"], DT[case["dtype"]]
    st = _pools(case, lens, gen, dev, False)
    st["case"], st["lens"] = dict(case), torch.tensor(lens, dtype=torch.int32, device=dev)
    st["starts"], st["rows"] = _starts(news, dev)
    # the projection of queries, keys and values, whose slices the call takes
    n_q = h * case["group"]
    qkv = torch.randn((st["rows"], n_q + 2 * h, d), generator=gen, device=dev)
    qkv[..., d // 3] *= 4
    qkv = qkv.to(dt)
    st["q"], st["k"], st["v"] = qkv[:, :n_q], qkv[:, n_q:n_q + h], qkv[:, n_q + h:]
    # tokens that a sequence has had before: its slots, or (of a bounded cache) many more
    seq, i, slot = _seq_rows(st)
    away = torch.randint(0, max(case["far"], 1), (case["seqs"],), generator=gen, device=dev)
    pos = (slot + away[seq])[None]
    if case["axes"] > 1:                                              # frames of 16 x 24 patches
        pos = torch.stack([pos[0] // 384, pos[0] // 24 % 16, pos[0] % 24][:case["axes"]])
    st["positions"] = pos.int().contiguous()
    if own:
        import paper_2407_19775_b200 as bq
        st["cache"] = bq.KvCache4(st["kc"], st["vc"], st["ks"], st["vs"], st["table"], st["lens"], bq.Codebook4())
        st["rotary"] = bq.Rotary(d, base=BASE, sections=_sections(case), interleaved=case["interleaved"])
    else:
        st["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device=dev)
        st["axis"] = torch.tensor([a for a, n in enumerate(_sections(case)) for _ in range(n)], device=dev)
    return st


def _prepare_shared(case, gen, dev):
    news, lens, h, d = _news(case), _lens(case), case["heads"], case["dim"]
    plens, members = _prefixes(case)
    st = _pools(case, lens + plens, gen, dev, True)                   # one pool of pages for the beginnings and what follows them
    st["case"] = dict(case)
    width = (max(lens) + case["page"] - 1) // case["page"]
    st["prefix_table"], st["table"] = st["table"][len(lens):], st["table"][:len(lens), :width]
    st["lens"], st["prefix_lens"] = (torch.tensor(v, dtype=torch.int32, device=dev) for v in (lens, plens))
    st["starts"], st["rows"] = _starts(news, dev)
    st["members"] = torch.tensor(members, dtype=torch.int32, device=dev)
    st["q"] = torch.randn((st["rows"], h * case["group"], d), generator=gen, device=dev).to(DT[case["dtype"]])
    st["max_new"], st["max_len"], st["max_prefix"] = max(news), max(lens), max(plens)
    st["most"] = max(sum(news[a:b]) for a, b in zip(members, members[1:]))
    if case["weights"]:
        st["weights"] = torch.zeros((case["seqs"], h, width * case["page"]), device=dev)
    if own:
        import paper_2407_19775_b200 as bq
        book = bq.Codebook4()
        pools = [st[c] for c in ("kc", "vc", "ks", "vs")]
        st["cache"] = bq.KvCache4(*pools, st["table"], st["lens"], book)
        st["prefix"] = bq.KvCache4(*pools, st["prefix_table"], st["prefix_lens"], book)
    return st


def _prepare_adapted(case, gen, dev):
    k, n, f, a, r, dt = case["k"], case["n"], case["features"], case["adapters"], case["rank"], DT[case["dtype"]]
    starts, m = _starts(_news(case), dev)
    feat = torch.randperm(k, generator=gen, device=dev)[:f].sort().values
    x = torch.randn((m, k), generator=gen, device=dev) * 0.5
    x[:, feat] *= 30                                                  # the outlier channels that make a feature critical
    draw_ = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    st = {"case": dict(case), "x": x.to(dt), "w": (draw_(n, k) * 0.02).to(dt), "feat": feat.int(), "starts": starts, "rows": m,
          "ids": torch.tensor(_ids(case), dtype=torch.int32, device=dev),
          "a": (draw_(a, r, k) * k ** -0.5).to(dt), "b": (draw_(a, n, r) * 0.1).to(dt), "scale": torch.rand(a, generator=gen, device=dev) + 0.5,
          "gamma": (1 + 0.1 * draw_(k)).to(dt), "res": (draw_(m, k) * 0.5).to(dt) if case["norm"] else None}
    if own:
        import paper_2407_19775_b200 as bq
        st["layer"] = bq.DecomposedLinear(st["w"], feat.cpu().numpy())
        st["adapters"] = bq.Adapters(st["a"], st["b"], st["scale"])
    else:
        st["qw"], st["sw"] = _row_codes(st["w"].float(), feat)        # the weights' 8-bit rows are made once
    return st


def _row_codes(t, feat):
    """8-bit codes (as fp32) and absmax / 127 of rows; the critical features hold no code."""
    t = t.index_fill(1, feat, 0.0)
    a = t.abs().amax(1, keepdim=True)
    q = torch.round(t * 127.0 / torch.where(a == 0, torch.ones_like(a), a))
    return q, a / 127.0


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    return {"rotary": _run_rotary, "shared": _run_shared, "adapted": _run_adapted}[state["case"]["op"]](state)


def _seq_rows(st):
    """Sequence of each of the call's rows, its number among the sequence's rows of the call, and its slot."""
    starts = st["starts"].long()
    r = torch.arange(st["rows"], device=starts.device)
    seq = torch.bucketize(r, starts[1:], right=True)
    i = r - starts[seq]
    return seq, i, st["lens"].long()[seq] - (starts[1:] - starts[:-1])[seq] + i


def _turn(x, cos, sin, interleaved):
    """Pairs of x [rows, heads, D] by cos, sin [rows, 1, D / 2]: (2i, 2i + 1), or (i, i + D / 2)."""
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _run_rotary(st):
    case, dt = st["case"], DT[st["case"]["dtype"]]
    if own:
        q = st["cache"].append_rotary(st["q"], st["k"], st["v"], st["rotary"], st["positions"], st["starts"])
        return (q, *st["cache"].read(st["starts"], st["rows"], dt))
    # far positions' angles, and keys next to the borders between codes, in 64 bits
    angle = st["positions"].double()[st["axis"]].t()[:, None] * st["freq"]
    cos, sin = torch.cos(angle), torch.sin(angle)
    q = _turn(st["q"].float(), cos.float(), sin.float(), case["interleaved"]).to(dt)
    k = _turn(st["k"].double(), cos, sin, case["interleaved"]).float()
    seq, _, slot = _seq_rows(st)
    pg, row = st["table"][seq, slot // st["page"]].long(), slot % st["page"]
    got = [q]
    for x, c, b in ((k, "kc", "ks"), (st["v"], "vc", "vs")):
        codes, scale = _quantize(x, st["block"], st["thr"])
        st[c][pg, :, row] = codes
        st[b][pg, :, row] = scale
        got.append(_dequantize(st[c][pg, :, row], st[b][pg, :, row], st["vals"]).to(dt))
    return tuple(got)


def _run_shared(st):
    case = st["case"]
    if own:
        out = st["cache"].attend_shared(st["q"], st["prefix"], st["members"], st["starts"], st["max_new"], max_len=st["max_len"], max_shared=st["most"],
                                        max_prefix=st["max_prefix"], weights=st.get("weights"))
        return (out, st["weights"]) if case["weights"] else out
    s, h, g, d, n, length, p, rows = case["seqs"], case["heads"], case["group"], case["dim"], st["max_new"], st["max_len"], case["prefixes"], st["rows"]
    seq, i, slot = _seq_rows(st)
    members = st["members"].long()
    of = torch.bucketize(seq, members[1:], right=True)                # the beginning that a row's sequence shares
    j = torch.arange(rows, device=seq.device) - st["starts"].long()[members[:-1]][of]      # the row's number among those that share it
    q = st["q"].float().view(rows, h, g, d) * (1.0 / math.sqrt(d))
    qs, qp = (torch.zeros((*shape, h, g, d), device=seq.device) for shape in ((s, n), (p, st["most"])))
    qs[seq, i], qp[of, j] = q, q
    ks, vs = _fetch(st, st["table"], length)
    kp, vp = _fetch(st, st["prefix_table"], st["max_prefix"])
    last = torch.full((s, n), -1, device=seq.device)
    last[seq, i] = slot
    xs = qs.permute(0, 2, 1, 3, 4).reshape(s, h, n * g, d) @ ks.transpose(2, 3)
    hidden = (torch.arange(length, device=seq.device) > last[..., None]).repeat_interleave(g, 1)[:, None]
    xs.masked_fill_(hidden, -math.inf)
    xp = qp.permute(0, 2, 1, 3, 4).reshape(p, h, -1, d) @ kp.transpose(2, 3)
    xp.masked_fill_(torch.arange(st["max_prefix"], device=seq.device) >= st["prefix_lens"][:, None, None, None], -math.inf)
    # back to one row of the call each, the two parts' softmax joined
    own_part = lambda y: y.unflatten(2, (n, g)).permute(0, 2, 1, 3, 4)[seq, i]  # noqa: E731
    shared_part = lambda y: y.unflatten(2, (st["most"], g)).permute(0, 2, 1, 3, 4)[of, j]  # noqa: E731
    tops = [x.amax(-1, keepdim=True).clamp(min=-1e30) for x in (xs, xp)]
    es, ep = (x.sub_(t).exp_() for x, t in zip((xs, xp), tops))
    ts, tp = own_part(tops[0]), shared_part(tops[1])
    top = torch.maximum(ts, tp)
    fs, fp = torch.exp(ts - top), torch.exp(tp - top)
    total = fs * own_part(es.sum(-1, keepdim=True)) + fp * shared_part(ep.sum(-1, keepdim=True))
    out = (fs * own_part(es @ vs) + fp * shared_part(ep @ vp)) / total
    out = out.reshape(rows, h * g, d).to(st["q"].dtype)
    if not case["weights"]:
        return out
    factor = torch.zeros((s, n, h, g, 1), device=seq.device)
    factor[seq, i] = fs / total
    st["weights"][:, :, :length] += (es * factor.permute(0, 2, 1, 3, 4).reshape(s, h, n * g, 1)).sum(2)
    return out, st["weights"]


def _run_adapted(st):
    case = st["case"]
    if own:
        if case["norm"]:
            return st["layer"].norm_linear(st["x"], st["gamma"], EPS, residual=st["res"], adapters=st["adapters"], ids=st["ids"], starts=st["starts"])
        return st["layer"].linear(st["x"], adapters=st["adapters"], ids=st["ids"], starts=st["starts"])
    dt, feat = st["x"].dtype, st["feat"].long()
    h = st["x"]
    t = h.float()
    if case["norm"]:
        h = (t + st["res"].float()).to(dt)
        f = h.float()
        t = f * st["gamma"].float()
        r = 1.0 / torch.sqrt((f * f).sum(1, keepdim=True) / case["k"] + EPS)
    q, s = _row_codes(t, feat)                                        # the norm's factor of a row drops out of its codes
    if case["norm"]:
        s, t = s * r, t * r
    y = (q @ st["qw"].t()) * (s * st["sw"].t()) + t[:, feat].to(dt).float() @ st["w"][:, feat].float().t()
    # the adapters of all requests side by side; a row keeps its own
    ids = torch.repeat_interleave(st["ids"].long(), (st["starts"][1:] - st["starts"][:-1]).long(), output_size=st["rows"])
    a, rank = case["adapters"], case["rank"]
    mine = (ids[:, None] == torch.arange(a, device=ids.device)).float() * st["scale"]
    u = (t @ st["a"].float().view(a * rank, -1).t()).view(-1, a, rank) * mine[..., None]
    y = y + u.view(-1, a * rank) @ st["b"].float().permute(0, 2, 1).reshape(a * rank, -1)
    return (y.to(dt), h) if case["norm"] else y.to(dt)


# ---------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"rotary": _exact_rotary, "shared": _exact_shared, "adapted": _exact_adapted}[case["op"]](st, case)


def _exact_rotary(st, case):
    dev, d, half = st["q"].device, case["dim"], case["dim"] // 2
    pos = st["positions"].double().cpu().numpy()
    axis = np.repeat(np.arange(case["axes"]), _sections(case))
    z = torch.from_numpy(np.exp(1j * pos[axis].T * BASE ** (-np.arange(half) * 2.0 / d))).to(dev)[:, None]      # a turn of every pair

    def turned(x):
        x = x.double()
        pairs = x.view(*x.shape[:2], half, 2) if case["interleaved"] else x.view(*x.shape[:2], 2, half).transpose(2, 3)
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
        return (y if case["interleaved"] else y.transpose(2, 3)).reshape(x.shape)

    vals = torch.from_numpy(_codebook()[0]).double().to(dev)

    def stored(x):
        # by definition the cache's codec sees a row in 32 bits, and its quotient by the scale is one of 32 bits
        x = x.float().double().reshape(-1, case["block"])
        a = x.abs().amax(1)
        scale = a.to(torch.bfloat16)                                  # nearest, then one step up where that fell short
        bits = scale.view(torch.int16).int() + (scale.double() < a).int()
        scale = bits.to(torch.int16).view(torch.bfloat16).double()
        y = torch.empty_like(x)
        for p in range(0, len(x), 1 << 17):
            quotient = (x[p:p + (1 << 17)] / torch.where(scale == 0, 1.0, scale)[p:p + (1 << 17), None]).float().double()
            near = (quotient[..., None] - vals).abs()
            y[p:p + (1 << 17)] = vals[near.argmin(2)] * scale[p:p + (1 << 17), None]
        return y.view(-1, case["heads"], d)

    return turned(st["q"]), stored(turned(st["k"])), stored(st["v"].double())


def _exact_shared(st, case):
    dev, d, g, page = st["q"].device, case["dim"], case["group"], case["page"]
    vals = torch.from_numpy(_codebook()[0]).double().to(dev)

    def rows(table, n):
        """The first n rows of all heads of a sequence with this row of a table, in 64 bits."""
        at, got = torch.arange(n, device=dev), []
        for names in (("kc", "ks"), ("vc", "vs")):
            pg = table[at // page].long()
            c, b = st[names[0]][pg, :, at % page].long(), st[names[1]][pg, :, at % page].double()
            both = torch.stack([vals[c % 16], vals[c // 16]], 3).reshape(n, -1, d)
            got.append((both * torch.repeat_interleave(b, case["block"], 2)).transpose(0, 1))
        return got

    lens, plens, starts, members = (st[x].tolist() for x in ("lens", "prefix_lens", "starts", "members"))
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=dev)
    w = torch.zeros_like(st["weights"], dtype=torch.float64) if case["weights"] else None
    for p, pn in enumerate(plens):
        kp, vp = rows(st["prefix_table"][p], pn)
        for s in range(members[p], members[p + 1]):
            n, lo, hi = lens[s], starts[s], starts[s + 1]
            ks, vs = rows(st["table"][s], n)
            hidden = torch.arange(n, device=dev)[None] > (n - (hi - lo) + torch.arange(hi - lo, device=dev))[:, None]
            hidden = torch.cat([torch.zeros((hi - lo, pn), dtype=torch.bool, device=dev), hidden], 1)
            k, v = torch.cat([kp, ks], 1), torch.cat([vp, vs], 1)
            q = st["q"][lo:hi].double().view(hi - lo, -1, g, d).permute(1, 2, 0, 3)
            prob = torch.softmax((q @ k[:, None].transpose(2, 3) / math.sqrt(d)).masked_fill_(hidden, -math.inf), -1)
            out[lo:hi] = (prob @ v[:, None]).permute(2, 0, 1, 3).reshape(hi - lo, -1, d)
            if w is not None:
                w[s, :, :n] += prob[..., pn:].sum((1, 2))
    return out if w is None else (out, w)


def _exact_adapted(st, case):
    feat = st["feat"].long()
    y = st["x"].double()
    if case["norm"]:
        h = y + st["res"].double()
        h16 = h.to(st["x"].dtype).double()
        y = h16 * st["gamma"].double() / torch.sqrt(h16.square().mean(1, keepdim=True) + EPS)
    w = st["w"].double()
    critical = torch.zeros(case["k"], dtype=torch.bool, device=y.device)
    critical[feat] = True

    def eight(v):
        v = v.masked_fill(critical, 0.0)
        top = v.abs().amax(1, keepdim=True)
        return torch.round(127 * v / torch.where(top == 0, 1.0, top)) * top / 127

    z = eight(y) @ eight(w).t() + y[:, feat] @ w[:, feat].t()
    starts = st["starts"].tolist()
    for s, a in enumerate(st["ids"].tolist()):
        if a >= 0:
            part = slice(starts[s], starts[s + 1])
            z[part] += st["scale"][a].double() * (y[part] @ st["a"][a].double().t()) @ st["b"][a].double().t()
    return (z, h) if case["norm"] else z
