"""The operators of a decoder layer around the decomposed linear layers: the store of new key/value rows in a
4-bit cache, attention over that cache, eviction from it by accumulated attention weight, and the root-mean-square
norm that feeds a decomposed linear layer.  Every case can be run in a plain form (elementary torch operations in
fp32) or through the package's calls.

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


# ---------------------------------------------------------------------------------------------- cases
def _store(name, seqs, new, ctx, heads, dim, block, page, dtype):
    return {"name": name, "op": "store", "seqs": seqs, "new": new, "ctx": ctx, "heads": heads, "dim": dim, "block": block, "page": page, "dtype": dtype}


def _attend(name, seqs, new, ctx, heads, group, dim, block, page, dtype, weights):
    return {"name": name, "op": "attend", "seqs": seqs, "new": new, "ctx": ctx, "heads": heads, "group": group, "dim": dim, "block": block,
            "page": page, "dtype": dtype, "weights": weights}


def _evict(name, seqs, length, budget, sinks, recent, heads, dim, block, page):
    return {"name": name, "op": "evict", "seqs": seqs, "len": length, "budget": budget, "sinks": sinks, "recent": recent, "heads": heads, "dim": dim,
            "block": block, "page": page}


def _norm(name, tokens, k, n, features, residual, dtype):
    return {"name": name, "op": "norm", "tokens": tokens, "k": k, "n": n, "features": features, "residual": residual, "dtype": dtype}


def listed():
    return [
        # one decode step of a batch: a row per sequence and head
        _store("store_step", 64, 1, 300, 8, 128, 64, 64, "f16"),
        # prompts of a batch, ragged, written at once
        _store("store_prompts", 8, 2048, 0, 8, 128, 128, 64, "bf16"),
        # a single user's next token after a short prompt: latency
        _attend("attend_one", 1, 1, 500, 8, 4, 128, 128, 64, "f16", False),
        # a decode step of a serving batch with ragged contexts
        _attend("attend_batch", 64, 1, 8191, 8, 8, 128, 64, 64, "bf16", False),
        # two long documents
        _attend("attend_long", 2, 1, 131071, 8, 8, 128, 128, 128, "bf16", False),
        # a decode step that also accumulates the weights an eviction goes by; small pages, one query head per cache head
        _attend("attend_weights", 16, 1, 4099, 16, 1, 64, 32, 16, "f16", True),
        # prompts in chunks of 2048 tokens over a context of as many
        _attend("attend_chunk", 4, 2048, 2048, 8, 4, 128, 128, 64, "bf16", False),
        # short ragged prompts whose accumulated weights are wanted
        _attend("attend_prompt_weights", 6, 777, 0, 4, 7, 64, 64, 32, "f16", True),
        # steady state of a bounded cache: one row in, one row out, per sequence and head
        _evict("evict_step", 32, 1025, 1024, 4, 64, 8, 128, 64, 64),
        # long prompts cut down to what the decode steps will keep
        _evict("evict_prompts", 8, 32768, 2048, 16, 256, 8, 128, 64, 64),
        # the norm and the layer behind it, decode step
        _norm("norm_step", 64, 8192, 8192, 8, True, "f16"),
        # the same for a prefill batch
        _norm("norm_prefill", 4096, 6144, 16384, 6, True, "bf16"),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, v))


def _rows(rng):
    dim, block = rng.choice([(128, 128), (128, 64), (128, 32), (64, 64), (64, 32), (128, 64), (80, 40)])
    return dim, block, rng.choice([16, 32, 64, 128])


def draw(rng):
    while True:
        c = _one(rng)
        if 3072 not in {*c.values(), *([] if c["op"] == "norm" else _lens(c) + _news(c))}:
            return c


def _one(rng):
    op = rng.choice(["store", "attend", "attend", "attend", "evict", "norm"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "norm":
        tokens, k = _log(rng, 1, 4096), 16 * _log(rng, 16, 512)
        n = _log(rng, 64, 8192)
        n = n if rng.random() < 0.2 else (n + 7) // 8 * 8
        c = _norm("", tokens, k, n, rng.choice([0, 1, 6, 16, 40]), rng.random() < 0.8, dtype)
    else:
        dim, block, page = _rows(rng)
        heads = rng.choice([1, 2, 4, 8])
        if op == "store":
            seqs = _log(rng, 1, 64)
            c = _store("", seqs, _log(rng, 1, 16384 // seqs), rng.randrange(0, 400), heads, dim, block, page, dtype)
        elif op == "evict":
            seqs = _log(rng, 1, 32)
            length = _log(rng, 40, min(32768, 262144 // seqs))
            budget = max(8, int(length * rng.uniform(0.05, 1.0)))
            sinks = rng.randrange(0, budget // 4 + 1)
            c = _evict("", seqs, length, budget, sinks, rng.randrange(0, budget // 2 + 1), heads, dim, block, page)
        else:
            group, weights = rng.choice([1, 2, 4, 5, 7, 8, 16]), rng.random() < 0.4
            kind = rng.random()
            if kind < 0.6:
                seqs = _log(rng, 1, 64)
                new, ctx = 1, _log(rng, 1, min(131072, 524288 // seqs))
            elif kind < 0.75:                                        # a few tokens at once: drafted tokens to be checked
                seqs = _log(rng, 1, 32)
                new, ctx = rng.randrange(2, 9), _log(rng, 8, min(65536, 131072 // seqs))
            else:
                seqs, group = _log(rng, 1, 8), min(group, 8)
                new = _log(rng, 9, 2048 // seqs * 2 if seqs > 2 else 1024)
                ctx = rng.choice([0, _log(rng, 1, 2048)])
            c = _attend("", seqs, new, ctx, heads, group, dim, block, page, dtype, weights)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------- sizes that go by the case alone
def _news(case):
    """New rows of each sequence: the first has all of `new`, the others between a quarter and all of it."""
    s, new = case["seqs"], case.get("new", 1)
    return [max(1, new - (i * 7 % s) * (new * 3 // 4) // s) for i in range(s)]


def _lens(case):
    """Rows of each sequence at the call: the first has the longest context, the others down to a quarter of it."""
    s = case["seqs"]
    if case["op"] == "evict":
        return [case["len"] - (i * 5 % s) * (case["len"] // 8) // s for i in range(s)]
    return [case["ctx"] - (i * 5 % s) * (case["ctx"] * 3 // 4) // s + n for i, n in enumerate(_news(case))]


def _pairs(case):
    """(query, key) pairs that the causal mask leaves, over all sequences."""
    return sum(n * (l - n) + n * (n + 1) // 2 for n, l in zip(_news(case), _lens(case)))


def _row_bytes(case):
    return case["dim"] // 2 + 2 * (case["dim"] // case["block"])


def work(case):
    op = case["op"]
    if op == "norm":
        m, k, n, f = case["tokens"], case["k"], case["n"], case["features"]
        side = 2 * f * (m + n)
        return {"bytes": m * k * 2 * (3 if case["residual"] else 1) + 2 * k + n * k + 4 * n + side + 2 * m * n, "flops": 2.0 * m * n * k}
    h, d = case["heads"], case["dim"]
    if op == "store":
        rows = sum(_news(case)) * h
        # in and out through the 16-bit type, and the cache's rows written and read
        return {"bytes": 2 * rows * (2 * 2 * d + 2 * _row_bytes(case)), "flops": 2.0 * rows * d * 6}
    if op == "evict":
        lens = _lens(case)
        kept = sum(min(l, case["budget"]) for l in lens) * h
        moved = sum(min(l - case["budget"], case["budget"]) for l in lens if l > case["budget"]) * h
        return {"bytes": 4 * sum(lens) * h + 2 * moved * 2 * _row_bytes(case) + kept * 2 * (_row_bytes(case) + 2 * d), "flops": float(sum(lens) * h)}
    q = sum(_news(case)) * h * case["group"] * d * 2
    w = 8 * sum(_lens(case)) * h if case["weights"] else 0
    return {"bytes": 2 * q + sum(_lens(case)) * h * 2 * _row_bytes(case) + w, "flops": 4.0 * _pairs(case) * h * case["group"] * d}


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


def _pool_index(table, page, slots):
    """Page and row in the page of slots [S, n] of each sequence."""
    return torch.gather(table, 1, slots // page).long(), slots % page


def _fetch(st, slots):
    """The fp32 keys and values of slots [S, H, n]."""
    s, h, n = slots.shape
    pg, row = _pool_index(st["table"].long(), st["page"], slots.reshape(s, -1))
    pg, row = pg.view(s, h, n), row.view(s, h, n)
    hd = torch.arange(h, device=slots.device)[None, :, None]
    return [_dequantize(st[c][pg, hd, row], st[b][pg, hd, row], st["vals"]) for c, b in (("kc", "ks"), ("vc", "vs"))]


# ---------------------------------------------------------------------------------------------- inputs
def _pools(case, lens, gen, dev, fill):
    """Page table of shuffled pages, and pools with a page more than the sequences need.  `fill`: rows as a model writes them."""
    page, h, d, block = case["page"], case["heads"], case["dim"], case["block"]
    width = (max(lens) + page - 1) // page
    n_pages = case["seqs"] * width + 1
    table = torch.randperm(n_pages, generator=gen, device=dev)[:case["seqs"] * width].view(case["seqs"], width).int()
    vals, thr = (torch.from_numpy(a).to(dev) for a in _codebook())
    st = {"table": table, "lens": torch.tensor(lens, dtype=torch.int32, device=dev), "page": page, "block": block, "vals": vals, "thr": thr}
    for c, b, amp in (("kc", "ks", 1.0), ("vc", "vs", 0.7)):
        st[c] = torch.zeros((n_pages, h, page, d // 2), dtype=torch.uint8, device=dev)
        st[b] = torch.zeros((n_pages, h, page, d // block), dtype=torch.bfloat16, device=dev)
        step = max(1, (1 << 25) // (h * page * d))
        for p in range(0, n_pages if fill else 0, step):
            x = torch.randn((min(step, n_pages - p), h, page, d), generator=gen, device=dev) * amp
            x[..., d // 3] *= 4                                       # a heavy channel, as keys and values have them
            st[c][p:p + step], st[b][p:p + step] = _quantize(x.to(torch.bfloat16), block, thr)
    return st


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 2 + 1)
    if case["op"] == "norm":
        return _prepare_norm(case, gen, dev)
    lens, news = _lens(case), _news(case)
    st = _pools(case, lens, gen, dev, case["op"] != "store")
    st["case"] = dict(case)
    starts = [0]
    for n in news if case["op"] != "evict" else [min(l, case["budget"]) for l in lens]:
        starts.append(starts[-1] + n)
    st["starts"], st["rows"] = torch.tensor(starts, dtype=torch.int32, device=dev), starts[-1]
    h, d = case["heads"], case["dim"]
    if case["op"] == "store":
        dt = DT[case["dtype"]]
        # keys and values as they leave the projection of queries, keys and values: slices of wider rows
        qkv = torch.randn((st["rows"], 3 * h, d), generator=gen, device=dev)
        qkv[..., d // 3] *= 4
        qkv = qkv.to(dt)
        st["k"], st["v"] = qkv[:, h:2 * h], qkv[:, 2 * h:]
    elif case["op"] == "attend":
        st["q"] = torch.randn((st["rows"], h * case["group"], d), generator=gen, device=dev).to(DT[case["dtype"]])
        st["max_new"], st["max_len"] = max(news), max(lens)
        if case["weights"]:
            st["weights"] = torch.zeros((case["seqs"], h, st["table"].shape[1] * case["page"]), device=dev)
    else:
        st["full"] = st["lens"].clone()
        # weights as attention leaves them: a few heavy rows, many light ones
        w = torch.rand((case["seqs"], h, st["table"].shape[1] * case["page"]), generator=gen, device=dev)
        st["weights"] = w ** 8
    if own:
        import paper_2407_19775_b200 as bq
        st["cache"] = bq.KvCache4(st["kc"], st["vc"], st["ks"], st["vs"], st["table"], st["lens"], bq.Codebook4())
    return st


def _prepare_norm(case, gen, dev):
    m, k, n, f, dt = case["tokens"], case["k"], case["n"], case["features"], DT[case["dtype"]]
    feat = torch.randperm(k, generator=gen, device=dev)[:f].sort().values
    x = torch.randn((m, k), generator=gen, device=dev) * 0.5
    x[:, feat] *= 30                                                  # the outlier channels that make a feature critical
    w = torch.randn((n, k), generator=gen, device=dev) * 0.02
    st = {"case": dict(case), "x": x.to(dt), "w": w.to(dt), "feat": feat.int(),
          "gamma": (1 + 0.1 * torch.randn(k, generator=gen, device=dev)).to(dt),
          "res": (torch.randn((m, k), generator=gen, device=dev) * 0.5).to(dt) if case["residual"] else None}
    if own:
        import paper_2407_19775_b200 as bq
        st["layer"] = bq.DecomposedLinear(st["w"], feat.cpu().numpy())
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
    return {"store": _run_store, "attend": _run_attend, "evict": _run_evict, "norm": _run_norm}[state["case"]["op"]](state)


def _seq_rows(st):
    """Sequence of each of the call's rows, its number among the sequence's rows of the call, and its slot."""
    starts = st["starts"].long()
    r = torch.arange(st["rows"], device=starts.device)
    seq = torch.bucketize(r, starts[1:], right=True)
    i = r - starts[seq]
    return seq, i, st["lens"].long()[seq] - (starts[1:] - starts[:-1])[seq] + i


def _rows_of(st, dt):
    """The values of the call's rows, [rows, heads, dim] in a 16-bit type."""
    seq, _, slot = _seq_rows(st)
    pg = st["table"][seq, slot // st["page"]].long()
    return [_dequantize(st[c][pg, :, slot % st["page"]], st[b][pg, :, slot % st["page"]], st["vals"]).to(dt) for c, b in (("kc", "ks"), ("vc", "vs"))]


def _run_store(st):
    dt = DT[st["case"]["dtype"]]
    if own:
        st["cache"].append(st["k"], st["v"], st["starts"])
        return st["cache"].read(st["starts"], st["rows"], dt)
    seq, _, slot = _seq_rows(st)
    pg, row = st["table"][seq, slot // st["page"]].long(), slot % st["page"]
    for x, c, b in ((st["k"], "kc", "ks"), (st["v"], "vc", "vs")):
        codes, scale = _quantize(x, st["block"], st["thr"])
        st[c][pg, :, row] = codes
        st[b][pg, :, row] = scale
    return _rows_of(st, dt)


def _run_attend(st):
    case = st["case"]
    if own:
        out = st["cache"].attend(st["q"], st["starts"], st["max_new"], max_len=st["max_len"], weights=st.get("weights"))
        return (out, st["weights"]) if case["weights"] else out
    s, h, g, d, n, length = case["seqs"], case["heads"], case["group"], case["dim"], st["max_new"], st["max_len"]
    seq, i, slot = _seq_rows(st)
    slots = torch.arange(length, device=slot.device).expand(s, h, length)
    k, v = _fetch(st, slots)                                          # [s, h, length, d]
    q = torch.zeros((s, n, h, g, d), device=slot.device)
    q[seq, i] = st["q"].float().view(-1, h, g, d)
    last = torch.full((s, n), -1, device=slot.device)
    last[seq, i] = slot
    seen = (slots[:, :1] <= last[:, :, None]).repeat_interleave(g, 1)[:, None]         # [s, 1, n g, length]
    x = (q.permute(0, 2, 1, 3, 4).reshape(s, h, n * g, d) @ k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    out = (p @ v).view(s, h, n, g, d).permute(0, 2, 1, 3, 4)[seq, i].reshape(-1, h * g, d).to(st["q"].dtype)
    if not case["weights"]:
        return out
    st["weights"][:, :, :length] += p.sum(2)
    return out, st["weights"]


def _run_evict(st):
    case = st["case"]
    st["lens"].copy_(st["full"])                                      # the rows that came in since the last pass
    if own:
        st["cache"].evict(st["weights"], case["budget"], sinks=case["sinks"], recent=case["recent"])
        return (*st["cache"].read(st["starts"], st["rows"], torch.bfloat16), st["weights"], st["lens"])
    b, sinks, recent, length, page = case["budget"], case["sinks"], case["recent"], case["len"], case["page"]
    w, lens = st["weights"], st["full"].long()
    s, h = w.shape[:2]
    slot = torch.arange(length, device=w.device).expand(s, h, length)
    n = lens[:, None, None]
    middle = (slot >= sinks) & (slot < n - recent)
    order = torch.sort(torch.where(middle, w[:, :, :length], torch.full_like(w[:, :, :length], -1.0)), dim=2, descending=True, stable=True).indices
    kept = torch.zeros_like(middle).scatter_(2, order[:, :, :b - sinks - recent], True)
    kept = kept & middle
    hole = middle & ~kept & (slot < b - recent)
    late = middle & kept & (slot >= b - recent)
    # the i-th hole takes the i-th late survivor; the recent rows slide down
    src = torch.sort(torch.where(late, slot, length + slot), dim=2).values
    src = torch.gather(src, 2, (hole.cumsum(2) - 1).clamp(min=0))
    src = torch.where(hole, src, slot)[:, :, :b]
    src = torch.where(slot[:, :, :b] >= b - recent, slot[:, :, :b] + n - b, src)
    src = torch.where(n > b, src, slot[:, :, :b])
    spg, srow = _pool_index(st["table"].long(), page, src.reshape(s, -1))
    dpg, drow = _pool_index(st["table"].long(), page, slot[:, :, :b].reshape(s, -1))
    hd = torch.arange(h, device=w.device)[None, :, None].expand(s, h, b).reshape(s, -1)
    for c in ("kc", "vc", "ks", "vs"):
        st[c][dpg, hd, drow] = st[c][spg, hd, srow]
    w[:, :, :b] = torch.gather(w, 2, src)
    st["lens"].copy_(lens.clamp(max=b))
    return (*_rows_of(st, torch.bfloat16), w, st["lens"])


def _run_norm(st):
    case = st["case"]
    if own:
        return st["layer"].norm_linear(st["x"], st["gamma"], EPS, residual=st["res"])
    feat = st["feat"].long()
    h = st["x"] if st["res"] is None else (st["x"].float() + st["res"].float()).to(st["x"].dtype)
    f = h.float()
    r = 1.0 / torch.sqrt((f * f).sum(1, keepdim=True) / case["k"] + EPS)
    t = f * st["gamma"].float()
    q, s = _row_codes(t, feat)                                        # the factor r of a row drops out of its codes
    y = (q @ st["qw"].t()) * ((s * r) * st["sw"].t())
    side = (t[:, feat] * r).to(h.dtype).float() @ st["w"][:, feat].float().t()
    return (y + side).to(h.dtype), h


# ---------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(st, case)
    dev = st["lens"].device
    vals = torch.from_numpy(_codebook()[0]).double().to(dev)
    lens, table, page, d = st["lens"].tolist(), st["table"].long(), case["page"], case["dim"]

    def rows(s, names, slots, h):
        """Rows `slots` of head h of sequence s, in 64 bits."""
        pg = table[s, slots // page]
        c, b = st[names[0]][pg, h, slots % page].long(), st[names[1]][pg, h, slots % page].double()
        both = torch.stack([vals[c % 16], vals[c // 16]], 2).reshape(len(slots), d)
        return both * torch.repeat_interleave(b, case["block"], 1)

    if case["op"] == "store":
        got = []
        for x in (st["k"].double(), st["v"].double()):
            x = x.reshape(-1, case["block"])
            a = x.abs().amax(1)
            scale = a.to(torch.bfloat16)                              # nearest, then one step up where that fell short
            bits = scale.view(torch.int16).int() + (scale.double() < a).int()
            scale = bits.to(torch.int16).view(torch.bfloat16).double()
            y = torch.empty_like(x)
            for p in range(0, len(x), 1 << 17):
                near = (x[p:p + (1 << 17), :, None] / torch.where(scale == 0, 1.0, scale)[p:p + (1 << 17), None, None] - vals).abs()
                y[p:p + (1 << 17)] = vals[near.argmin(2)] * scale[p:p + (1 << 17), None]
            got.append(y.view(-1, case["heads"], d))
        return got
    if case["op"] == "evict":
        b, sinks, recent = case["budget"], case["sinks"], case["recent"]
        w, ks, vs = st["weights"].double().cpu().numpy(), [], []
        out_w = w.copy()
        for s, n in enumerate(lens):
            k, v = [], []
            for h in range(case["heads"]):
                place = np.arange(min(n, b))
                if n > b:
                    mid = np.arange(sinks, n - recent)
                    best = mid[np.lexsort((mid, -w[s, h, mid]))[:b - sinks - recent]]
                    free = np.setdiff1d(np.arange(sinks, b - recent), best)
                    place[free] = np.sort(best[best >= b - recent])
                    place[b - recent:] = np.arange(n - recent, n)
                    out_w[s, h, :b] = w[s, h, place]
                at = torch.from_numpy(place).to(dev)
                k.append(rows(s, ("kc", "ks"), at, h))
                v.append(rows(s, ("vc", "vs"), at, h))
            ks.append(torch.stack(k, 1))
            vs.append(torch.stack(v, 1))
        return torch.cat(ks), torch.cat(vs), torch.from_numpy(out_w), np.minimum(np.array(lens, np.int32), b)
    starts, g = st["starts"].tolist(), case["group"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=dev)
    w = torch.zeros_like(st["weights"], dtype=torch.float64) if case["weights"] else None
    for s, n in enumerate(lens):
        lo, hi = starts[s], starts[s + 1]
        at = torch.arange(n, device=dev)
        hidden = at[None] > (n - (hi - lo) + torch.arange(hi - lo, device=dev))[:, None]
        for h in range(case["heads"]):
            k, v = rows(s, ("kc", "ks"), at, h), rows(s, ("vc", "vs"), at, h)
            for j in range(h * g, h * g + g):
                p = torch.softmax((st["q"][lo:hi, j].double() @ k.t() / math.sqrt(d)).masked_fill_(hidden, -math.inf), 1)
                out[lo:hi, j] = p @ v
                if w is not None:
                    w[s, h, :n] += p.sum(0)
    return out if w is None else (out, w)


def _exact_norm(st, case):
    feat = st["feat"].long()
    h = st["x"].double() + (0 if st["res"] is None else st["res"].double())
    h16 = h.to(st["x"].dtype).double()
    y = h16 * st["gamma"].double() / torch.sqrt(h16.square().mean(1, keepdim=True) + EPS)
    w = st["w"].double()
    critical = torch.zeros(case["k"], dtype=torch.bool, device=y.device)
    critical[feat] = True

    def eight(v):
        v = v.masked_fill(critical, 0.0)
        top = v.abs().amax(1, keepdim=True)
        return torch.round(127 * v / torch.where(top == 0, 1.0, top)) * top / 127

    return eight(y) @ eight(w).t() + y[:, feat] @ w[:, feat].t(), h
