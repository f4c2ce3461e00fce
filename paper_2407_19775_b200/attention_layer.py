"""The attention half of a transformer layer on compressed operands: weights in 8 bits, keys and values in 4.

    residual + x -> rms norm -> query/key/value projection      DecomposedLinear.norm_linear
    new keys and values into the cache                          KvCache4.append, append_rotary
    causal attention over it, slot weights accumulated          KvCache4.attend, attend_shared
    sequences over their budget lose their lightest slots       KvCache4.evict
    output projection                                           DecomposedLinear.linear

Queries and keys turn by their positions where the layer has a Rotary; sequences that begin alike share the rows of a prefix
cache; each sequence may have low-rank adapters of its own beside both projections.

    python -m paper_2407_19775_b200.attention_layer --sequences 8 --prompt 700 --steps 64 --budget 512 --positions --prefix 1000 --adapters 3

draws a layer, feeds it prompts of different lengths and then single tokens, and prints the time of both and the cache's size.
"""
from __future__ import annotations

import argparse

import torch

from .binding import BqError
from .bq4 import Codebook4
from .kvcache import KvCache4, Rotary
from .mmd import Adapters, DecomposedLinear


class AttentionLayer:
    """One layer's attention for a fixed set of sequences.  w_qkv: [(q_heads + 2 kv_heads) * head_dim, hidden]; w_out: [hidden,
    q_heads * head_dim]; gamma: [hidden]; all of one 16-bit type, on the GPU.  ``budget``: the slots that a sequence keeps
    after each call (None: all of them), ``sinks`` and ``recent`` among them whatever their weight.

    ``rotary``: how queries and keys turn by their positions (None: not at all).  ``prefix``: a cache whose sequences are beginnings that
    the layer's sequences share, ``members`` as for KvCache4.attend_shared; begin() runs rows into it, and it is never evicted from.
    ``qkv_adapters``, ``out_adapters``: the Adapters of the two projections (either may be None).

    A call whose rows the cache has no room for is refused; a refused call leaves lens, weights and bounds as they were.  ``longest`` is the host's bound on the cache's lens: it is kept
    without asking the device, and replaced by what the device holds (which waits for it) only where it no longer shows that the
    rows fit (``prefix_longest`` likewise for the prefix).  Whoever raises lens by other means, or replays a captured call of a layer
    without a budget, sets it to None.  (A call that is being captured is refused unless a call before it has shown that there is
    room, up to the budget if there is one.)"""

    def __init__(self, w_qkv, w_out, gamma, q_heads: int, kv_heads: int, cache: KvCache4, features=(), out_features=(), eps: float = 1e-5,
                 budget: int | None = None, sinks: int = 4, recent: int = 32, rotary: Rotary | None = None, prefix: KvCache4 | None = None,
                 members: torch.Tensor | None = None, qkv_adapters: Adapters | None = None, out_adapters: Adapters | None = None):
        if budget is not None and (min(budget - 1, sinks, recent) < 0 or sinks + recent > budget):
            raise BqError(f"a budget of {budget} slots has no room for {sinks} first and {recent} last ones")
        if rotary is not None and rotary.dim > cache.head_dim:
            raise BqError(f"{rotary.dim} elements of a row of {cache.head_dim} cannot turn")
        if prefix is not None:
            cache.check_prefix(prefix, members)
        elif members is not None:
            raise BqError("members without a prefix")
        self.qkv, self.out = DecomposedLinear(w_qkv, features), DecomposedLinear(w_out, out_features)
        self.gamma, self.eps, self.cache = gamma, eps, cache
        self.q_heads, self.kv_heads = q_heads, kv_heads
        self.budget, self.sinks, self.recent = budget, sinks, recent
        self.rotary, self.prefix, self.members = rotary, prefix, members
        self._adapters: tuple[Adapters | None, Adapters | None] = (None, None)
        self.qkv_adapters, self.out_adapters = qkv_adapters, out_adapters
        self.longest: int | None = None
        self.prefix_longest: int | None = None
        self.weights = None
        if budget is not None:
            self.weights = torch.zeros(cache.n_seq, kv_heads, cache.capacity, device=cache.device)

    @property
    def qkv_adapters(self) -> Adapters | None:
        return self._adapters[0]

    @qkv_adapters.setter
    def qkv_adapters(self, adapters: Adapters | None) -> None:
        if adapters is not None:
            self.qkv.check_adapters(adapters)
        self._adapters = (adapters, self._adapters[1])

    @property
    def out_adapters(self) -> Adapters | None:
        return self._adapters[1]

    @out_adapters.setter
    def out_adapters(self, adapters: Adapters | None) -> None:
        if adapters is not None:
            self.out.check_adapters(adapters)
        self._adapters = (self._adapters[0], adapters)

    @staticmethod
    def _count(c: KvCache4, longest: int | None, budget: int | None, n: int, starts: torch.Tensor | None, max_new: int) -> int:
        """Counts the new rows into lens, or refuses them before anything has changed; the new bound on lens."""
        news = 1 if starts is None else starts[1:] - starts[:-1]
        # a max_new that cannot be a bound (more rows than it allows) is replaced by one that is
        most = 1 if starts is None else max_new if max_new * c.n_seq >= n else n
        capturing = torch.cuda.is_current_stream_capturing()
        # a captured call is replayed until its sequences have reached the budget
        known = longest if not capturing or budget is None else longest and max(longest, budget)
        if known is None or known + most > c.capacity:
            if capturing:
                raise BqError("the cache is not known to have room for the rows, which cannot be found out during a capture")
            longest = int((c.lens + news).max())
            if longest > c.capacity:
                raise BqError(f"a sequence would hold {longest} slots of {c.capacity}")
        else:
            longest = longest + most
        c.lens.add_(news)
        return longest if budget is None else min(longest, budget)

    def _stored(self, c: KvCache4, x, residual, starts, positions, adapted: dict, attend):
        """(attend(queries), x + residual) of the rows, whose keys and values go into the cache; their sequences have been counted into
        lens, which is taken back where a step is refused (what it has stored by then lies in slots that are free again)."""
        n, hd = x.shape[0], c.head_dim
        try:
            qkv, h = self.qkv.norm_linear(x, self.gamma, self.eps, residual=residual, **adapted)
            q, k, v = qkv.view(n, self.q_heads + 2 * self.kv_heads, hd).split((self.q_heads, self.kv_heads, self.kv_heads), dim=1)      # slices, taken as they are
            if self.rotary is None:
                c.append(k, v, starts)
            else:
                q = c.append_rotary(q, k, v, self.rotary, positions, starts, q)       # in place
            return attend(q), h
        except Exception:
            c.lens.sub_(1 if starts is None else starts[1:] - starts[:-1])
            raise

    def _check_call(self, c: KvCache4, positions, ids, starts, n: int) -> None:
        c.check_starts(starts, n)
        if positions is not None and self.rotary is None:
            raise BqError("positions without a rotary")
        if ids is not None:
            if self.qkv_adapters is None and self.out_adapters is None:
                raise BqError("ids without adapters")
            self.out.check_ids(ids, starts, n)                         # whichever projection takes them

    def __call__(self, x: torch.Tensor, residual: torch.Tensor | None = None, starts: torch.Tensor | None = None, max_new: int = 1, max_len: int = 0,
                 positions: torch.Tensor | None = None, ids: torch.Tensor | None = None):
        """x: [rows, hidden], the new rows of all sequences, sequence s's at starts[s] .. starts[s + 1] (None: one row each).
        Returns (the projected attention, x + residual).  ``max_new`` and ``max_len`` bound the rows and slots of a sequence.
        ``positions``: of the rows, as for KvCache4.append_rotary (None: their places in the cache, which a layer with a budget or a
        prefix cannot tell).  ``ids``: the sequences' adapters (-1: none; None: none at all)."""
        c, n, hd = self.cache, x.shape[0], self.cache.head_dim
        self._check_call(c, positions, ids, starts, n)
        if self.rotary is not None and positions is None and (self.budget is not None or self.prefix is not None):
            raise BqError("rows of a bounded cache, or behind a prefix, need their positions")
        adapted = [dict(adapters=a, ids=ids, starts=starts) if a is not None and ids is not None else {} for a in self._adapters]
        longest = self._count(c, self.longest, self.budget, n, starts, max_new)

        def attend(q):
            if self.prefix is None:
                return c.attend(q, starts, max_new, max_len, weights=self.weights)
            return c.attend_shared(q, self.prefix, self.members, starts, max_new, max_len, max_prefix=self.prefix_longest or 0, weights=self.weights)

        a, h = self._stored(c, x, residual, starts, positions, adapted[0], attend)
        self.longest = longest
        if self.budget is not None:
            c.evict(self.weights, self.budget, self.sinks, self.recent)
            self.weights[:, :, self.budget:].zero_()                   # of slots that are free again
        return self.out.linear(a.view(n, self.q_heads * hd), **adapted[1]), h

    def begin(self, x: torch.Tensor, residual: torch.Tensor | None = None, starts: torch.Tensor | None = None, max_new: int = 1, max_len: int = 0,
              positions: torch.Tensor | None = None):
        """The same for rows of the prefixes, sequence s of ``starts`` the s-th: into the prefix cache, whose rows all its sequences
        share, so without adapters.  Positions default to the rows' places."""
        if self.prefix is None:
            raise BqError("the layer has no prefix")
        c, n, hd = self.prefix, x.shape[0], self.prefix.head_dim
        self._check_call(c, positions, None, starts, n)
        longest = self._count(c, self.prefix_longest, None, n, starts, max_new)
        a, h = self._stored(c, x, residual, starts, positions, {}, lambda q: c.attend(q, starts, max_new, max_len))
        self.prefix_longest = longest
        return self.out.linear(a.view(n, self.q_heads * hd)), h


def random_layer(sequences: int, capacity: int, hidden: int, q_heads: int, kv_heads: int, head_dim: int, block: int, dtype, seed: int = 0, **kw) -> AttentionLayer:
    g = torch.Generator().manual_seed(seed)
    draw = lambda *shape, s: (torch.randn(*shape, generator=g) * s).to(dtype).cuda()
    w_qkv = draw((q_heads + 2 * kv_heads) * head_dim, hidden, s=hidden ** -0.5)
    w_out = draw(hidden, q_heads * head_dim, s=(q_heads * head_dim) ** -0.5)
    gamma = draw(hidden, s=0.1) + 1
    cache = KvCache4.empty(sequences, capacity, kv_heads, head_dim, block, Codebook4())
    return AttentionLayer(w_qkv, w_out, gamma, q_heads, kv_heads, cache, **kw)


def random_adapters(layer: DecomposedLinear, count: int, rank: int, seed: int = 0) -> Adapters:
    g = torch.Generator().manual_seed(seed)
    draw = lambda *shape, s: (torch.randn(*shape, generator=g) * s).to(layer.dtype).to(layer.device)
    return Adapters(draw(count, rank, layer.K, s=layer.K ** -0.5), draw(count, layer.N, rank, s=0.1), torch.ones(count, device=layer.device))


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=700, help="tokens of the longest prompt")
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--budget", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--q-heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--positions", action="store_true", help="turn queries and keys by their positions")
    ap.add_argument("--prefix", type=int, default=0, help="tokens that all sequences begin with")
    ap.add_argument("--adapters", type=int, default=0, help="low-rank adapters, dealt out to the sequences")
    a = ap.parse_args()
    dtype, hd = torch.bfloat16, 128
    kw = dict(rotary=Rotary(hd)) if a.positions else {}
    if a.prefix:
        kw["prefix"] = KvCache4.empty(1, a.prefix, a.kv_heads, hd, 64, Codebook4())
    layer = random_layer(a.sequences, a.prompt + max(a.steps, 64), a.hidden, a.q_heads, a.kv_heads, hd, 64, dtype, budget=a.budget, **kw)
    ids = None
    if a.adapters:
        layer.qkv_adapters, layer.out_adapters = (random_adapters(w, a.adapters, 16) for w in (layer.qkv, layer.out))
        ids = torch.arange(a.sequences, dtype=torch.int32, device="cuda") % a.adapters
    if a.prefix:
        layer.begin(torch.randn(a.prefix, a.hidden, device="cuda").to(dtype), None, torch.tensor([0, a.prefix], dtype=torch.int32, device="cuda"), a.prefix)
    news = [max(1, a.prompt - 37 * s) for s in range(a.sequences)]
    starts = torch.tensor([0] + news).cumsum(0).int().cuda()
    x = torch.randn(sum(news), a.hidden, device="cuda").to(dtype)
    at = lambda first, n: torch.cat([torch.arange(f, f + m, dtype=torch.int32) for f, m in zip(first, n)]).cuda() if a.positions else None
    pos = at([a.prefix] * a.sequences, news)
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    marks[0].record()
    y, h = layer(x, None, starts, max(news), max(news), positions=pos, ids=ids)
    marks[1].record()
    x, residual = y[starts[1:].long() - 1], h[starts[1:].long() - 1]
    pos = at([a.prefix + n for n in news], [1] * a.sequences)
    for _ in range(a.steps):
        x, residual = layer(x, residual, max_len=max(max(news), a.budget + 1), positions=pos, ids=ids)
        pos = pos + 1 if a.positions else None
    marks[2].record()
    torch.cuda.synchronize()
    c = layer.cache
    held = int(c.lens.sum()) * a.kv_heads * (hd + 2 * 2 * hd // c.block)
    print("prompts of %d tokens: %.2f ms; a step of %d sequences: %.1f us; slots %s; %.2f MB held (16 bits: %.2f)" %
          (sum(news), marks[0].elapsed_time(marks[1]), a.sequences, marks[1].elapsed_time(marks[2]) / max(a.steps, 1) * 1e3,
           c.lens.tolist(), held / 1e6, int(c.lens.sum()) * a.kv_heads * hd * 4 / 1e6))


if __name__ == "__main__":
    main()
