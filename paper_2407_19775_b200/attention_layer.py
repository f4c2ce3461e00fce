"""The attention half of a transformer layer without positions on compressed operands: weights in 8 bits, keys and values in 4.

    residual + x -> rms norm -> query/key/value projection      DecomposedLinear.norm_linear
    new keys and values into the cache                          KvCache4.append
    causal attention over it, slot weights accumulated          KvCache4.attend
    sequences over their budget lose their lightest slots       KvCache4.evict
    output projection                                           DecomposedLinear.linear

Nothing happens to queries and keys between their projection and the cache: a model that turns them by their position calls the
same operators and does so in between.

    python -m paper_2407_19775_b200.attention_layer --sequences 8 --prompt 700 --steps 64 --budget 512

draws a layer, feeds it prompts of different lengths and then single tokens, and prints the time of both and the cache's size.
"""
from __future__ import annotations

import argparse

import torch

from .binding import BqError
from .bq4 import Codebook4
from .kvcache import KvCache4
from .mmd import DecomposedLinear


class AttentionLayer:
    """One layer's attention for a fixed set of sequences.  w_qkv: [(q_heads + 2 kv_heads) * head_dim, hidden]; w_out: [hidden,
    q_heads * head_dim]; gamma: [hidden]; all of one 16-bit type, on the GPU.  ``budget``: the slots that a sequence keeps
    after each call (None: all of them), ``sinks`` and ``recent`` among them whatever their weight.

    A call whose rows the cache has no room for is refused.  ``longest`` is the host's bound on the cache's lens: it is kept
    without asking the device, and replaced by what the device holds (which waits for it) only where it no longer shows that the
    rows fit.  Whoever raises lens by other means, or replays a captured call of a layer without a budget, sets it to None.  (A
    call that is being captured is refused unless a call before it has shown that there is room, up to the budget if there is one.)"""

    def __init__(self, w_qkv, w_out, gamma, q_heads: int, kv_heads: int, cache: KvCache4, features=(), out_features=(), eps: float = 1e-5,
                 budget: int | None = None, sinks: int = 4, recent: int = 32):
        if budget is not None and (min(budget - 1, sinks, recent) < 0 or sinks + recent > budget):
            raise BqError(f"a budget of {budget} slots has no room for {sinks} first and {recent} last ones")
        self.qkv, self.out = DecomposedLinear(w_qkv, features), DecomposedLinear(w_out, out_features)
        self.gamma, self.eps, self.cache = gamma, eps, cache
        self.q_heads, self.kv_heads = q_heads, kv_heads
        self.budget, self.sinks, self.recent = budget, sinks, recent
        self.longest: int | None = None
        self.weights = None
        if budget is not None:
            self.weights = torch.zeros(cache.n_seq, kv_heads, cache.capacity, device=cache.device)

    def _count(self, n: int, starts: torch.Tensor | None, max_new: int) -> None:
        """Counts the new rows into lens, or refuses them before anything has changed."""
        c = self.cache
        news = 1 if starts is None else starts[1:] - starts[:-1]
        # a max_new that cannot be a bound (more rows than it allows) is replaced by one that is
        most = 1 if starts is None else max_new if max_new * c.n_seq >= n else n
        capturing = torch.cuda.is_current_stream_capturing()
        # a captured call is replayed until its sequences have reached the budget
        known = self.longest if not capturing or self.budget is None else self.longest and max(self.longest, self.budget)
        if known is None or known + most > c.capacity:
            if capturing:
                raise BqError("the cache is not known to have room for the rows, which cannot be found out during a capture")
            longest = int((c.lens + news).max())
            if longest > c.capacity:
                raise BqError(f"a sequence would hold {longest} slots of {c.capacity}")
        else:
            longest = self.longest + most
        c.lens.add_(news)
        self.longest = longest if self.budget is None else min(longest, self.budget)

    def __call__(self, x: torch.Tensor, residual: torch.Tensor | None = None, starts: torch.Tensor | None = None, max_new: int = 1, max_len: int = 0):
        """x: [rows, hidden], the new rows of all sequences, sequence s's at starts[s] .. starts[s + 1] (None: one row each).
        Returns (the projected attention, x + residual).  ``max_new`` and ``max_len`` bound the rows and slots of a sequence."""
        c, n, hd = self.cache, x.shape[0], self.cache.head_dim
        self._count(n, starts, max_new)
        qkv, h = self.qkv.norm_linear(x, self.gamma, self.eps, residual=residual)
        q, k, v = qkv.view(n, self.q_heads + 2 * self.kv_heads, hd).split((self.q_heads, self.kv_heads, self.kv_heads), dim=1)      # slices, taken as they are
        c.append(k, v, starts)
        a = c.attend(q, starts, max_new, max_len, weights=self.weights)
        if self.budget is not None:
            c.evict(self.weights, self.budget, self.sinks, self.recent)
            self.weights[:, :, self.budget:].zero_()                   # of slots that are free again
        return self.out.linear(a.view(n, self.q_heads * hd)), h


def random_layer(sequences: int, capacity: int, hidden: int, q_heads: int, kv_heads: int, head_dim: int, block: int, dtype, seed: int = 0, **kw) -> AttentionLayer:
    g = torch.Generator().manual_seed(seed)
    draw = lambda *shape, s: (torch.randn(*shape, generator=g) * s).to(dtype).cuda()
    w_qkv = draw((q_heads + 2 * kv_heads) * head_dim, hidden, s=hidden ** -0.5)
    w_out = draw(hidden, q_heads * head_dim, s=(q_heads * head_dim) ** -0.5)
    gamma = draw(hidden, s=0.1) + 1
    cache = KvCache4.empty(sequences, capacity, kv_heads, head_dim, block, Codebook4())
    return AttentionLayer(w_qkv, w_out, gamma, q_heads, kv_heads, cache, **kw)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=700, help="tokens of the longest prompt")
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--budget", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--q-heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    a = ap.parse_args()
    dtype, hd = torch.bfloat16, 128
    layer = random_layer(a.sequences, a.prompt + max(a.steps, 64), a.hidden, a.q_heads, a.kv_heads, hd, 64, dtype, budget=a.budget)
    news = [max(1, a.prompt - 37 * s) for s in range(a.sequences)]
    starts = torch.tensor([0] + news).cumsum(0).int().cuda()
    x = torch.randn(sum(news), a.hidden, device="cuda").to(dtype)
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    marks[0].record()
    y, h = layer(x, None, starts, max(news), max(news))
    marks[1].record()
    x, residual = y[starts[1:].long() - 1], h[starts[1:].long() - 1]
    for _ in range(a.steps):
        x, residual = layer(x, residual, max_len=max(max(news), a.budget + 1))
    marks[2].record()
    torch.cuda.synchronize()
    c = layer.cache
    held = int(c.lens.sum()) * a.kv_heads * (hd + 2 * 2 * hd // c.block)
    print("prompts of %d tokens: %.2f ms; a step of %d sequences: %.1f us; slots %s; %.2f MB held (16 bits: %.2f)" %
          (sum(news), marks[0].elapsed_time(marks[1]), a.sequences, marks[1].elapsed_time(marks[2]) / max(a.steps, 1) * 1e3,
           c.lens.tolist(), held / 1e6, int(c.lens.sum()) * a.kv_heads * hd * 4 / 1e6))


if __name__ == "__main__":
    main()
