"""GPU tests of the attention layer at the edges of its cache."""
import pytest
import torch

from paper_2407_19775_b200 import attention_layer
from paper_2407_19775_b200.binding import BqError

pytestmark = pytest.mark.gpu


def make(budget=None):
    return attention_layer.random_layer(2, 64, 256, 4, 2, 64, 64, torch.float16, budget=budget)      # one page of 64 slots per sequence


def rows(n):
    return torch.randn(n, 256, device="cuda").to(torch.float16)


def test_rows_that_do_not_fit_are_refused(bq):
    """Single tokens up to the last slot, then no more; prompts likewise; what is refused changes nothing."""
    layer = make()
    starts = torch.tensor([0, 61, 64], dtype=torch.int32, device="cuda")
    layer(rows(64), None, starts, 61)
    for _ in range(3):
        layer(rows(2))
    assert layer.cache.lens.tolist() == [64, 6]
    before = [p.clone() for p in layer.cache._pools]
    for call in (lambda: layer(rows(2)), lambda: layer(rows(3), None, torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda"), 2),
                 lambda: layer(rows(3), None, torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda"))):
        with pytest.raises(BqError):
            call()
    assert layer.cache.lens.tolist() == [64, 6]
    assert all(torch.equal(a, b) for a, b in zip(layer.cache._pools, before))
    layer(rows(58), None, torch.tensor([0, 0, 58], dtype=torch.int32, device="cuda"), 58)      # only the sequence with room grows
    assert layer.cache.lens.tolist() == [64, 64]
    layer.cache.lens.zero_()                                         # sequences that end free their slots
    layer(rows(2))
    assert layer.cache.lens.tolist() == [1, 1]
    with pytest.raises(BqError):                                     # a max_new that does not hold is no excuse
        layer(rows(65), None, torch.tensor([0, 64, 65], dtype=torch.int32, device="cuda"))


def test_a_budget_keeps_room(bq):
    layer = make(budget=40)
    layer(rows(60), None, torch.tensor([0, 50, 60], dtype=torch.int32, device="cuda"), 50)
    for _ in range(70):
        y, _ = layer(rows(2))
    assert layer.cache.lens.tolist() == [40, 40] and bool(torch.isfinite(y).all())
    with pytest.raises(BqError):
        layer(rows(30), None, torch.tensor([0, 25, 30], dtype=torch.int32, device="cuda"), 25)


def test_a_call_without_rows(bq):
    """No new rows in any sequence: empty results, and the cache as it was."""
    for budget in (None, 40):
        layer = make(budget)
        none = torch.zeros(3, dtype=torch.int32, device="cuda")
        y, h = layer(rows(0), None, none)
        assert y.shape == (0, 256) and h.shape == (0, 256) and layer.cache.lens.tolist() == [0, 0]
        layer(rows(2))
        y, h = layer(rows(0), rows(0), none)
        assert y.shape == (0, 256) and h.shape == (0, 256) and layer.cache.lens.tolist() == [1, 1]


def test_captured_steps(bq):
    """A step captured early is replayed until the sequences are at their budget, and beyond; it is refused where they would not fit
    then."""
    for budget, fits in ((40, True), (63, True), (64, False), (None, True)):
        layer = make(budget)
        x, s = rows(2), torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            with pytest.raises(BqError):                             # nothing is known of the cache yet
                with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
                    layer(x)
            layer(x)
            s.synchronize()
            if not fits:
                with pytest.raises(BqError):
                    with torch.cuda.graph(graph, stream=s):
                        layer(x)
                continue
            with torch.cuda.graph(graph, stream=s):
                y, _ = layer(x)
            for _ in range(80 if budget else 60):
                graph.replay()
            s.synchronize()
            assert layer.cache.lens.tolist() == [budget or 61] * 2 and bool(torch.isfinite(y).all())
            if budget is None:
                layer.longest = None                                 # the replays went unseen
                for _ in range(3):
                    layer(x)
                with pytest.raises(BqError):
                    layer(x)
                assert layer.cache.lens.tolist() == [64, 64]


def test_budgets_that_hold_less_than_they_have_to_keep(bq):
    """Refused when the layer is made, not after the first call has stored its rows."""
    for args in (dict(budget=16), dict(budget=0, sinks=0, recent=0), dict(budget=8, sinks=-1, recent=2), dict(budget=8, sinks=5, recent=4)):
        with pytest.raises(BqError):
            attention_layer.random_layer(2, 64, 256, 4, 2, 64, 64, torch.float16, **args)
    layer = attention_layer.random_layer(2, 64, 256, 4, 2, 64, 64, torch.float16, budget=9, sinks=5, recent=4)
    for _ in range(12):
        layer(rows(2))
    assert layer.cache.lens.tolist() == [9, 9]
