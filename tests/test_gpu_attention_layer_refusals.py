"""A refused call of the attention layer leaves everything as it was, whichever step of the call the refused argument belongs to."""
import numpy as np
import pytest
import torch

from paper_2407_19775_b200 import attention_layer
from paper_2407_19775_b200.binding import BqError
from test_gpu_attention_layer_shared import G, H, HD, HIDDEN, make

pytestmark = pytest.mark.gpu


def state(layer):
    tensors = [t for c in (layer.cache, layer.prefix) if c is not None for t in (*c._pools, c.lens)] + ([] if layer.weights is None else [layer.weights])
    return [t.clone() for t in tensors], (layer.longest, layer.prefix_longest)


def unchanged(layer, before, pools=True):
    now = state(layer)
    same = [torch.equal(a, b) for a, b in zip(now[0], before[0])]
    if not pools:                                                      # free slots may have been written
        same = [torch.equal(a, b) for a, b in zip(now[0], before[0]) if a.dim() == 1 or a.dtype == torch.float32]
    return all(same) and now[1] == before[1]


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("which", ["qkv_adapters", "out_adapters"])
@pytest.mark.parametrize("budget", [None, 6])
def test_ids_of_either_projection(bq, which, budget):
    layer = make(bq, torch.float16, budget=budget and 40)
    layer.budget, layer.sinks, layer.recent = budget, 1, 2
    setattr(layer, {"qkv_adapters": "out_adapters", "out_adapters": "qkv_adapters"}[which], None)
    x, pos = torch.randn(8, HIDDEN, device="cuda").half(), ints(*range(4))
    for i in range(8):
        layer(x[:4], positions=pos + i, ids=ints(0, 1, 2, -1))
    before = state(layer)
    starts = ints(0, 3, 5, 5, 8)
    for kw in (dict(ids=ints(0, 1, 2)), dict(ids=ints(0, 1, 2, 0).long()), dict(ids=ints(0, 1, 2, 0).cpu()), dict(ids=ints(0, 1, 2, 0, 1, 2)[::2]), dict(ids=ints(0, 1, 2, 0)[None]),
               dict(ids=ints(0, 1, 2, 0, 1), starts=starts), dict(ids=ints(0, 1, 2, 0), starts=starts.long()), dict(ids=ints(0, 1, 2, 0, 1), starts=ints(0, 1, 2, 3, 4, 4))):
        rows = 8 if "starts" in kw and kw["starts"].shape[0] == 5 else 4
        with pytest.raises(BqError):
            layer(x[:rows], positions=torch.arange(rows, dtype=torch.int32, device="cuda"), max_new=3, **kw)
        assert unchanged(layer, before)
    layer(x[:4], positions=pos, ids=ints(0, 1, 2, -1))


def test_members_and_prefixes(bq):
    """Known when the layer is made; members given later are refused by the attention, behind the store."""
    cb = bq.Codebook4()
    empty = bq.KvCache4.empty
    cache, prefix, members = empty(4, 64, H, HD, 32, cb), empty(2, 96, H, HD, 32, cb), ints(0, 2, 3)
    w = torch.zeros((H * G + 2 * H) * HD, HIDDEN, dtype=torch.float16, device="cuda")
    args = (w, torch.zeros(HIDDEN, H * G * HD, dtype=torch.float16, device="cuda"), torch.ones(HIDDEN, dtype=torch.float16, device="cuda"), H * G, H, cache)
    bad_members = (None, ints(0, 2), ints(0, 1, 2, 3), members.long(), members.cpu(), ints(0, 0, 2, 2, 3, 3)[::2])
    bad_prefixes = (empty(2, 96, 2 * H, HD, 32, cb), empty(2, 96, H, 2 * HD, 32, cb), empty(2, 96, H, HD, 64, cb), empty(2, 96, H, HD, 32, bq.Codebook4(bq.USER, np.linspace(-1, 1, 16, dtype=np.float32))))
    for kw in [dict(prefix=prefix, members=m) for m in bad_members] + [dict(prefix=p, members=members) for p in bad_prefixes]:
        with pytest.raises(BqError):
            attention_layer.AttentionLayer(*args, **kw)
    layer = make(bq, torch.float16, budget=40, adapters=False)
    x, pos = torch.randn(4, HIDDEN, device="cuda").half(), ints(*range(4))
    layer(x, positions=pos)
    before, good = state(layer), layer.members
    for m in bad_members:
        layer.members = m
        with pytest.raises(BqError):
            layer(x, positions=pos)
        assert unchanged(layer, before, pools=False)
    layer.members = good
    y, _ = layer(x, positions=pos)
    assert layer.cache.lens.tolist() == [2] * 4 and layer.longest == 2 and bool(torch.isfinite(y).all())


def test_adapters_of_another_layer(bq):
    layer = make(bq, torch.float16)
    good = layer.qkv_adapters, layer.out_adapters
    assert good[0].N != good[1].N
    for name, other in (("qkv_adapters", good[1]), ("out_adapters", good[0])):
        with pytest.raises(BqError):
            setattr(layer, name, other)
    assert (layer.qkv_adapters, layer.out_adapters) == good


def test_arguments_of_the_attention(bq):
    """max_new is first looked at by the attention; the bounds on lens are as before, so that a captured call still finds room."""
    for prefix in (True, False):
        layer = make(bq, torch.float16, prefix=prefix, adapters=False, capacity=64)
        x, pos, starts = torch.randn(4, HIDDEN, device="cuda").half(), ints(*range(4)), ints(*range(5))
        layer(x, positions=pos)
        before = state(layer)
        for _ in range(70):                                            # more often than the cache has slots
            with pytest.raises(BqError):
                layer(x, positions=pos, starts=starts, max_new=-1)
            with pytest.raises(BqError):
                layer(x, positions=pos[:3])
        assert unchanged(layer, before, pools=False)
        if prefix:
            for _ in range(100):
                with pytest.raises(BqError):
                    layer.begin(x[:2], None, ints(0, 1, 2), -1)
                with pytest.raises(BqError):
                    layer.begin(x[:2], None, ints(0, 1, 2), 1, positions=pos[:3])
            assert unchanged(layer, before, pools=False)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer(x, positions=pos)
