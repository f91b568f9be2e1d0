"""Calls around the blocks of a graph transformer that the host decides by itself: how lists of gradients are given, and which node types a path takes.  CPU only."""
import pytest
import torch

from paper_2412_12218_amd import binding as B
from paper_2412_12218_amd.models import GraphTransformerPath


def test_gradients_from_an_iterator():
    """What a program writes as (p.grad for p in parameters): each of them is there once, and its own output."""
    grads = [torch.arange(6.0), torch.zeros(2, 3), torch.ones(4).half()]
    for given in ((g for g in grads), iter(grads), tuple(grads), map(lambda g: g, grads)):
        listed = B.GradList(given)
        assert [g.grad for g in listed.c] == [g.out for g in listed.c] == [g.data_ptr() for g in grads]
        assert all(a is b for a, b in zip(listed.grads, grads)) and len(listed.out) == 3
    outs = [torch.empty_like(g) for g in grads]
    listed = B.GradList((g for g in grads), out=(o for o in outs))
    assert [g.grad for g in listed.c] == [g.data_ptr() for g in grads] and [g.out for g in listed.c] == [o.data_ptr() for o in outs]


def test_node_types_that_a_path_takes(monkeypatch):
    """The order of the types is computed from their memory, as 32-bit numbers one behind the other on the device of the batch; anything else would be read as other
    types, or beyond its end."""
    n, calls = 6, []

    def order(keys, ws=None):
        calls.append(keys)
        perm = torch.sort(keys, stable=True).indices.int()
        return perm, torch.argsort(perm).int(), None
    monkeypatch.setattr(B, "ftc_order_by_key", order)
    good = torch.tensor([2, 0, 1, 1, 0, 2], dtype=torch.int32)
    make = lambda types: GraphTransformerPath(torch.tensor([0, n], dtype=torch.int32), n, 10, d=8, heads=2, types=types, n_types=3)
    path = make(good)
    assert path.group_ptr.tolist() == [0, 2, 4, 6] and good[path.perm.long()].tolist() == [0, 0, 1, 1, 2, 2] and len(calls) == 1
    for bad in (good.long(), good.short(), good.to(torch.uint8), good.float(), good.repeat_interleave(2)[::2], good[:-1], good.view(2, 3), good.to("meta"), good - 1, good + 1):
        with pytest.raises(ValueError):
            make(bad)
    assert len(calls) == 1
