"""Calls around the blocks of a graph transformer that the host decides by itself: how lists of gradients are given, and which node types a path takes.  CPU only."""
import torch

from paper_2412_12218_amd import binding as B


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
