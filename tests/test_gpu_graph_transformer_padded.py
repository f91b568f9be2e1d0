"""The graph transformer path on a batch that is filled up: nodes behind the graphs are one more graph, masked, without ids."""
import pytest
import torch

from paper_2412_12218_amd.models import GraphTransformerPath
from test_gpu_graph_transformer import D, HEADS, HIDDEN, KV, LAYERS, OUT, TOL, VOCAB, batch, flat, reference, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TOL))
def test_padded_batch(dtype):
    lens, n, ptr, ids, mask, d_out = batch(dtype, lens=(5, 0, 40, 1, 64, 90, 56))
    ids[-56:], mask[-56:], d_out[-56:] = -1, 0, 0
    w = weights(dtype)
    path = GraphTransformerPath(ptr, n, VOCAB, D, HEADS, KV, HIDDEN, OUT, LAYERS, act_dtype=dtype)
    want, want_grads = reference(lens, ids, w, mask, d_out)
    logits = path.forward(ids, w, mask=mask)
    grads = flat(path.backward(ids, w, d_out, mask=mask))
    off = lambda a, b: float((a.cpu().double() - b).norm() / b.norm())
    errors = [off(logits, want)] + [off(a, b) for a, b in zip(grads, want_grads)]
    assert max(errors) < TOL[dtype]
    # features of the padded places that were never written reach no other node
    path.h[0].fill_(float("nan"))
    path.qkv[0].fill_(float("nan"))
    again = path.forward(ids, w, mask=mask).clone()
    assert torch.equal(again, logits)
