"""What the graph transformer's entry points refuse beyond test_graph_transformer_host.py.  CPU only."""
import pytest
import torch

from paper_2412_12218_amd import binding as B
from paper_2412_12218_amd.models import GraphTransformerPath
from test_graph_transformer_host import INVALID, attention, attention_backward


@pytest.mark.parametrize("call", [attention, attention_backward])
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf")])
def test_scales_that_are_not_finite(call, scale):
    assert call(scale=scale) == INVALID
    assert b"scale" in B.lib().ftc_last_error()


@pytest.mark.parametrize("layers", [0, 1, 3])
def test_path_with_weights_of_another_number_of_layers(layers):
    """The head reads the output of the path's last layer, which would be that of an earlier pass."""
    path = GraphTransformerPath(torch.tensor([0, 4], dtype=torch.int32), 4, 10, d=16, heads=2, layers=2)
    weights = dict(table=None, head=None, head_bias=None, layers=[{}] * layers)
    ids = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="2 layers"):
        path.forward(ids, weights)
    with pytest.raises(ValueError, match="2 layers"):
        path.backward(ids, weights, torch.zeros((4, 8)))
