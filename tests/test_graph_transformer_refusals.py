"""What the graph transformer's entry points refuse beyond test_graph_transformer_host.py.  CPU only."""
import pytest

from paper_2412_12218_amd import binding as B
from test_graph_transformer_host import INVALID, attention, attention_backward


@pytest.mark.parametrize("call", [attention, attention_backward])
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf")])
def test_scales_that_are_not_finite(call, scale):
    assert call(scale=scale) == INVALID
    assert b"scale" in B.lib().ftc_last_error()
